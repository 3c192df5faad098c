// The LM head in 8-bit floating point (e4m3) with one scale for each block of 128.
//
//   z[n][v] = sum_kb 2^(ex[n][kb] + ew[v / 128][kb]) sum_{k in kb} qx[n][k] qw[v][k]
//
// A block is 128 columns of one row of X, or 128 ids x 128 columns of W; its scale is the least
// power of two 2^e with max |x| <= 448 * 2^e, kept as the byte e + 127 (E8M0; 255: the block holds an
// infinity or a NaN, and every logit it enters is NaN). Scaling by a power of two is exact, so each
// value is rounded once, to the nearest code (ties to even).
//
// The products run on the bf16 matrix instructions: a code has four significant bits and its scale is a
// power of two, so bf16 holds its value exactly, and the sums are fp32 sums. The 8-bit matrix
// instructions (v_mfma_f32_16x16x128_f8f6f4, v_mfma_f32_16x16x32_fp8_fp8) are not used, as what they give are
// not fp32 sums: they align the products of one instruction to the largest and keep 9 to 13 bits below it
// (128 normal values: errors up to 2^-13 of the largest product, 1.5e-5 in the 2-norm against the 1e-7 of
// these kernels; values over twelve binades: 6.4e-5).
//
// What 8 bits buy is the weight's stream, which bounds the product up to a few hundred rows: W
// goes to LDS as codes, half of K1's bytes, and each fragment is widened in registers by
// v_cvt_scalef32_pk_bf16_fp8 (two values an instruction, the scale included) while the matrix unit
// runs. The rounded X is small and is written once as bf16 (K12 k_round_rows); the rest is K1's: its tile
// shapes, its epilogue (lmhead_block), or the logits stored (k_lmhead_logits).
//
// Whole calls at H = 4096, against the same step on the packed bf16 weight: 60 rows at V = 128256 87 us
// against 157 (the weight's read at 7.1 TB/s: 74), 2048 rows 1540 against 1520: there the matrix unit, the
// widening beside it and the power cap bound both, at 1.40 PFLOP/s.
#pragma once

#include "k_lmhead.h"

namespace asv {

constexpr int kQBlock = 128;          // columns (and ids of W) of one scale

__host__ __device__ __forceinline__ int q8_blocks(int H) { return (H + kQBlock - 1) / kQBlock; }
// scale bytes of a row of blocks: whole 32-bit words
__host__ __device__ __forceinline__ int q8_pitch(int H) { return (q8_blocks(H) + 3) / 4 * 4; }

// E8M0 byte of a block whose largest |bf16| has the bits `a` (sign cleared): 448 = 1.75 * 2^8.
__host__ __device__ __forceinline__ int q8_scale(int a) {
  const int e = a >> 7;
  if (e == 255) return 255;
  const int s = e - 8 + ((a & 127) > 96 ? 1 : 0);
  return s < 1 ? 1 : s;
}
// 2^(127 - s), which a block with scale byte s is multiplied by; NaN for 255.
__device__ __forceinline__ float q8_factor(int s) {
  return __int_as_float(s == 255 ? 0x7fc00000 : (254 - s) << 23);
}
// 2^(s - 127); NaN for 255.
__device__ __forceinline__ float q8_step(int s) {
  return __int_as_float(s == 255 ? 0x7fc00000 : s << 23);
}

__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
// Four codes of f * the bf16 pairs p, q.
__device__ __forceinline__ uint32_t q8_codes(uint32_t p, uint32_t q, float f) {
  const int r = __builtin_amdgcn_cvt_pk_fp8_f32(bf16_lo(p) * f, bf16_hi(p) * f, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(bf16_lo(q) * f, bf16_hi(q) * f, r, true);
}
// Two codes (half `HI` of c) times step, as a bf16 pair: every such value is a bf16 value, but for those
// below 2^-126, where step's smallest is left.
template <bool HI>
__device__ __forceinline__ uint32_t q8_value_pair(uint32_t c, float step) {
  return __builtin_bit_cast(uint32_t,
                            __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c, step, HI));
}
__device__ __forceinline__ int max_abs_bf16(uint32_t p) {
  return max((int)(p & 0x7fff), (int)((p >> 16) & 0x7fff));
}
__device__ __forceinline__ int max_abs_bf16(const uint4& x) {
  return max(max(max_abs_bf16(x.x), max_abs_bf16(x.y)),
             max(max_abs_bf16(x.z), max_abs_bf16(x.w)));
}

constexpr int kRoundThreads = 256;
constexpr int kRoundCols = kRoundThreads * 8;

// K12. Grid (rows, ceil(H / kRoundCols)): eight columns a thread, a block per 16 lanes. X bf16 [N][H] from the
// launch's first row on, out the values that its codes and scales stand for, bf16 [N][H]. A launch has fewer
// than 2^32 threads along x, so at most kRoundRows rows.
constexpr int kRoundRows = 1 << 23;

static __global__ __launch_bounds__(kRoundThreads)
void k_round_rows(const uint16_t* __restrict__ X, int H, uint16_t* __restrict__ out) {
  const int col = blockIdx.y * kRoundCols + threadIdx.x * 8;
  const size_t at = (size_t)blockIdx.x * H + col;
  uint4 x = make_uint4(0u, 0u, 0u, 0u);
  if (col < H) x = *reinterpret_cast<const uint4*>(X + at);
  int a = max_abs_bf16(x);
  a = max(a, row_ror<8>(a));
  a = max(a, row_ror<4>(a));
  a = max(a, row_ror<2>(a));
  a = max(a, row_ror<1>(a));
  if (col >= H) return;
  const int s = q8_scale(a);
  const float f = q8_factor(s), step = q8_step(s);
  const uint32_t c0 = q8_codes(x.x, x.y, f), c1 = q8_codes(x.z, x.w, f);
  *reinterpret_cast<uint4*>(out + at) =
      make_uint4(q8_value_pair<false>(c0, step), q8_value_pair<true>(c0, step),
                 q8_value_pair<false>(c1, step), q8_value_pair<true>(c1, step));
}

// ---- the packed weight (see asv.h): tiles of [256 ids][64 columns], column block major, behind them
// the scales of its 2 S blocks of 128 ids, q8_pitch(H) bytes each. Within the 64 columns of an id the
// codes stand in the order of the fragments: 16 bytes hold columns 8 g .. 8 g + 7 and 32 + 8 g .. 32 +
// 8 g + 7, what lane group g takes in the two matrix steps of the stage, in one LDS read.

// Grid (2 S, ceil(H / 128)): one block of 128 ids x 128 columns; thread t takes 64 columns of id t / 2.
// QUANT: w is bf16 and quantised here; else w are codes and `scale` [ceil(V / 128)][ceil(H / 128)]
// their scales.
template <bool QUANT>
__global__ __launch_bounds__(256)
void k_pack_q8_tiles(const void* __restrict__ w, const uint8_t* __restrict__ scale, int V, int H,
                     uint8_t* __restrict__ packed, uint8_t* __restrict__ packed_scale) {
  __shared__ int s_max[4];
  const int blk = blockIdx.x, kb = blockIdx.y, S = gridDim.x / 2, t = threadIdx.x;
  const int r = t / 2, v = blk * kQBlock + r, k64 = 2 * kb + (t & 1), col = k64 * 64;
  const bool in = v < V && col < H;                 // H is a multiple of 64
  uint32_t c[16] = {};                              // the 64 codes in order
  int s = 127;
  if constexpr (QUANT) {
    uint4 x[8] = {};
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(w) +
                                                      (size_t)v * H + col);
    int a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (in) x[i] = src[i];
      a = max(a, max_abs_bf16(x[i]));
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) a = max(a, __shfl_xor(a, m, kWave));
    if ((t & 63) == 0) s_max[t >> 6] = a;
    __syncthreads();
    s = q8_scale(max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3])));
    const float f = q8_factor(s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      c[2 * i] = q8_codes(x[i].x, x[i].y, f);
      c[2 * i + 1] = q8_codes(x[i].z, x[i].w, f);
    }
  } else {
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(w) +
                                                      (size_t)v * H + col);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 x = in ? src[i] : make_uint4(0u, 0u, 0u, 0u);
      c[4 * i] = x.x;
      c[4 * i + 1] = x.y;
      c[4 * i + 2] = x.z;
      c[4 * i + 3] = x.w;
    }
    if (blk * kQBlock < V) s = scale[(size_t)blk * gridDim.y + kb];
  }
  if (col < H) {
    uint4* dst = reinterpret_cast<uint4*>(packed +
                                          (((size_t)k64 * S * 2 + blk) * kQBlock + r) * 64);
#pragma unroll
    for (int g = 0; g < 4; ++g)
      dst[g] = in ? make_uint4(c[2 * g], c[2 * g + 1], c[8 + 2 * g], c[9 + 2 * g])
                  : make_uint4(0u, 0u, 0u, 0u);
  }
  if (t == 0) packed_scale[(size_t)blk * q8_pitch(H) + kb] = (uint8_t)s;
}

// ---- a tile's logits

// Position of 16-byte chunk c of staged id r (64 bytes), in 16-byte units: four ids span the LDS's 16 bank
// groups. A pass of a wave's ds_read_b128 (see swz_phase) holds lanes of one bit 5 and one parity of
// bits 2, 3 and 4; with row l % 16 and chunk l / 16 the groups 4 (r & 3) + (c ^ 2 (r >> 3 & 1)) of its 16
// lanes are distinct.
__host__ __device__ __forceinline__ int q8_swz(int r, int c) { return r * 4 + (c ^ ((r >> 2) & 2)); }

// Sizes of a tile family with W in codes (see LmheadCfg).
template <int TV, int TR, int WV, int WR, int NST>
struct Q8Cfg {
  using B = LmheadCfg<TV, TR, WV, WR, 64, 2, Mfma16>;   // what the epilogue shares
  static constexpr int kWaves = B::kWaves, kThreads = B::kThreads, kWaveV = B::kWaveV,
                       kWaveR = B::kWaveR, MV = B::MV, MR = B::MR, NS = B::NS, kCand = B::kCand,
                       kCap = B::kCap, kScrOff = B::kScrOff, kRedOff = B::kRedOff,
                       kCntOff = B::kCntOff;
  static constexpr int kStageW = TV * 64, kStageX = TR * 128, kOffX = NST * kStageW;
  static constexpr int DW = kStageW / 1024 / kWaves, DX = kStageX / 1024 / kWaves;
  static constexpr int kLoads = DW + DX;
  static constexpr int kLds = NST * (kStageW + kStageX);
  static_assert(DW >= 1 && DX >= 1 && DW * kWaves * 1024 == kStageW &&
                DX * kWaves * 1024 == kStageX, "each wave copies whole 1 KB groups");
  static_assert(NST >= 2 && NST <= 5, "ring depth");
  static_assert(kCntOff + 8 <= kLds && kLds <= 160 * 1024, "LDS per workgroup");
};

// A tile family of the 8-bit LM head (see TileFamily), its waves along the ids. SPREAD: the spread K loop,
// else the burst ring, which copies W with the non-temporal hint.
template <int TV_, int TR_, int NST_, bool SPREAD_>
struct Q8Family {
  static constexpr int TV = TV_, TR = TR_, WV = 4, WR = 1, BK = 64, NST = NST_;
  static constexpr bool kFp8 = true, kSpread = SPREAD_;
  using MF = Mfma16;
  using C = Q8Cfg<TV, TR, WV, WR, NST>;
  static __device__ __forceinline__ void logits(const LmheadArgs& a, int v0, int v_end, int r0,
                                                uint4* smem, f32x4 (&acc)[C::MV][C::MR]);
};

// What the K loops of a tile share (see TileIo): copies, fragments and scales. The tile's first id is a
// multiple of 16, so 16 ids lie in one block of 128 and their scale is scalar.
template <class F>
struct Q8Io {
  using C = typename F::C;
  typedef const __attribute__((address_space(4))) uint32_t* ConstWords;
  const uint4* lds;
  int lane, wave, lds0, w_frag0, x_frag0[C::NS];
  unsigned w_kstep;
  __amdgpu_buffer_rsrc_t w_rsrc, x_rsrc;
  int v_rows, x_pitch;
  ConstWords wa, wb;                  // scales of the wave's first block of 128 ids and of the next
  int split;                          // 16-id blocks i >= split take wb

  __device__ __forceinline__ Q8Io(const LmheadArgs& a, int v0, int v_end, int r0,
                                  const uint4* smem)
      : lds(smem) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wv = wave % F::WV, wr = wave / F::WV;
    const int row = lane & 15, grp = lane >> 4;
    w_frag0 = q8_swz(wv * C::kWaveV + row, grp);
    static_for<C::NS>([&](auto sc) {
      constexpr int s = decltype(sc)::value;
      x_frag0[s] = C::kOffX / 16 + swz<8>(wr * C::kWaveR + row, 4 * s + grp);
    });
    lds0 = __builtin_amdgcn_readfirstlane((int)(size_t)smem);
    const unsigned Vp = ((unsigned)a.V + 255) / 256 * 256;
    w_kstep = Vp * 64;
    int w_rows = F::TV;               // ids whose copies keep their offset
    w_rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(a.W) + (size_t)v0 * 64), (short)0,
        (int)((unsigned)(a.H / 64 - 1) * w_kstep + min((unsigned)F::TV, Vp - v0) * 64),
        kRsrcWord3);
    if ((unsigned)(a.H / 64) * w_kstep <= 0x80000000u) w_rows = v_end - v0;
    const int r_last = min(r0 + F::TR, a.N) - 1;
    x_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(a.X + (size_t)r0 * a.H),
                                               (short)0, (r_last + 1 - r0) * a.H * 2, kRsrcWord3);
    v_rows = w_rows;
    x_pitch = a.H * 2;
    const int vw = v0 + wv * C::kWaveV, blk = vw / kQBlock, last = (int)(Vp / kQBlock) - 1;
    const uintptr_t base = reinterpret_cast<uintptr_t>(a.w_scale);
    wa = (ConstWords)(base + (size_t)min(blk, last) * a.scale_pitch);
    wb = (ConstWords)(base + (size_t)min(blk + 1, last) * a.scale_pitch);
    split = ((blk + 1) * kQBlock - vw) / 16;
  }
  // byte offsets at K stage 0 of this lane's 16 bytes of copy j of a stage: ids 16 j .. 16 j + 15 of W,
  // four lanes an id; rows 8 j .. 8 j + 7 of X, eight lanes a row
  __device__ __forceinline__ int w_voff(int j) const {
    const int r = j * 16 + lane / 4;
    return r < v_rows ? r * 64 + (q8_swz(r, lane & 3) & 3) * 16 : (int)0x80000000;
  }
  __device__ __forceinline__ int x_voff(int j) const {
    const int r = j * 8 + lane / 8;
    return r * x_pitch + ((lane & 7) ^ swz_phase<8>(r)) * 16;
  }
  // the codes of 16-id block i for both matrix steps of a stage; the fragment of X block j for step s
  __device__ __forceinline__ uint4 w_codes(int slot, int i) const {
    return (lds + slot * (C::kStageW / 16) + w_frag0)[64 * i];
  }
  __device__ __forceinline__ bf16x8 x_frag(int slot, int s, int j) const {
    return __builtin_bit_cast(bf16x8, (lds + slot * (C::kStageX / 16) + x_frag0[s])[128 * j]);
  }
  // the scales of K stage ks, of the wave's first block of ids and of the next one: the words that hold
  // them, and the scales themselves
  __device__ __forceinline__ void step_words(int ks, uint32_t& a, uint32_t& b) const {
    a = wa[ks >> 3];
    b = wb[ks >> 3];
  }
  __device__ __forceinline__ void steps_of(int ks, uint32_t wa_, uint32_t wb_, float& a,
                                           float& b) const {
    const int sh = 8 * ((ks >> 1) & 3);
    a = q8_step((wa_ >> sh) & 255);
    b = q8_step((wb_ >> sh) & 255);
  }
  __device__ __forceinline__ void steps(int ks, float& a, float& b) const {
    uint32_t x, y;
    step_words(ks, x, y);
    steps_of(ks, x, y, a, b);
  }
};

// The fragment of matrix step s from a block's codes.
template <int s>
__device__ __forceinline__ bf16x8 q8_widen(const uint4& c, float step) {
  const uint32_t lo = s == 0 ? c.x : c.z, hi = s == 0 ? c.y : c.w;
  return __builtin_bit_cast(bf16x8, make_uint4(q8_value_pair<false>(lo, step),
                                               q8_value_pair<true>(lo, step),
                                               q8_value_pair<false>(hi, step),
                                               q8_value_pair<true>(hi, step)));
}

// The ring of NST stages of 64 columns: read a stage's fragments, refill its slot with stage k + NST behind
// the barrier that also says stage k + 1 has landed, widen and multiply. Two workgroups share a CU
// where the ring allows it and cover each other's reads.
template <class F>
__device__ __forceinline__ void q8_ring(const LmheadArgs& a, int v0, int v_end, int r0, uint4* smem,
                                        f32x4 (&acc)[F::C::MV][F::C::MR]) {
  using C = typename F::C;
  constexpr int NST = F::NST;
  const Q8Io<F> io(a, v0, v_end, r0, smem);
  const int KT = a.H / F::BK;
  int w_voff[C::DW], x_voff[C::DX];
  static_for<C::DW>([&](auto c) {
    w_voff[decltype(c)::value] = io.w_voff(decltype(c)::value * C::kWaves + io.wave);
  });
  static_for<C::DX>([&](auto c) {
    x_voff[decltype(c)::value] = io.x_voff(decltype(c)::value * C::kWaves + io.wave);
  });
  static_assert((NST - 2) * C::kLoads <= 63, "vmcnt range");
  auto issue_stage = [&](int ks) {
    const int w_at = io.lds0 + ks % NST * C::kStageW + io.wave * 1024;
    const int x_at = io.lds0 + C::kOffX + ks % NST * C::kStageX + io.wave * 1024;
    const int w_so = __builtin_amdgcn_readfirstlane((int)((unsigned)ks * io.w_kstep));
    const int x_so = __builtin_amdgcn_readfirstlane(ks * 128);
    static_for<C::DW>([&](auto cc) {
      constexpr int c = decltype(cc)::value;
      dma16_stream(w_at + c * C::kWaves * 1024, w_voff[c], w_so, io.w_rsrc);
    });
    static_for<C::DX>([&](auto cc) {
      constexpr int c = decltype(cc)::value;
      dma16(x_at + c * C::kWaves * 1024, x_voff[c], x_so, io.x_rsrc);
    });
  };
  zero_acc(acc);
  const int pro = min(NST, KT);
  for (int ks = 0; ks < pro; ++ks) issue_stage(ks);
  wait_stage_barrier<C::kLoads>(pro - 1);
  for (int k = 0; k < KT; ++k) {
    const int slot = k % NST;
    uint4 w[C::MV];
    bf16x8 x[C::NS][C::MR];
    float sa, sb;
    io.steps(k, sa, sb);
    static_for<C::MV>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      w[i] = io.w_codes(slot, i);
    });
    static_for<C::NS * C::MR>([&](auto m) {
      constexpr int s = decltype(m)::value / C::MR, j = decltype(m)::value % C::MR;
      x[s][j] = io.x_frag(slot, s, j);
    });
    if (k + 1 < KT) {
      wait_stage_barrier<C::kLoads>(min(NST - 2, KT - 2 - k));
      if (k + NST < KT) issue_stage(k + NST);
    }
    static_for<C::NS * C::MV>([&](auto m) {
      constexpr int s = decltype(m)::value / C::MV, i = decltype(m)::value % C::MV;
      const bf16x8 f = q8_widen<s>(w[i], i < io.split ? sa : sb);
      static_for<C::MR>([&](auto jc) {
        constexpr int j = decltype(jc)::value;
        acc[i][j] = Mfma16::mma(f, x[s][j], acc[i][j]);
      });
    });
  }
  // every copy was waited for by the last stage's predecessor
  __syncthreads();
}

// Half h of the fragment of matrix step s (four codes).
template <int s, int h>
__device__ __forceinline__ void q8_widen_half(const uint4& c, float step, uint32_t (&f)[4]) {
  const uint32_t x = s == 0 ? (h == 0 ? c.x : c.y) : (h == 0 ? c.z : c.w);
  f[2 * h] = q8_value_pair<false>(x, step);
  f[2 * h + 1] = q8_value_pair<true>(x, step);
}

// The spread K loop in a three-slot ring, one barrier per stage (see lmhead_tile_spread3): copies, LDS
// reads and widening stand between the matrix instructions, one position m = (s MV + i) MR + j each.
// Waves 0 and 1 copy W, waves 2 and 3 X. The waves split the ids only (WV = 4): each id is widened
// once, and with one wave a SIMD the instructions of a stage count (128 rows at V = 128256, two by two waves
// and one by four: 133 and 129 us). Deeper rings of either operand change nothing. Per stage k:
//   m < MR          the X fragments of step 1 of slot k;
//   m < Q2          the remaining copies of stage k + 2;
//   m = Q2 - 1      wait until stage k + 1 has landed (only copies of stage k + 2 may be outstanding) +
//                   barrier;
//   m >= Q2         of stage k + 1: the codes of block 0, the X fragments of step 0, the other codes (the
//                   codes of a block are overwritten after its last widening, which is just
//                   before they may be); the first copies of stage k + 3.
// Block i of step s is widened at the last positions of the block before it, into the other of two
// fragments. Past the last stage the copies repeat the last stage into slots no later stage reads,
// and what is read of the stage after the last is discarded.
template <class F>
__device__ __forceinline__ void q8_spread(const LmheadArgs& a, int v0, int v_end, int r0,
                                          uint4* smem, f32x4 (&acc)[F::C::MV][F::C::MR]) {
  using C = typename F::C;
  constexpr int NST = 3, MV = C::MV, MR = C::MR, NS = C::NS, NF = MV + MR;
  constexpr int NM = NS * MV * MR, Q2 = NM - NF;
  constexpr int GW = C::kStageW / 2048, GX = C::kStageX / 2048, G = GW > GX ? GW : GX;
  static_assert(F::NST == NST && NS == 2 && C::kWaves == 4 && MR >= 2, "schedule");
  static_assert(Q2 >= MR + 2 && Q2 >= MV * MR, "reads of a stage end before the next one's");
  static_assert(2 * G <= 63, "vmcnt range");
  // copy c of the wave sits c NM / G positions after the barrier that opens its window; the first n1 of n
  // fall in the same stage as that barrier
  constexpr auto rel = [](int c) { return c * NM / G; };
  constexpr auto first = [=](int n) {
    int k = 0;
    for (int c = 0; c < n; ++c) k += Q2 + rel(c) < NM ? 1 : 0;
    return k;
  };
  constexpr int n1w = first(GW), n1x = first(GX), n1 = first(G);
  const Q8Io<F> io(a, v0, v_end, r0, smem);
  const int KT = a.H / F::BK;
  const bool is_w = io.wave < 2;
  const int sub = io.wave & 1;
  const __amdgpu_buffer_rsrc_t rsrc = is_w ? io.w_rsrc : io.x_rsrc;
  const unsigned kstep = is_w ? io.w_kstep : 128u;
  const int n_copies = is_w ? GW : GX;
  const int slot_bytes = is_w ? C::kStageW : C::kStageX;
  const int lds_at = io.lds0 + (is_w ? 0 : C::kOffX) + sub * 1024;
  int voff[G];
  static_for<G>([&](auto cc) {
    constexpr int c = decltype(cc)::value;
    voff[c] = is_w ? io.w_voff(2 * c + sub) : io.x_voff(2 * c + sub);
  });
  // copy c of stage j of this wave's operand into ring slot `to`
  auto issue = [&](int j, int to, auto cc) {
    constexpr int c = decltype(cc)::value;
    if (c < (GW < GX ? GW : GX) || c < n_copies)
      dma16(lds_at + to * slot_bytes + c * 2048, voff[c],
            __builtin_amdgcn_readfirstlane((int)((unsigned)min(j, KT - 1) * kstep)), rsrc);
  };
  zero_acc(acc);
  uint4 w[MV];
  bf16x8 x[NS][MR];
  uint32_t f[2][4];

  for (int j = 0; j < NST - 1; ++j) static_for<G>([&](auto cc) { issue(j, j, cc); });
  static_for<n1>([&](auto cc) { issue(NST - 1, NST - 1, cc); });
  float sa, sb, na, nb;
  io.steps(0, sa, sb);
  if (is_w) wait_vm_barrier<GW + n1w>();
  else wait_vm_barrier<GX + n1x>();
  static_for<MV>([&](auto ic) { w[decltype(ic)::value] = io.w_codes(0, decltype(ic)::value); });
  static_for<MR>([&](auto jc) {
    x[0][decltype(jc)::value] = io.x_frag(0, 0, decltype(jc)::value);
  });
  q8_widen_half<0, 0>(w[0], sa, f[0]);
  q8_widen_half<0, 1>(w[0], sa, f[0]);

  int slot = 0;
  for (int k = 0; k < KT; ++k) {
    const int nslot = slot == NST - 1 ? 0 : slot + 1;
    const int free_slot = slot == 0 ? NST - 1 : slot - 1;      // of stages k - 1 and k + 2
    const int kn = min(k + 1, KT - 1);
    uint32_t wa = 0, wb = 0;
    static_for<NM>([&](auto mc) {
      constexpr int m = decltype(mc)::value;
      constexpr int s = m / (MV * MR), q = m % (MV * MR), i = q / MR, j = q % MR;
      constexpr int b = s * MV + i, bn = (b + 1) % (NS * MV), ns = bn / MV, ni = bn % MV;
      const bf16x8 fw = __builtin_bit_cast(
          bf16x8, make_uint4(f[b & 1][0], f[b & 1][1], f[b & 1][2], f[b & 1][3]));
      // pinned in the last step only (see mma_chained)
      if constexpr (s == NS - 1) acc[i][j] = Mfma16::mma(fw, x[s][j], acc[i][j]);
      else acc[i][j] = Mfma16::mma_chained(fw, x[s][j], acc[i][j]);
      if constexpr (m == 0) io.step_words(kn, wa, wb);
      if constexpr (m == NM / 2) io.steps_of(kn, wa, wb, na, nb);
      if constexpr (j >= MR - 2) {
        const float step = b + 1 == NS * MV ? (ni < io.split ? na : nb) : (ni < io.split ? sa : sb);
        q8_widen_half<ns, j - (MR - 2)>(w[ni], step, f[(b + 1) & 1]);
      }
      if constexpr (m < MR) x[1][m] = io.x_frag(slot, 1, m);
      static_for<G>([&](auto cc) {
        constexpr int c = decltype(cc)::value;
        if constexpr (c >= n1 && Q2 + rel(c) - NM == m) issue(k + 2, free_slot, cc);
        if constexpr (c < n1 && Q2 + rel(c) == m) issue(k + 3, slot, cc);
      });
      if constexpr (m == Q2 - 1) {
        if (is_w) wait_vm_barrier<GW>();
        else wait_vm_barrier<GX>();
      }
      if constexpr (m == Q2) w[0] = io.w_codes(nslot, 0);
      if constexpr (m > Q2 && m <= Q2 + MR) x[0][m - Q2 - 1] = io.x_frag(nslot, 0, m - Q2 - 1);
      if constexpr (m > Q2 + MR) w[m - Q2 - MR] = io.w_codes(nslot, m - Q2 - MR);
      __builtin_amdgcn_sched_barrier(0);
    });
    sa = na;
    sb = nb;
    slot = nslot;
  }
  // every copy lands before the caller reuses the ring and before the workgroup can exit
  asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
  __syncthreads();
}

template <int TV, int TR, int NST, bool SPREAD>
__device__ __forceinline__ void Q8Family<TV, TR, NST, SPREAD>::logits(
    const LmheadArgs& a, int v0, int v_end, int r0, uint4* smem, f32x4 (&acc)[C::MV][C::MR]) {
  // the tile's place in scalar registers, whatever the compiler computed it with: the copies'
  // buffer resources have to be
  v0 = __builtin_amdgcn_readfirstlane(v0);
  v_end = __builtin_amdgcn_readfirstlane(v_end);
  r0 = __builtin_amdgcn_readfirstlane(r0);
  if constexpr (kSpread) q8_spread<Q8Family>(a, v0, v_end, r0, smem, acc);
  else q8_ring<Q8Family>(a, v0, v_end, r0, smem, acc);
}

// The logits themselves, `type` ASV_F32, ASV_BF16 or ASV_F16, rows `pitch` elements apart.
struct StoreArgs {
  void* out;
  int64_t pitch;
  int type;
};

template <class T, class F>
__device__ __forceinline__ void store_tile(const StoreArgs& st, int N, int v0, int v_end, int r0,
                                           const f32x4 (&acc)[F::C::MV][F::C::MR], float one) {
  using C = typename F::C;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  T* out = static_cast<T*>(st.out);
  typedef T Tv __attribute__((__vector_size__(4 * sizeof(T))));
  const bool wide = st.pitch % 4 == 0 && reinterpret_cast<uintptr_t>(out) % sizeof(Tv) == 0;
  static_for<C::MR>([&](auto jc) {
    constexpr int j = decltype(jc)::value;
    const int n = r0 + (wave / F::WV) * C::kWaveR + 16 * j + (lane & 15);
    T* row = out + (size_t)n * st.pitch;
    static_for<C::MV>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      const int v = v0 + (wave % F::WV) * C::kWaveV + 16 * i + 4 * (lane >> 4);
      Tv x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (T)(acc[i][j][e] * one);
      if (n >= N) return;
      if (wide && v + 4 <= v_end) {
        *reinterpret_cast<Tv*>(row + v) = x;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v + e < v_end) row[v + e] = x[e];
      }
    });
    __builtin_amdgcn_sched_barrier(0);
  });
}

template <class F>
__device__ __forceinline__ void logits_block(const LmheadArgs& a, const StoreArgs& st, int v0,
                                             int v_end, int r0, uint4* smem) {
  f32x4 acc[F::C::MV][F::C::MR];
  F::logits(a, v0, v_end, r0, smem, acc);
  const float one = opaque_one();
  if (st.type == ASV_F32) store_tile<float, F>(st, a.N, v0, v_end, r0, acc, one);
  else if (st.type == ASV_BF16) store_tile<__bf16, F>(st, a.N, v0, v_end, r0, acc, one);
  else store_tile<_Float16, F>(st, a.N, v0, v_end, r0, acc, one);
}

// The tiles of cut's slabs x RT row tiles on family M, its tail's on family T. A lane stores four consecutive
// ids of a row, 16 lanes 16 rows, so a row gets 32 (16-bit types) or 64 bytes of a wave's block; up to 64 rows
// the stores of one workgroup run under the reads of the others. H = 4096: one row at V = 128256 77 us (the
// weight at 6.8 TB/s), 57 rows of bf16 at V = 151936 101 us (6.3 TB/s with the logits); 333 rows at V =
// 40003, H = 2880 101 us (760 TFLOP/s: three row tiles of 128, 1.8 rounds).
template <class M, class T>
__global__ __launch_bounds__(M::C::kThreads, 1)
void k_lmhead_logits(LmheadArgs a, SlabCut cut, int RT, int blk_slabs, int blk_rows, StoreArgs st) {
  static_assert(M::TR == T::TR, "one row cut");
  __shared__ uint4 smem[(M::C::kLds > T::C::kLds ? M::C::kLds : T::C::kLds) / 16];
  const TileAt t = tile_at(cut, a.V, RT, RT, blk_slabs, blk_rows);
  if constexpr (!std::is_same_v<M, T>) {
    if (t.tail) return logits_block<T>(a, st, t.v0, t.v_end, t.rt * T::TR, smem);
  }
  logits_block<M>(a, st, t.v0, t.v_end, t.rt * M::TR, smem);
}

}  // namespace asv
