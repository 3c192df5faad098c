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
// instructions (v_mfma_f32_16x16x128_f8f6f4, v_mfma_f32_16x16x32_fp8_fp8) are not used: they
// align the products of one instruction to the largest and keep about 13 bits below it (measured: errors
// up to 2^-12 of the largest product, logits 1.5e-5 off in the 2-norm against 1e-7), which would turn the
// top-1 of rows with close logits.
//
// What 8 bits buy is the weight's stream, which bounds the product up to a few hundred rows: W
// goes to LDS as codes, half of K1's bytes, and each fragment is widened in registers by
// v_cvt_scalef32_pk_bf16_fp8 (two values an instruction, the scale included) while the matrix unit
// runs. The rounded X is small and is written once as bf16 (K12 k_round_rows); the rest is K1's: its tile
// shapes, its epilogue (lmhead_block), or the logits stored (k_lmhead_logits).
#pragma once

#include "k_lmhead.h"

namespace asv {

constexpr int kQBlock = 128;          // columns (and ids of W) of one scale
typedef int i32x8 __attribute__((__vector_size__(32)));
typedef __bf16 bf16x2 __attribute__((__vector_size__(4)));

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

// K12. Grid (N, ceil(H / kRoundCols)): eight columns a thread, a block per 16 lanes. X bf16 [N][H], out the
// values that its codes and scales stand for, bf16 [N][H].
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
  static constexpr int kStageW = TV * 64, kStageX = TR * 128, kStage = kStageW + kStageX;
  static constexpr int DW = kStageW / 1024 / kWaves, DX = kStageX / 1024 / kWaves;
  static constexpr int kLoads = DW + DX;
  static constexpr int kLds = NST * kStage;
  static_assert(DW >= 1 && DX >= 1 && DW * kWaves * 1024 == kStageW &&
                DX * kWaves * 1024 == kStageX, "each wave copies whole 1 KB groups");
  static_assert(NST >= 2 && NST <= 5 && (NST - 2) * kLoads <= 63, "ring depth, vmcnt range");
  static_assert(kCntOff + 8 <= kLds && kLds <= 160 * 1024, "LDS per workgroup");
};

// A tile family of the 8-bit LM head (see TileFamily). LOOP: 0 the burst ring, 3 the spread loop.
template <int TV_, int TR_, int WV_, int WR_, int NST_, int LOOP_, bool STREAM_W_>
struct Q8Family {
  static constexpr int TV = TV_, TR = TR_, WV = WV_, WR = WR_, BK = 64, NST = NST_, LOOP = LOOP_;
  static constexpr bool STREAM_W = STREAM_W_, kFp8 = true;
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
  int w_voff[C::DW], x_voff[C::DX];
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
      x_frag0[s] = C::kStageW / 16 + swz<8>(wr * C::kWaveR + row, 4 * s + grp);
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
    static_for<C::DW>([&](auto ic) {   // copy j: ids 16 j .. 16 j + 15, four lanes an id
      constexpr int i = decltype(ic)::value;
      const int r = (i * C::kWaves + wave) * 16 + lane / 4;
      w_voff[i] = r < w_rows ? r * 64 + (q8_swz(r, lane & 3) & 3) * 16 : (int)0x80000000;
    });
    static_for<C::DX>([&](auto ic) {   // copy j: rows 8 j .. 8 j + 7, eight lanes a row
      constexpr int i = decltype(ic)::value;
      const int r = (i * C::kWaves + wave) * 8 + lane / 8;
      x_voff[i] = r * a.H * 2 + ((lane & 7) ^ swz_phase<8>(r)) * 16;
    });
    const int vw = v0 + wv * C::kWaveV, blk = vw / kQBlock, last = (int)(Vp / kQBlock) - 1;
    const uintptr_t base = reinterpret_cast<uintptr_t>(a.w_scale);
    wa = (ConstWords)(base + (size_t)min(blk, last) * a.scale_pitch);
    wb = (ConstWords)(base + (size_t)min(blk + 1, last) * a.scale_pitch);
    split = ((blk + 1) * kQBlock - vw) / 16;
  }
  // copy c of this wave (W first) of K stage ks into ring slot `slot`
  template <int c>
  __device__ __forceinline__ void copy(int slot, int ks) const {
    const int base = lds0 + slot * C::kStage;
    if constexpr (c < C::DW) {
      const int at = base + (c * C::kWaves + wave) * 1024;
      const int so = __builtin_amdgcn_readfirstlane((int)((unsigned)ks * w_kstep));
      if constexpr (F::STREAM_W) dma16_stream(at, w_voff[c], so, w_rsrc);
      else dma16(at, w_voff[c], so, w_rsrc);
    } else
      dma16(base + C::kStageW + ((c - C::DW) * C::kWaves + wave) * 1024, x_voff[c - C::DW],
            __builtin_amdgcn_readfirstlane(ks * 128), x_rsrc);
  }
  // the codes of 16-id block i for both matrix steps of a stage; the fragment of X block j for step s
  __device__ __forceinline__ uint4 w_codes(int slot, int i) const {
    return (lds + slot * (C::kStage / 16) + w_frag0)[64 * i];
  }
  __device__ __forceinline__ bf16x8 x_frag(int slot, int s, int j) const {
    return __builtin_bit_cast(bf16x8, (lds + slot * (C::kStage / 16) + x_frag0[s])[128 * j]);
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
  auto issue_stage = [&](int ks) {
    static_for<C::kLoads>([&](auto cc) { io.template copy<decltype(cc)::value>(ks % NST, ks); });
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
__device__ __forceinline__ void q8_spread3(const LmheadArgs& a, int v0, int v_end, int r0,
                                           uint4* smem, f32x4 (&acc)[F::C::MV][F::C::MR]) {
  using C = typename F::C;
  constexpr int NST = 3, MV = C::MV, MR = C::MR, NS = C::NS, NF = MV + MR;
  constexpr int NM = NS * MV * MR, G = C::kLoads, Q2 = NM - NF;
  static_assert(F::NST == NST && NS == 2 && MV % 2 == 0 && MR >= 2, "schedule");
  static_assert(Q2 >= MR + 2 && Q2 >= MV * MR, "reads of a stage end before the next one's");
  static_assert(2 * G <= 63, "vmcnt range");
  constexpr auto rel = [](int c) { return c * NM / G; };
  constexpr int n1 = [&] {
    int n = 0;
    for (int c = 0; c < G; ++c) n += Q2 + rel(c) < NM ? 1 : 0;
    return n;
  }();
  const Q8Io<F> io(a, v0, v_end, r0, smem);
  const int KT = a.H / F::BK;
  auto issue_copy = [&](int j, auto cc) {
    io.template copy<decltype(cc)::value>(j % NST, min(j, KT - 1));
  };
  zero_acc(acc);
  uint4 w[MV];
  bf16x8 x[NS][MR];
  uint32_t f[2][4];

  static_for<G>([&](auto cc) { issue_copy(0, cc); });
  static_for<G>([&](auto cc) { issue_copy(1, cc); });
  static_for<G>([&](auto cc) {
    if constexpr (decltype(cc)::value < n1) issue_copy(2, cc);
  });
  float sa, sb, na, nb;
  io.steps(0, sa, sb);
  wait_vm_barrier<G + n1>();
  static_for<MV>([&](auto ic) { w[decltype(ic)::value] = io.w_codes(0, decltype(ic)::value); });
  static_for<MR>([&](auto jc) {
    x[0][decltype(jc)::value] = io.x_frag(0, 0, decltype(jc)::value);
  });
  q8_widen_half<0, 0>(w[0], sa, f[0]);
  q8_widen_half<0, 1>(w[0], sa, f[0]);

  int slot = 0;
  for (int k = 0; k < KT; ++k) {
    const int nslot = slot == NST - 1 ? 0 : slot + 1;
    uint32_t wa = 0, wb = 0;
    const int kn = min(k + 1, KT - 1);
    static_for<NM>([&](auto mc) {
      constexpr int m = decltype(mc)::value;
      constexpr int s = m / (MV * MR), q = m % (MV * MR), i = q / MR, j = q % MR;
      constexpr int b = s * MV + i, nb_ = (b + 1) % (NS * MV), ns = nb_ / MV, ni = nb_ % MV;
      acc[i][j] = Mfma16::mma(
          __builtin_bit_cast(bf16x8, make_uint4(f[b & 1][0], f[b & 1][1], f[b & 1][2], f[b & 1][3])),
          x[s][j], acc[i][j]);
      if constexpr (m == 0) io.step_words(kn, wa, wb);
      if constexpr (m == NM / 2) io.steps_of(kn, wa, wb, na, nb);
      if constexpr (j >= MR - 2) {
        constexpr int h = j - (MR - 2);
        const float step = b + 1 == NS * MV ? (ni < io.split ? na : nb) : (ni < io.split ? sa : sb);
        q8_widen_half<ns, h>(w[ni], step, f[(b + 1) & 1]);
      }
      if constexpr (m < MR) x[1][m] = io.x_frag(slot, 1, m);
      static_for<G>([&](auto cc) {
        constexpr int c = decltype(cc)::value;
        if constexpr (c >= n1 && Q2 + rel(c) - NM == m) issue_copy(k + 2, cc);
        if constexpr (c < n1 && Q2 + rel(c) == m) issue_copy(k + 3, cc);
      });
      if constexpr (m == Q2 - 1) wait_vm_barrier<G>();
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

template <int TV, int TR, int WV, int WR, int NST, int LOOP, bool STREAM_W>
__device__ __forceinline__ void Q8Family<TV, TR, WV, WR, NST, LOOP, STREAM_W>::logits(
    const LmheadArgs& a, int v0, int v_end, int r0, uint4* smem, f32x4 (&acc)[C::MV][C::MR]) {
  // the tile's place in scalar registers, whatever the compiler computed it with: the copies'
  // buffer resources have to be
  v0 = __builtin_amdgcn_readfirstlane(v0);
  v_end = __builtin_amdgcn_readfirstlane(v_end);
  r0 = __builtin_amdgcn_readfirstlane(r0);
  if constexpr (LOOP == 3) q8_spread3<Q8Family>(a, v0, v_end, r0, smem, acc);
  else q8_ring<Q8Family>(a, v0, v_end, r0, smem, acc);
}

// The logits themselves: the tiles of cut's slabs x RT row tiles, rows of `pitch` elements of T.
template <class F, class T>
__global__ __launch_bounds__(F::C::kThreads, 1)
void k_lmhead_logits(LmheadArgs a, SlabCut cut, int RT, int blk_slabs, int blk_rows, T* out,
                     int64_t pitch) {
  using C = typename F::C;
  __shared__ uint4 smem[C::kLds / 16];
  const TileAt t = tile_at(cut, a.V, RT, RT, blk_slabs, blk_rows);
  const int r0 = t.rt * F::TR;
  f32x4 acc[C::MV][C::MR];
  F::logits(a, t.v0, t.v_end, r0, smem, acc);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wv = wave % F::WV, wr = wave / F::WV;
  typedef T Tv __attribute__((__vector_size__(4 * sizeof(T))));
  const bool wide = pitch % 4 == 0 && reinterpret_cast<uintptr_t>(out) % sizeof(Tv) == 0;
  const float one = opaque_one();
  static_for<C::MR>([&](auto jc) {
    constexpr int j = decltype(jc)::value;
    const int n = r0 + wr * C::kWaveR + 16 * j + (lane & 15);
    T* row = out + (size_t)n * pitch;
    static_for<C::MV>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      const int v = t.v0 + wv * C::kWaveV + 16 * i + 4 * (lane >> 4);
      Tv x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (T)(acc[i][j][e] * one);
      if (n >= a.N) return;
      if (wide && v + 4 <= t.v_end) {
        *reinterpret_cast<Tv*>(row + v) = x;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (v + e < t.v_end) row[v + e] = x[e];
      }
    });
    __builtin_amdgcn_sched_barrier(0);
  });
}

}  // namespace asv
