// Sampling rules on logits: penalties for tokens that a request has seen, a bias, a grammar mask.
//
// For row n of request b and id v, with g = how often v was generated in b (the history table) or
// drafted on the path from the root to n (the root excluded), and seen = g > 0 or v in the prompt:
//   z1 = seen ? (z > 0 ? z / repetition : z * repetition) : z
//   z2 = g > 0 ? z1 - (presence + frequency g) : z1
//   z3 = z2 + bias[v]
//   z4 = allowed[n][v] ? z3 : -inf
// K10 k_token_counts: the history table from token lists. K11 k_adjust: the rules on logits in
// memory. apply_rules: the rules on a tile of logits in the accumulators of the LM-head kernel.
#pragma once

#include "asv.h"
#include "k_common.h"

namespace asv {

constexpr int kCountMask = ASV_COUNT_PROMPT - 1;

// Epilogue policies of the LM-head kernels: none, or the rules.
struct NoRules {
  static constexpr bool kRules = false;
};
struct RuleArgs {
  static constexpr bool kRules = true;
  const int32_t* counts;             // [B][V] or null
  const float* repetition;           // [B] or null, as the next two
  const float* presence;
  const float* frequency;
  const float* bias;                 // [V] (bias_pitch 0) or [B][V], or null
  int64_t bias_pitch;
  const uint32_t* allowed;           // [N][words] or null
  int words;
};

struct RowRule {
  float rep, pres, freq;
};

// A logit under its row's penalties: table entry c, drafted `path` times on the row's path.
__device__ __forceinline__ float penalised(float z, int c, int path, const RowRule& r) {
  const int g = (c & kCountMask) + path;
  if (c != 0 || path != 0) z = z > 0.f ? z / r.rep : z * r.rep;
  if (g > 0) z -= fmaf(r.freq, (float)g, r.pres);
  return z;
}

// What the rows r0 .. r0 + TR - 1 need, in LDS: each row's request (-1: none, no rules) with its
// penalties, and the links and tokens of the nodes up to the last row, from the first row's root on.
// A path is a few tokens out of V, so most workgroups have none of their ids on any path: `hit` says
// whether one of these nodes drafted one of the ids v0 .. v_end - 1.
constexpr int kPathStage = 512;      // nodes whose links and tokens are walked in LDS

template <int TR>
struct RuleRows {
  int req[TR], lo[TR];
  RowRule rule[TR];
  int seg_lo, hit;
  int tok[kPathStage], par[kPathStage];

  // All threads of the workgroup, T of them; draft_tok null: no paths, off null: row n is request n.
  template <int T>
  __device__ __forceinline__ void build(const RuleArgs& a, const int32_t* __restrict__ off,
                                        const int32_t* __restrict__ parent,
                                        const int32_t* __restrict__ draft_tok, int B, int N,
                                        int r0, int v0, int v_end) {
    const int tid = threadIdx.x, r_end = min(r0 + TR, N);
    auto row_rule = [&](int b) {
      return RowRule{a.repetition ? a.repetition[b] : 1.f, a.presence ? a.presence[b] : 0.f,
                     a.frequency ? a.frequency[b] : 0.f};
    };
    if (tid == 0) {
      seg_lo = r0;
      hit = 0;
    }
    if (!off) {
      for (int i = tid; r0 + i < r_end; i += T) {
        req[i] = r0 + i;
        rule[i] = row_rule(r0 + i);
      }
      __syncthreads();
      return;
    }
    for (int i = tid; i < TR; i += T) {
      req[i] = -1;
      lo[i] = 0;
    }
    __syncthreads();
    for (int b = tid; b < B; b += T) {
      const int first = off[b], from = max(first, r0), to = min(off[b + 1], r_end);
      if (first < 0 || from >= to) continue;
      const RowRule r = row_rule(b);
      for (int n = from; n < to; ++n) {
        req[n - r0] = b;
        lo[n - r0] = first;
        rule[n - r0] = r;
      }
      if (first < r0) seg_lo = first;         // the one request that starts before the rows
    }
    __syncthreads();
    if (!draft_tok) return;
    const int base = seg_lo;
    bool any = false;
    for (int c = base + tid; c < r_end; c += T) {
      const int d = draft_tok[c];
      any |= d >= v0 && d < v_end;
      if (c - base < kPathStage) {
        tok[c - base] = d;
        par[c - base] = parent[c];
      }
    }
    if (any) hit = 1;
    __syncthreads();
  }

  // f(token) for the nodes on the path of row r0 + i, from node r0 + i up, the root left out. A link that
  // leaves the request or does not lead back ends the walk (the request is malformed).
  template <class Fn>
  __device__ __forceinline__ void walk(int i, int r0, const int32_t* __restrict__ parent,
                                       const int32_t* __restrict__ draft_tok, Fn&& f) const {
    if (req[i] < 0) return;
    const int base = seg_lo, first = lo[i];
    for (int c = r0 + i; c > first;) {
      const bool in = (unsigned)(c - base) < (unsigned)kPathStage;
      const int d = in ? tok[c - base] : draft_tok[c], p = in ? par[c - base] : parent[c];
      f(d);
      if (p < first || p >= c) break;
      c = p;
    }
  }
};

// The same for a tile of the LM-head kernel, with how often each row's path drafted each of the
// tile's ids, filled only where `hit`: 16 bits hold any path of so many rows.
constexpr int kMaxRuledRows = 65535;

template <int TR, int TV>
struct RuleTile {
  RuleRows<TR> rows;
  uint16_t path[TR][TV];
};

// Four consecutive entries of a [..][V] row from id v on (a multiple of 4), 0 past V.
template <class T4, class T>
__device__ __forceinline__ T4 load4(const T* __restrict__ row, int v, int V, bool wide) {
  T4 x = {};
  if (wide) {
    if (v < V) x = *reinterpret_cast<const T4*>(row + v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (v + e < V) x[e] = row[v + e];
  }
  return x;
}

typedef int i32x4 __attribute__((__vector_size__(16)));
typedef float fx4 __attribute__((__vector_size__(16)));

// The rules on one tile of the LM-head kernel, in its accumulators. Every tile reads its ids' slice
// of the table, the bias and the mask once per 16 rows, through the caches: with one request that is
// 9 bytes an id beside the weight's 2 H. The loads of a row block are issued together.
template <class F, class A>
__device__ __forceinline__ void apply_rules(const RuleArgs& r, const A& a, int v0, int v_end, int r0,
                                            void* smem,
                                            typename F::MF::Acc (&acc)[F::C::MV][F::C::MR]) {
  using C = typename F::C;
  static_assert(F::MF::kBlock == 16 && F::MF::kRegs == 4, "four consecutive ids a lane and block");
  constexpr int T = C::kThreads;
  auto& tile = *reinterpret_cast<RuleTile<F::TR, F::TV>*>(smem);
  auto& rows = tile.rows;
  rows.template build<T>(r, a.req_offsets, a.parent, a.draft_tok, a.B, a.N, r0, v0, v_end);
  const bool hit = __builtin_amdgcn_readfirstlane(rows.hit);
  if (hit) {
    uint32_t* words = reinterpret_cast<uint32_t*>(tile.path);
    for (int i = threadIdx.x; i < F::TR * F::TV / 2; i += T) words[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < min(F::TR, a.N - r0); i += T)
      rows.walk(i, r0, a.parent, a.draft_tok, [&](int d) {
        if (d >= v0 && d < v_end) ++tile.path[i][d - v0];
      });
    __syncthreads();
  }
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wv = wave % F::WV, wr = wave / F::WV;
  const int V = a.V;
  const bool wide_c = (V & 3) == 0 && (reinterpret_cast<uintptr_t>(r.counts) & 15) == 0;
  const bool wide_b = (r.bias_pitch & 3) == 0 && (V & 3) == 0 &&
                      (reinterpret_cast<uintptr_t>(r.bias) & 15) == 0;
  const int vw = wv * C::kWaveV + 4 * (lane >> 4);    // this lane's ids of block 0, from v0
  constexpr int G = C::MV % 4 == 0 ? 4 : C::MV % 3 == 0 ? 3 : C::MV % 2 == 0 ? 2 : 1;   // blocks whose
                                                                     // loads are issued together
  static_for<C::MR * (C::MV / G)>([&](auto jc) {
    constexpr int j = decltype(jc)::value / (C::MV / G), i0 = decltype(jc)::value % (C::MV / G) * G;
    const int i_row = wr * C::kWaveR + 16 * j + (lane & 15), n = r0 + i_row;
    const int b = rows.req[i_row];
    const bool on = b >= 0;
    const RowRule rr = rows.rule[i_row];
    i32x4 c[G];
    fx4 bias[G];
    uint32_t bits[G];
    static_for<G>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      const int v = v0 + vw + 16 * (i0 + i);
      c[i] = i32x4{};
      bias[i] = fx4{};
      bits[i] = ~0u;
      if (on && v < v_end) {
        if (r.counts) c[i] = load4<i32x4>(r.counts + (size_t)b * V, v, V, wide_c);
        if (r.bias) bias[i] = load4<fx4>(r.bias + (size_t)b * r.bias_pitch, v, V, wide_b);
        if (r.allowed) bits[i] = r.allowed[(size_t)n * r.words + (v >> 5)] >> (v & 31);
      }
    });
    static_for<G>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      const int vl = vw + 16 * (i0 + i);
      const uint2 p4 = hit && on ? *reinterpret_cast<const uint2*>(&tile.path[i_row][vl])
                                 : make_uint2(0u, 0u);
      const bool special =
          !__all((c[i][0] | c[i][1] | c[i][2] | c[i][3] | (int)(p4.x | p4.y)) == 0);
      fx4 z = acc[i0 + i][j];
      if (special) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int path = ((e < 2 ? p4.x : p4.y) >> (16 * (e & 1))) & 0xffff;
          z[e] = penalised(z[e], c[i][e], path, rr);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (r.bias) z[e] += bias[i][e];
        z[e] = (bits[i] >> e) & 1 ? z[e] : kNegInf;
      }
      // back into the accumulator registers: left to itself the compiler keeps every value that it has
      // changed in vector registers, and spills
      asm volatile("" : "+a"(z));
      acc[i0 + i][j] = z;
      __builtin_amdgcn_sched_barrier(0);
    });
  });
  __syncthreads();
}

// ---- the rules on logits in memory (K11)

template <class T>
__device__ __forceinline__ float to_f32(T x) {
  if constexpr (std::is_same_v<T, float>) return x;
  else return (float)x;
}

constexpr int kAdjThreads = 256;
constexpr int kAdjRows = 8;           // rows of a workgroup

struct AdjustArgs {
  RuleArgs r;
  const void* in;
  void* out;
  int64_t in_pitch, out_pitch;        // elements
  const int32_t* off;
  const int32_t* parent;
  const int32_t* draft_tok;
  int B, N, V;
};

// Grid ceil(V / kIds) * ceil(N / kAdjRows), the ids fastest: the workgroup takes kIds ids of its rows, each thread
// PT consecutive ones (16 bytes of input). Memory bound: one read and one write of the logits; the
// rows of one request read the table and the bias once, into registers.
template <class T, int PT>
__global__ __launch_bounds__(kAdjThreads)
void k_adjust(AdjustArgs a) {
  constexpr int kIds = kAdjThreads * PT;
  __shared__ RuleRows<kAdjRows> rows;
  const int chunks = (a.V + kIds - 1) / kIds, group = blockIdx.x / chunks;
  const int tid = threadIdx.x, r0 = group * kAdjRows, v0 = (blockIdx.x - group * chunks) * kIds;
  const int v_end = min(v0 + kIds, a.V), r_end = min(r0 + kAdjRows, a.N);
  rows.template build<kAdjThreads>(a.r, a.off, a.parent, a.draft_tok, a.B, a.N, r0, v0, v_end);
  const bool hit = __builtin_amdgcn_readfirstlane(rows.hit);
  const int v = v0 + tid * PT;
  if (v >= v_end) return;
  const RuleArgs& r = a.r;
  const int V = a.V;
  const bool wide_c = (V & 3) == 0 && (reinterpret_cast<uintptr_t>(r.counts) & 15) == 0;
  const bool wide_b = (r.bias_pitch & 3) == 0 && (V & 3) == 0 &&
                      (reinterpret_cast<uintptr_t>(r.bias) & 15) == 0;
  const T* in = static_cast<const T*>(a.in);
  T* out = static_cast<T*>(a.out);
  const bool wide_in = a.in_pitch % PT == 0 && (reinterpret_cast<uintptr_t>(in) & 15) == 0 &&
                       v + PT <= V;
  const bool wide_out = a.out_pitch % PT == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0 &&
                        v + PT <= V;
  typedef T Tv __attribute__((__vector_size__(PT * sizeof(T))));
  int cur = -1;
  int c[PT];
  float bias[PT];
  for (int n = r0; n < r_end; ++n) {
    const int i = n - r0, b = rows.req[i];
    float z[PT];
    if (wide_in) {
      const Tv x = *reinterpret_cast<const Tv*>(in + (size_t)n * a.in_pitch + v);
#pragma unroll
      for (int e = 0; e < PT; ++e) z[e] = to_f32<T>(x[e]);
    } else {
#pragma unroll
      for (int e = 0; e < PT; ++e)
        z[e] = v + e < V ? to_f32<T>(in[(size_t)n * a.in_pitch + v + e]) : 0.f;
    }
    uint32_t bits = ~0u;
    if (b >= 0) {
      if (r.allowed) bits = r.allowed[(size_t)n * r.words + (v >> 5)] >> (v & 31);
      if (b != cur) {
        cur = b;
#pragma unroll
        for (int q = 0; q < PT; q += 4) {
          const i32x4 cc = r.counts ? load4<i32x4>(r.counts + (size_t)b * V, v + q, V, wide_c)
                                    : i32x4{};
          const fx4 bb = r.bias ? load4<fx4>(r.bias + (size_t)b * r.bias_pitch, v + q, V, wide_b)
                                : fx4{};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            c[q + e] = cc[e];
            bias[q + e] = bb[e];
          }
        }
      }
      const RowRule rr = rows.rule[i];
      int path[PT] = {};
      if (hit)
        rows.walk(i, r0, a.parent, a.draft_tok, [&](int d) {
#pragma unroll
          for (int e = 0; e < PT; ++e) path[e] += d == v + e;
        });
#pragma unroll
      for (int e = 0; e < PT; ++e) {
        if (c[e] != 0 || path[e] != 0) z[e] = penalised(z[e], c[e], path[e], rr);
        if (r.bias) z[e] += bias[e];
        z[e] = (bits >> e) & 1 ? z[e] : kNegInf;
      }
    }
    if (wide_out) {
      Tv x;
#pragma unroll
      for (int e = 0; e < PT; ++e) x[e] = (T)z[e];
      *reinterpret_cast<Tv*>(out + (size_t)n * a.out_pitch + v) = x;
    } else {
#pragma unroll
      for (int e = 0; e < PT; ++e)
        if (v + e < V) out[(size_t)n * a.out_pitch + v + e] = (T)z[e];
    }
  }
}

// ---- the history table (K10)

constexpr int kCountThreads = 256;
constexpr int kCountIds = 8192;       // ids of a workgroup, 32 KB of LDS

struct CountArgs {
  const int32_t* tok;                 // [T]
  const int32_t* off;                 // [B + 1]
  const int32_t* prompt;              // [B] or null
  int T, B, V;
  int add;
  int32_t* counts;
  int32_t* status;
};

// Grid ceil(V / kCountIds) * B: the workgroup counts its ids of request b in LDS over all of the
// request's tokens and writes (or adds) its part of the table: no fill, and every count is the sum
// of integers, the same in any order. Tokens outside [0, V) are passed over and reported.
static __global__ __launch_bounds__(kCountThreads)
void k_token_counts(CountArgs a) {
  __shared__ int s_n[kCountIds];
  const int chunks = (a.V + kCountIds - 1) / kCountIds, b = blockIdx.x / chunks;
  const int v0 = (blockIdx.x - b * chunks) * kCountIds, tid = threadIdx.x;
  const int ids = min(kCountIds, a.V - v0);
  int lo = a.off[b], hi = a.off[b + 1], bad = 0;
  if (lo < 0 || hi < lo || hi > a.T) {
    bad = ASV_RS_BAD_OFFSETS;
    lo = hi = 0;
  }
  const int n_prompt = a.prompt ? min(max(a.prompt[b], 0), hi - lo) : 0;
  for (int i = tid; i < ids; i += kCountThreads) s_n[i] = 0;
  __syncthreads();
  bool out = false;
  for (int t = lo + tid; t < hi; t += kCountThreads) {
    const int v = a.tok[t];
    out |= v < 0 || v >= a.V;
    if (v < v0 || v >= v0 + ids) continue;
    if (t - lo < n_prompt) atomicOr(&s_n[v - v0], ASV_COUNT_PROMPT);
    else atomicAdd(&s_n[v - v0], 1);
  }
  bad |= __syncthreads_or(out) ? ASV_RS_BAD_TOKEN : 0;
  if (tid == 0 && v0 == 0) a.status[b] = bad;
  int32_t* row = a.counts + (size_t)b * a.V + v0;
  for (int i = tid; i < ids; i += kCountThreads) {
    const int c = s_n[i];
    if (!a.add) row[i] = c;
    else if (c != 0) {
      const int old = row[i];
      row[i] = ((old & kCountMask) + (c & kCountMask)) | ((old | c) & ASV_COUNT_PROMPT);
    }
  }
}

}  // namespace asv
