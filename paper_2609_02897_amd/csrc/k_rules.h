// Sampling rules on logits: penalties for tokens that a request has seen, a bias, a grammar mask.
//
// For row n of request b and id v, with g = how often v was generated in b (the history table) or
// drafted on the path from the root to n (the root excluded), and seen = g > 0 or v in the prompt:
//   z1 = seen ? (z > 0 ? z / repetition : z * repetition) : z
//   z2 = g > 0 ? z1 - (presence + frequency g) : z1
//   z3 = z2 + bias[v]
//   z4 = allowed[n][v] ? z3 : -inf
// K10 k_token_counts: the history table from token lists. K11 k_adjust: the rules on logits in
// memory. TileRules: the rules on a tile of logits in the accumulators of the LM-head kernel.
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
  float rep, inv, pres, freq;        // inv = 1 / rep: a quotient z / rep is z inv, one rounding more
};

// A logit under its row's penalties: table entry c, drafted `path` times on the row's path. Rounded
// operation by operation: a token's logit is the same wherever it is computed.
__device__ __forceinline__ float penalised(float z, int c, int path, const RowRule& r) {
  const int g = (c & kCountMask) + path;
  const float scaled = __fmul_rn(z, z > 0.f ? r.inv : r.rep);
  z = (c | path) != 0 ? scaled : z;
  const float less = __fsub_rn(z, __fmaf_rn(r.freq, (float)g, r.pres));
  return g > 0 ? less : z;
}

// What the rows r0 .. r0 + TR - 1 need, in LDS: each row's request (-1: none, no rules) with its
// penalties, and the links and tokens of the nodes up to the last row, from the first row's root on.
// A path is a few tokens out of V, so most workgroups have none of their ids on any path: `hit` says
// whether one of these nodes drafted one of the ids v0 .. v_end - 1.
constexpr int kPathStage = 256;      // nodes whose links and tokens are walked in LDS

__device__ __forceinline__ RowRule row_rule(const RuleArgs& a, int b) {
  return RowRule{a.repetition ? a.repetition[b] : 1.f, 0.f, a.presence ? a.presence[b] : 0.f,
                 a.frequency ? a.frequency[b] : 0.f};     // inv: see RuleRows::put_rule
}

// What a thread may have loaded before RuleRows::build: the offsets and penalties of request threadIdx.x
// (where there is one), and nodes c = r0 + 1 + k T + threadIdx.x with their links and tokens.
struct NoPrefetch {
  static constexpr bool kHas = false;
  int lo, hi;
  RowRule rule;
};
template <int CAND>
struct RulePrefetch {
  static constexpr bool kHas = true;
  static constexpr int kCand = CAND;
  int lo, hi;
  RowRule rule;
  const int *c, *p, *d;
};

template <int TR>
struct RuleRows {
  int2 at[TR];                 // request and its first row
  RowRule rules[TR];           // of the request that starts, or goes on, at this row
  int seg_lo, hit;
  int2 node[kPathStage];       // link and token

  // All threads of the workgroup, T of them; draft_tok null: no paths, off null: row n is request n. `pre`:
  // what the thread has loaded beforehand (NoPrefetch: nothing).
  template <int T, class P>
  __device__ __forceinline__ void build(const RuleArgs& a, const int32_t* __restrict__ off,
                                        const int32_t* __restrict__ parent,
                                        const int32_t* __restrict__ draft_tok, int B, int N,
                                        int r0, int v0, int v_end, const P& pre) {
    const int tid = threadIdx.x, r_end = min(r0 + TR, N);
    if (tid == 0) {
      seg_lo = r0;
      hit = 0;
    }
    if (!off) {
      for (int i = tid; r0 + i < r_end; i += T) {
        at[i] = make_int2(r0 + i, r0 + i);
        put_rule(i, row_rule(a, r0 + i));
      }
      __syncthreads();
      return;
    }
    for (int i = tid; i < TR; i += T) at[i] = make_int2(-1, r0);
    __syncthreads();
    for (int b0 = 0; b0 < B; b0 += T) {
      const int b = b0 + tid;
      int first = -1, from = 0, to = 0;
      if (b < B) {
        const bool known = P::kHas && b0 == 0;
        first = known ? pre.lo : off[b];
        from = max(first, r0);
        to = min(known ? pre.hi : off[b + 1], r_end);
      }
      const bool mine = first >= 0 && from < to, many = mine && to - from > 4;
      if (mine) {
        put_rule(from - r0, P::kHas && b0 == 0 ? pre.rule : row_rule(a, b));
        if (first < r0) seg_lo = first;       // the one request that starts before the rows
        if (!many)
          for (int n = from; n < to; ++n) at[n - r0] = make_int2(b, first);
      }
      // the rows of a larger request, by its whole wave (by its thread alone: 2 us for 60 rows)
      for (uint64_t m = __builtin_amdgcn_ballot_w64(many); m != 0; m &= m - 1) {
        const int l = __builtin_ctzll(m);
        const int2 x = make_int2(__builtin_amdgcn_readlane(b, l), __builtin_amdgcn_readlane(first, l));
        const int end = __builtin_amdgcn_readlane(to, l);
        for (int n = __builtin_amdgcn_readlane(from, l) + (tid & 63); n < end; n += kWave) at[n - r0] = x;
      }
    }
    __syncthreads();
    if (!draft_tok) return;
    const int base = seg_lo;
    bool any = false;
    auto put = [&](int c, int p, int d) {
      any |= d >= v0 && d < v_end;
      if (c - base < kPathStage) node[c - base] = make_int2(p, d);
    };
    if constexpr (P::kHas) {
      // nodes r0 + 1 .. of the rows are known; r0 is a root where no request starts before it
      static_assert(P::kCand * T >= TR, "every row's node is prefetched");
#pragma unroll
      for (int k = 0; k < P::kCand; ++k)
        if (pre.c[k] < r_end) put(pre.c[k], pre.p[k], pre.d[k]);
      if (base < r0)
        for (int c = base + tid; c <= r0; c += T) put(c, parent[c], draft_tok[c]);
    } else {
      for (int c = base + tid; c < r_end; c += T) put(c, parent[c], draft_tok[c]);
    }
    if (any) hit = 1;
    __syncthreads();
  }

  __device__ __forceinline__ void put_rule(int i, RowRule r) {
    r.inv = 1.f / r.rep;
    rules[i] = r;
  }
  __device__ __forceinline__ int req(int i) const { return at[i].x; }
  __device__ __forceinline__ const RowRule& rule(int i, int r0) const {
    return rules[max(at[i].y, r0) - r0];
  }

  // f(token) for the nodes on the path of row r0 + i, from node r0 + i up, the root left out. A link that
  // leaves the request or does not lead back ends the walk (the request is malformed).
  template <class Fn>
  __device__ __forceinline__ void walk(int i, int r0, const int32_t* __restrict__ parent,
                                       const int32_t* __restrict__ draft_tok, Fn&& f) const {
    if (at[i].x < 0) return;
    const int base = seg_lo, first = at[i].y;
    for (int c = r0 + i; c > first;) {
      int2 x;
      if ((unsigned)(c - base) < (unsigned)kPathStage) x = node[c - base];
      else x = make_int2(parent[c], draft_tok[c]);
      f(x.y);
      if (x.x < first || x.x >= c) break;
      c = x.x;
    }
  }
};

// PT entries of an array from entry `at` on, those past `left` as the last one; zeros without an array.
template <int PT, class T>
__device__ __forceinline__ void load_row(const T* __restrict__ p, size_t at, int left, bool wide,
                                         T (&x)[PT]) {
  typedef T T4 __attribute__((__vector_size__(16)));
  if (!p) {
#pragma unroll
    for (int e = 0; e < PT; ++e) x[e] = T(0);
  } else if (wide) {
#pragma unroll
    for (int q = 0; q < PT; q += 4) {
      const T4 y = *reinterpret_cast<const T4*>(p + at + q);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[q + e] = y[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < PT; ++e) x[e] = p[at + min(e, left - 1)];
  }
}

typedef int i32x4 __attribute__((__vector_size__(16)));
typedef float fx4 __attribute__((__vector_size__(16)));

// The rules on one tile of the LM-head kernel. Its accumulators are only read: the drafted logits' gather
// takes each of its logits through `one`, and the records come from row blocks that are staged in LDS,
// kStep at a time, and taken through `block` in a loop of one body. (Changed in place, the accumulators were moved
// between the register files on every pass of the K loop; with every block's code laid out like the
// records without rules, it was longer than the instruction cache and took longer to fetch than to
// run: 378 rows of the 8-bit head at V = 151936 428 us without rules, 583 with them; as it is 413 and 500,
// and 60 rows of the bf16 head at V = 128256 157 and 171. What is left is latency: the epilogue's code is
// fetched once a tile from far away, and a tile that has ids on some row's path runs 10 us longer.)
//
// Every tile reads its ids' slice of the table, the bias and the mask once per 16 rows, through the caches:
// with one request 9 bytes an id beside the weight's H or 2 H.
//
// LDS: the staged blocks, before them the gather's list and scratch; how often each row of a block (of
// each wave row) drafted each of the tile's ids on its path, in 16 bits, which hold any path of
// kMaxRuledRows rows, filled for the blocks that have one; the record exchange and the counters; the rows.
constexpr int kMaxRuledRows = 65535;

template <class F>
struct TileRules {
  using C = typename F::C;
  using Rows = RuleRows<F::TR>;
  static constexpr int kPitch = F::TV + 8;    // rows 4 banks apart
  static constexpr int kPath = F::WR * 16 * kPitch * 2;
  // as many blocks as a CU's LDS holds, or, where the ring leaves room for two workgroups, as half of it
  static constexpr int kList = F::TR == 256 ? 256 : 4 * F::TR;
  struct PathList {
    int n, steps;              // entries (kList kept), bit j: a row of block j has one
    int at[kList];             // row << 16 | id, from r0 and v0
  };
  static constexpr int kFixed =
      kPath + (C::kCntOff - C::kRedOff) + 32 + (int)(sizeof(Rows) + sizeof(PathList));
  static constexpr int kRoom = (C::kLds <= 80 * 1024 ? 80 : 160) * 1024 - kFixed;
  static constexpr int kBlockBytes = C::kWaves * C::MV * 1024;
  static constexpr int steps() {
    int n = C::MR;
    while (n * kBlockBytes > kRoom || C::MR % n != 0) --n;
    return n;
  }
  static constexpr int kStep = steps();
  static constexpr int kStage = kStep * kBlockBytes > C::kRedOff ? kStep * kBlockBytes : C::kRedOff;
  static constexpr int kRedOff = kStage + kPath;
  static constexpr int kCntOff = kRedOff + (C::kCntOff - C::kRedOff);
  static constexpr int kRowsOff = (kCntOff + 8 + 15) / 16 * 16;
  static constexpr int kBytes = kRowsOff + (int)(sizeof(Rows) + sizeof(PathList));
  static_assert(F::MF::kBlock == 16 && F::MF::kRegs == 4, "four consecutive ids a lane and block");
  const RuleArgs& r;
  const int32_t* parent;
  const int32_t* draft_tok;
  int N, V, v0, v_end, r0, lane, wr, vw;
  char* lds;
  Rows& rows;
  bool wide_c, wide_b;
  uint32_t paths;              // bit j: a row of block j has one of the tile's ids on its path

  template <class A, class P>
  __device__ __forceinline__ TileRules(const RuleArgs& r_, const A& a, int v0_, int v_end_, int r0_,
                                       void* smem, const P& pre)
      : r(r_), parent(a.parent), draft_tok(a.draft_tok), N(a.N), V(a.V), v0(v0_), v_end(v_end_),
        r0(r0_), lds(static_cast<char*>(smem)),
        rows(*reinterpret_cast<Rows*>(static_cast<char*>(smem) + kRowsOff)) {
    rows.template build<C::kThreads>(r, a.req_offsets, parent, draft_tok, a.B, N, r0, v0, v_end, pre);
    lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wr = wave / F::WV;
    vw = (wave % F::WV) * C::kWaveV + 4 * (lane >> 4);    // this lane's ids of block 0, from v0
    wide_c = V % 4 == 0 && reinterpret_cast<uintptr_t>(r.counts) % 16 == 0;
    wide_b = V % 4 == 0 && r.bias_pitch % 4 == 0 && reinterpret_cast<uintptr_t>(r.bias) % 16 == 0;
  }

  __device__ __forceinline__ PathList& list() const {
    return *reinterpret_cast<PathList*>(lds + kRowsOff + sizeof(Rows));
  }

  // The logit z of id v0 + dv in row r0 + i, for one lane.
  __device__ __forceinline__ float one(int i, int dv, float z) const {
    const int b = rows.req(i), v = v0 + dv;
    if (b < 0) return z;
    int n = 0;
    rows.walk(i, r0, parent, draft_tok, [&](int d) { n += d == v; });
    z = penalised(z, r.counts ? r.counts[(size_t)b * V + v] : 0, n, rows.rule(i, r0));
    if (r.bias) z = __fadd_rn(z, r.bias[(size_t)b * r.bias_pitch + v]);
    if (r.allowed && !((r.allowed[(size_t)(r0 + i) * r.words + (v >> 5)] >> (v & 31)) & 1))
      z = kNegInf;
    return z;
  }

  // Between the gather and the first block, by every thread: every row's path once, all rows side by side,
  // its ids of this tile into a list. (A walk is a chain of LDS reads, 0.15 us a node: walked again for
  // every block, a path of 24 nodes cost a tile that had one of its ids 20 us.)
  __device__ __forceinline__ void find_paths() {
    PathList& l = list();
    __syncthreads();
    if (threadIdx.x == 0) l.n = l.steps = 0;
    __syncthreads();
    if (rows.hit)
      for (int i = threadIdx.x; i < min(F::TR, N - r0); i += C::kThreads) {
        bool any = false;
        rows.walk(i, r0, parent, draft_tok, [&](int d) {
          if (d < v0 || d >= v_end) return;
          any = true;
          const int k = atomicAdd(&l.n, 1);
          if (k < kList) l.at[k] = i << 16 | (d - v0);
        });
        if (any) atomicOr(&l.steps, 1 << (i % C::kWaveR / 16));
      }
    __syncthreads();
    paths = __builtin_amdgcn_readfirstlane(l.steps);
  }
  __device__ __forceinline__ uint16_t* path() const {
    return reinterpret_cast<uint16_t*>(lds + kStage);
  }
  // The paths of block j, by every thread: from the list, or, where it was too short, by walking them.
  __device__ __forceinline__ void fill_paths(int j) const {
    uint32_t* words = reinterpret_cast<uint32_t*>(path());
    const PathList& l = list();
    __syncthreads();
    for (int i = threadIdx.x; i < kPath / 4; i += C::kThreads) words[i] = 0;
    __syncthreads();
    if (l.n <= kList) {
      for (int k = threadIdx.x; k < l.n; k += C::kThreads) {
        const int i = l.at[k] >> 16, id = l.at[k] & 0xffff;
        if (i % C::kWaveR / 16 != j) continue;
        const int at = (i / C::kWaveR * 16 + i % 16) * kPitch + id;
        atomicAdd(&words[at >> 1], 1u << (16 * (at & 1)));
      }
    } else {
      const int t = threadIdx.x, i = t / 16 * C::kWaveR + 16 * j + t % 16;
      if (t < 16 * F::WR && i < N - r0)
        rows.walk(i, r0, parent, draft_tok, [&](int d) {
          if (d >= v0 && d < v_end) ++path()[t * kPitch + d - v0];
        });
    }
    __syncthreads();
  }

  // Row block j of this wave, in the staged blocks: 16 bytes of lane l and 16-id block i at [i][l].
  __device__ __forceinline__ fx4* staged(int j) const {
    return reinterpret_cast<fx4*>(lds) +
           ((threadIdx.x >> 6) * kStep + j % kStep) * (C::MV * kWave);
  }

  // What a lane holds of the table and the bias for its ids, for the request of its last row, and of the
  // mask for its next row: the rows of a block mostly belong to one request, the block before's. The
  // mask's words, and another request's entries, are on their way while the block before is reduced
  // (378 rows of eight requests 513 -> 500 us). Every load is from a place inside its array, whatever the
  // row and the ids; what it brings of other rows and ids is masked or discarded.
  struct Held {
    int b = -2;
    bool fresh = false;            // c is new
    uint32_t seen = 0;             // bit i: some lane's entries of 16-id block i are in the table
    uint32_t ids = 0;              // bit 4 i + e: entry e of block i is one of the tile's ids
    i32x4 c[C::MV];
    fx4 bias[C::MV];
    uint32_t bits[C::MV];
  };
  static_assert(4 * C::MV <= 32, "a bit per entry");
  template <class T4, class T>
  __device__ __forceinline__ void load_ids(const T* __restrict__ row, bool wide,
                                           T4 (&x)[C::MV]) const {
    if (wide) {
      static_for<C::MV>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        x[i] = *reinterpret_cast<const T4*>(row + min(v0 + vw + 16 * i, V - 4));
      });
    } else {
      static_for<4 * C::MV>([&](auto ec) {
        constexpr int i = decltype(ec)::value / 4, e = decltype(ec)::value % 4;
        x[i][e] = row[min(v0 + vw + 16 * i + e, V - 1)];
      });
    }
  }
  __device__ __forceinline__ void load_bits(int j, uint32_t (&bits)[C::MV]) const {
    if (!r.allowed) return;
    const int n = min(r0 + wr * C::kWaveR + 16 * j + (lane & 15), N - 1);
    const uint32_t* row = r.allowed + (size_t)n * r.words;
    static_for<C::MV>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      bits[i] = row[min((v0 + vw + 16 * i) >> 5, r.words - 1)];
    });
  }
  __device__ __forceinline__ void load_request(int b, Held& h) const {
    if (r.counts) load_ids(r.counts + (size_t)b * V, wide_c, h.c);
    if (r.bias) load_ids(r.bias + (size_t)b * r.bias_pitch, wide_b, h.bias);
    h.b = b;
    h.fresh = true;
  }
  // The request of this lane's row of block j, or where it has none another.
  __device__ __forceinline__ int request_of(int j, int other) const {
    const int b = rows.req(wr * C::kWaveR + 16 * j + (lane & 15));
    return b < 0 ? other : b;
  }
  // Ahead of the gather, which covers the loads.
  __device__ __forceinline__ void begin(Held& h) const {
    static_for<C::MV>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      h.c[i] = i32x4{};
      h.bias[i] = fx4{};
      h.bits[i] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        h.ids |= (uint32_t)(v0 + vw + 16 * i + e < v_end) << (4 * i + e);
    });
    load_bits(0, h.bits);
    load_request(request_of(0, 0), h);
  }

  // Row block j through the rules, into z[4 i + e], -inf past the tile's ids; blocks in order, begin()
  // before the first. Rows of no request give no results (their offsets are malformed).
  __device__ __forceinline__ void block(int j, float (&z)[4 * C::MV], Held& h) const {
    const int i_row = wr * C::kWaveR + 16 * j + (lane & 15);
    if (h.fresh && r.counts) {
      h.seen = 0;
      static_for<C::MV>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        if (__any((h.c[i][0] | h.c[i][1] | h.c[i][2] | h.c[i][3]) != 0)) h.seen |= 1u << i;
      });
    }
    h.fresh = false;
    uint32_t keep = h.ids;
    if (r.allowed) {
      uint32_t on = 0;
      static_for<C::MV>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        on |= ((h.bits[i] >> ((v0 + vw + 16 * i) & 31)) & 15u) << (4 * i);
      });
      keep &= on;
    }
    if (j + 1 < C::MR) load_bits(j + 1, h.bits);
    const fx4* from = staged(j);
    static_for<C::MV>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      const fx4 y = from[i * kWave + lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) z[4 * i + e] = y[e];
    });
    const bool with_path = (paths >> j) & 1;
    const uint32_t seen = with_path ? ~0u : h.seen;
    if (seen != 0) {
      const RowRule rr = rows.rule(i_row, r0);
      const uint16_t* my_path = path() + (wr * 16 + (lane & 15)) * kPitch + vw;
      static_for<C::MV>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        if ((seen >> i) & 1) {
          const uint2 p4 = with_path ? *reinterpret_cast<const uint2*>(my_path + 16 * i)
                                     : make_uint2(0u, 0u);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int n_path = ((e < 2 ? p4.x : p4.y) >> (16 * (e & 1))) & 0xffff;
            z[4 * i + e] = penalised(z[4 * i + e], h.c[i][e], n_path, rr);
          }
        }
      });
    }
    if (r.bias) {
      static_for<4 * C::MV>([&](auto ec) {
        constexpr int i = decltype(ec)::value / 4, e = decltype(ec)::value % 4;
        z[4 * i + e] = __fadd_rn(z[4 * i + e], h.bias[i][e]);
      });
    }
    if (j + 1 < C::MR) {
      const int b = request_of(j + 1, h.b);
      if (!__all(b == h.b)) load_request(b, h);
    }
    // a bit of `keep` as a mask over the value: set, the value, else -inf
    static_for<4 * C::MV>([&](auto kc) {
      constexpr int k = decltype(kc)::value;
      const uint32_t m = (uint32_t)__builtin_amdgcn_sbfe((int)keep, k, 1);
      z[k] = __uint_as_float((__float_as_uint(z[k]) & m) | (0xff800000u & ~m));
    });
  }
};

// ---- the rules on logits in memory (K11)

constexpr int kAdjThreads = 256;
constexpr int kAdjRows = 8;           // most rows of a workgroup

struct AdjustArgs {
  RuleArgs r;
  const void* in;
  void* out;
  int64_t in_pitch, out_pitch;        // elements
  const int32_t* off;
  const int32_t* parent;
  const int32_t* draft_tok;
  int B, N, V;
  int rows;                           // of a workgroup, at most kAdjRows
};

// Grid ceil(V / kIds) * ceil(N / rows), the ids fastest: the workgroup takes kIds ids of its rows, each
// thread PT consecutive ones (16 bytes of input). Memory bound: one read and one write of the logits; the
// table and the bias are read once for the consecutive rows of one request. Many waves with one row under
// way each: 2048 rows of 128256 fp32 logits 454 to 494 us by box (4.4 to 4.8 TB/s; a copy of 2 GB 4.9); beside
// the 494 at 8 rows 513 at 4 and 511 at 16, and with two and four rows' loads issued together 527 and 611.
template <class T, int PT>
__global__ __launch_bounds__(kAdjThreads)
void k_adjust(AdjustArgs a) {
  constexpr int kIds = kAdjThreads * PT;
  __shared__ RuleRows<kAdjRows> rows;
  const int chunks = (a.V + kIds - 1) / kIds, group = blockIdx.x / chunks;
  const int tid = threadIdx.x, r0 = group * a.rows, v0 = (blockIdx.x - group * chunks) * kIds;
  const int v_end = min(v0 + kIds, a.V), r_end = min(r0 + a.rows, a.N);
  rows.template build<kAdjThreads>(a.r, a.off, a.parent, a.draft_tok, a.B, r_end, r0, v0, v_end,
                                   NoPrefetch{});
  const bool hit = __builtin_amdgcn_readfirstlane(rows.hit);
  const int v = v0 + tid * PT;
  if (v >= v_end) return;
  const RuleArgs& r = a.r;
  const int V = a.V;
  const bool full = v + PT <= V;
  const bool wide_c = full && V % 4 == 0 && reinterpret_cast<uintptr_t>(r.counts) % 16 == 0;
  const bool wide_b = full && r.bias_pitch % 4 == 0 && reinterpret_cast<uintptr_t>(r.bias) % 16 == 0;
  const T* in = static_cast<const T*>(a.in);
  T* out = static_cast<T*>(a.out);
  const bool wide_in = full && a.in_pitch % PT == 0 && reinterpret_cast<uintptr_t>(in) % 16 == 0;
  const bool wide_out = full && a.out_pitch % PT == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
  typedef T Tv __attribute__((__vector_size__(PT * sizeof(T))));
  int cur = -1;
  int c[PT] = {};
  float bias[PT] = {};
  for (int n = r0; n < r_end; ++n) {
    const int i = n - r0, b = __builtin_amdgcn_readfirstlane(rows.req(i));
    const T* from = in + (size_t)n * a.in_pitch + v;
    Tv x;
    if (wide_in) {
      x = *reinterpret_cast<const Tv*>(from);
    } else {
#pragma unroll
      for (int e = 0; e < PT; ++e) x[e] = from[min(e, V - 1 - v)];
    }
    const uint32_t bits =
        r.allowed ? r.allowed[(size_t)n * r.words + (v >> 5)] >> (v & 31) : ~0u;
    float z[PT];
    if (b >= 0) {
      if (b != cur) {
        cur = b;
        load_row<PT>(r.counts, (size_t)b * V + v, V - v, wide_c, c);
        load_row<PT>(r.bias, (size_t)b * r.bias_pitch + v, V - v, wide_b, bias);
      }
      const RowRule rr = rows.rule(i, r0);
      int path[PT] = {};
      if (hit)
        rows.walk(i, r0, a.parent, a.draft_tok, [&](int d) {
#pragma unroll
          for (int e = 0; e < PT; ++e) path[e] += d == v + e;
        });
      int any = 0;
#pragma unroll
      for (int e = 0; e < PT; ++e) {
        z[e] = (float)x[e];
        any |= c[e] | path[e];
      }
      if (any != 0) {
#pragma unroll
        for (int e = 0; e < PT; ++e) z[e] = penalised(z[e], c[e], path[e], rr);
      }
#pragma unroll
      for (int e = 0; e < PT; ++e) {
        if (r.bias) z[e] = __fadd_rn(z[e], bias[e]);
        z[e] = (bits >> e) & 1 ? z[e] : kNegInf;
        x[e] = (T)z[e];
      }
    }
    T* to = out + (size_t)n * a.out_pitch + v;
    if (wide_out) {
      *reinterpret_cast<Tv*>(to) = x;
    } else {
#pragma unroll
      for (int e = 0; e < PT; ++e)
        if (v + e < V) to[e] = x[e];
    }
  }
}

// ---- the history table (K10)

constexpr int kCountThreads = 1024;
constexpr int kCountIds = 20480;      // most ids of a workgroup, 80 KB of LDS: two workgroups a CU
constexpr int kCountLeast = 1024;     // fewest, where there are more
constexpr int kCountBatch = 8;        // tokens of a thread whose loads are issued together

struct CountArgs {
  const int32_t* tok;                 // [T]
  const int32_t* off;                 // [B + 1]
  const int32_t* prompt;              // [B] or null
  int T, B, V;
  int add;
  int ids;                            // of a workgroup, a multiple of 4
  int32_t* counts;
  int32_t* status;
};

// Grid ceil(V / ids) * B: the workgroup counts its ids of request b in LDS over all of the
// request's tokens and writes (or adds) its part of the table: no fill, and every count is the sum
// of integers, the same in any order. Tokens outside [0, V) are passed over and reported. A long list is
// a chain of loads, so each thread has kCountBatch of them under way, and as few workgroups as fill the
// chip read it. 64 lists of up to 14000 tokens at V = 151936, whose table takes 6 us to write: one load at a
// time and 8192 ids a workgroup 31.5 us, eight at a time 19.9, two workgroups a CU 18.2.
static __global__ __launch_bounds__(kCountThreads)
void k_token_counts(CountArgs a) {
  __shared__ __attribute__((aligned(16))) int s_n[kCountIds];
  const int chunks = (a.V + a.ids - 1) / a.ids, b = blockIdx.x / chunks;
  const int v0 = (blockIdx.x - b * chunks) * a.ids, tid = threadIdx.x;
  const int ids = min(a.ids, a.V - v0);
  int lo = a.off[b], hi = a.off[b + 1], bad = 0;
  if (lo < 0 || hi < lo || hi > a.T) {
    bad = ASV_RS_BAD_OFFSETS;
    lo = hi = 0;
  }
  const int n_prompt = a.prompt ? min(max(a.prompt[b], 0), hi - lo) : 0;
  for (int i = tid; i < ids; i += kCountThreads) s_n[i] = 0;
  __syncthreads();
  bool out = false;
  for (int64_t t0 = (int64_t)lo + tid; t0 < hi; t0 += kCountBatch * kCountThreads) {
    int tok[kCountBatch];
#pragma unroll
    for (int u = 0; u < kCountBatch; ++u)
      tok[u] = a.tok[min(t0 + u * kCountThreads, (int64_t)hi - 1)];
#pragma unroll
    for (int u = 0; u < kCountBatch; ++u) {
      const int64_t t = t0 + u * kCountThreads;
      const int v = tok[u];
      if (t >= hi) break;
      out |= v < 0 || v >= a.V;
      if (v < v0 || v >= v0 + ids) continue;
      if (t - lo < n_prompt) atomicOr(&s_n[v - v0], ASV_COUNT_PROMPT);
      else atomicAdd(&s_n[v - v0], 1);
    }
  }
  bad |= __syncthreads_or(out) ? ASV_RS_BAD_TOKEN : 0;
  if (tid == 0 && v0 == 0) a.status[b] = bad;
  int32_t* row = a.counts + (size_t)b * a.V + v0;
  if (a.add) {
    for (int i = tid; i < ids; i += kCountThreads) {
      const int c = s_n[i];
      if (c == 0) continue;
      const int old = row[i];
      row[i] = ((old & kCountMask) + (c & kCountMask)) | ((old | c) & ASV_COUNT_PROMPT);
    }
  } else if (a.V % 4 == 0 && reinterpret_cast<uintptr_t>(a.counts) % 16 == 0) {
    for (int i = 4 * tid; i < ids; i += 4 * kCountThreads)
      *reinterpret_cast<int4*>(row + i) = *reinterpret_cast<const int4*>(&s_n[i]);
  } else {
    for (int i = tid; i < ids; i += kCountThreads) row[i] = s_n[i];
  }
}

}  // namespace asv
