// Host side of the 8-bit LM head and of the sampling rules (include/asv.h): checks, workspace
// layouts and launches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "asv.h"
#include "asv_host.h"
#include "asv_k1_host.h"
#include "k_fp8.h"
#include "k_rules.h"

namespace asv {
namespace {

// ---- the 8-bit weight

// Bytes of the codes, which the kernels address with 32 bits, and of the whole packed copy.
bool fp8_size(int V, int H, uint64_t* codes, uint64_t* total) {
  if (V <= 0 || H <= 0 || H % kKAlign != 0 || H > (1 << 20)) return false;
  const uint64_t S = ((uint64_t)V + kSlab - 1) / kSlab;
  *codes = S * kSlab * H;
  if (*codes >= (uint64_t)1 << 32) return false;
  *total = *codes + 2 * S * q8_pitch(H);
  return true;
}

bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// Whether matrices of N rows of V elements of `eb` bytes, aligned to their elements, share one. Rows of one
// pitch may lie between each other's; with two pitches the ranges from the first to the last element count.
bool rows_overlap(const void* a, int64_t pitch_a, const void* b, int64_t pitch_b, int N, int V,
                  size_t eb) {
  const uint64_t last = (uint64_t)(N - 1);
  if (!overlap(a, (last * pitch_a + V) * eb, b, (last * pitch_b + V) * eb)) return false;
  if (pitch_a != pitch_b) return true;
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  const uint64_t between = (x < y ? y - x : x - y) / eb % (uint64_t)pitch_a;
  return between < (uint64_t)V || (uint64_t)pitch_a - between < (uint64_t)V;
}

template <bool QUANT>
int pack_fp8(const void* w, const uint8_t* scale, int V, int H, void* packed, uint64_t bytes,
             void* stream) {
  uint64_t codes = 0, total = 0;
  if (!fp8_size(V, H, &codes, &total) || !w || !packed || !aligned16(w) || !aligned16(packed) ||
      bytes < total || overlap(w, (uint64_t)V * H * (QUANT ? 2 : 1), packed, total))
    return ASV_EINVAL;
  const int S = (V + kSlab - 1) / kSlab, KB = q8_blocks(H);
  if (!QUANT && (!scale || overlap(scale, (uint64_t)((V + kQBlock - 1) / kQBlock) * KB, packed,
                                   total)))
    return ASV_EINVAL;
  (void)hipGetLastError();
  uint8_t* out = static_cast<uint8_t*>(packed);
  k_pack_q8_tiles<QUANT><<<dim3(2 * S, KB), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(
      w, scale, V, H, out, out + codes);
  return launch_status("k_pack_q8_tiles");
}

// ---- the hidden states, rounded into the workspace behind `at` bytes

size_t rounded_bytes(int N, int H) { return align_up((size_t)N * H * 2); }

int round_rows(const uint16_t* hidden, const void* w, int N, int H, int V, char* to, hipStream_t s,
               LmheadArgs* g) {
  uint16_t* x = reinterpret_cast<uint16_t*>(to);
  for (int n = 0; n < N; n += kRoundRows)
    k_round_rows<<<dim3(std::min(N - n, kRoundRows), (H + kRoundCols - 1) / kRoundCols), kRoundThreads, 0,
                   s>>>(hidden + (size_t)n * H, H, x + (size_t)n * H);
  g->X = x;
  g->W = static_cast<const uint16_t*>(w);
  g->H = H;
  uint64_t codes = 0, total = 0;
  fp8_size(V, H, &codes, &total);
  g->w_scale = static_cast<const uint8_t*>(w) + codes;
  g->scale_pitch = q8_pitch(H);
  return launch_status("k_round_rows");
}

// ---- launches of the 8-bit LM head

// Up to 64 rows: the tiles of 64, 128 and 256 ids by what share of the ids a CU has.
using Q8Ids64 = Q8Family<64, 64, 4, false>;
using Q8Ids128 = Q8Family<128, 64, 3, false>;
using Q8Ids256 = Q8Family<256, 64, 2, false>;
// Beyond: tiles of 256 ids, and what the tail of a launch runs.
template <int TR> using Q8Rows = Q8Family<256, TR, 3, true>;
template <int TR, int IDS> using Q8Tail = Q8Family<IDS, TR, TR == 256 ? 2 : 3, false>;

constexpr int kQ8Group = 16;          // slab widths: 16 ids share a scale
constexpr int kQ8MinCut = 48;         // narrowest slab up to 64 rows

// ids of a slab when n slabs share `ids`
int q8_share(int64_t ids, int64_t n) {
  return (int)std::max<int64_t>(kQ8MinCut,
                                ((ids + n - 1) / n + kQ8Group - 1) / kQ8Group * kQ8Group);
}

// Most records that a step of up to N rows writes, whatever the CU count (see max_records).
size_t q8_max_records(int N, int V) {
  const size_t narrow = (V + kQ8MinCut - 1) / kQ8MinCut, whole = (V + kSlab - 1) / kSlab;
  size_t n = std::min(N, 64) * narrow;
  if (N > 64) n = std::max(n, N * (whole + std::min<size_t>(narrow, kMaxCutTail)));
  return n;
}

struct Q8Plan {
  int rows;          // tile rows: 64, 128, 192 or 256
  int ids;           // 64 rows: ids of the tile; else ids of the tail's tile
  int tail;          // 64 rows: ids of the tail's tile, 0 without a tail
  SlabCut cut;
  int S;             // slabs in all
  int64_t est;       // beyond 64 rows
};

// Up to 64 rows: equal slabs, two or three a CU, where the tile that holds them has little left over; else whole
// tiles, as many on every CU, and a tail of one or two narrower ones each, which start as the first of the
// whole ones end. us of 57 rows' bf16 logits at H = 4096 on weights that are not in the caches (what they
// move at 7 TB/s, this rule, equal slabs only): V = 16000 10, 28; 32000 19, 35; 40000 24, 38, 44; 50000 30,
// 46; 64000 38, 52; 80000 48, 66, 69; 100000 60, 75; 128256 77, 85; 140000 84, 97, 120; 151936 91, 101, 128;
// 180000 108, 124, 154; 200000 120, 142, 161; 260000 156, 186, 196.
Q8Plan q8_rows64(int V, int cus) {
  const int64_t c = cus;
  auto even = [&](int ids, int width) {
    const int S = (V + width - 1) / width;
    return Q8Plan{64, ids, 0, SlabCut{S, width, width, 0, 0}, S, 0};
  };
  auto tailed = [&](int ids, int64_t a_cu, int width) {
    const int n_main = (int)(a_cu * c), S = n_main + (V - n_main * ids + width - 1) / width;
    return Q8Plan{64, ids, width <= 64 ? 64 : 128, SlabCut{n_main, ids, width, 0, 0}, S, 0};
  };
  const int two = q8_share(V, 2 * c);
  if (V <= c * 64) return even(64, 64);
  if (two <= 64) return even(64, two);
  for (int a_cu = 1; a_cu <= 2; ++a_cu) {
    if (V <= c * 128 * a_cu) return even(128, two);
    const int width = q8_share(V - c * 128 * a_cu, c);
    if (width <= 64) return tailed(128, a_cu, width);
  }
  if (two <= 256) return even(256, two);
  const int three = q8_share(V, 3 * c);
  if (three > 224 && three <= 256) return even(256, three);
  const int64_t a_cu = V / (c * 256), rest = V - a_cu * c * 256;
  if (rest == 0) return even(256, 256);
  const int width = q8_share(rest, c);
  return tailed(256, a_cu, width <= 128 ? width : q8_share(rest, 2 * c));
}

// us of a round of 128-, 192- and 256-row tiles at H = 4096, with records and with the logits stored, where
// the 256-row tile's accumulators fill the registers and it stores as it goes: 2048 rows at V = 128256
// 1714, 1657 and 1550 with records, 1744, 1685 and 1837 with logits; 640 rows 547, 604 and 572, and 558,
// 606 and 686. (K1's rounds of bf16 take 62, 80 and 98.)
constexpr int kQ8Records[3] = {56, 77, 98}, kQ8Logits[3] = {56, 78, 117};

// Up to 256 rows, in one row tile: whole rounds of 256-id tiles and a tail of one narrower tile a CU, where
// that is estimated to be faster than the best plan over whole slabs. us of bf16 logits at H = 4096 on weights
// that are not in the caches, whole slabs -> with the tail: 100 rows, V = 16000 55 -> 40, 32000 58 -> 55,
// 70003 119 -> 101; 128 rows, 32000 56 -> 49, 75003 127 -> 110, 90003 129 -> 125; 190 rows, 16000 56 -> 49,
// 67003 148 -> 140; 256 rows, 14000 56 -> 48; 250 rows with records, 75003 173 -> 163. Tails of 128 ids
// lose at 190 rows (20000: 56 -> 65), and any behind two row tiles (333 rows, 40003: 124 -> 137; 480 rows
// level).
Q8Plan q8_tail_plan(int N, int V, int cus, const int* cost, int64_t plan_est) {
  // a tail of 64 and of 128 ids (0: not taken), and what it takes more behind whole rounds
  struct Family { int rows, tail64, tail128, behind; };
  const Family families[3] = {{128, 40, 50, 3}, {192, 49, 0, 11}, {256, 48, 0, 20}};
  Q8Plan best{};
  best.est = plan_est;
  for (int i = 0; i < 3; ++i) {
    const Family& f = families[i];
    if (N > f.rows) continue;
    const int64_t rounds = V / ((int64_t)kSlab * cus);
    const int n_main = (int)(rounds * cus), rest = V - n_main * kSlab;
    const int width = q8_share(rest, cus), n_tail = (rest + width - 1) / width;
    const int tail = width <= 64 ? f.tail64 : width <= 128 ? f.tail128 : 0;
    const int64_t est = rounds * cost[i] + tail + (rounds > 0 ? f.behind : 0);
    if (rest == 0 || tail == 0 || n_tail > kMaxCutTail || est >= best.est) continue;
    best = Q8Plan{f.rows, width <= 64 ? 64 : 128, 0, SlabCut{n_main, kSlab, width, 0, 0},
                  n_main + n_tail, est};
  }
  return best;
}

// f(main family, tail family, cut, tiles of the tail, launch) for the launches of N rows; returns the
// records a row writes. cost: see kQ8Records.
template <class Fn>
int q8_launches(int N, int V, int cus, const int* cost, Fn&& f) {
  asv_k1_launch k{};
  if (N <= 64) {
    const Q8Plan p = q8_rows64(V, cus);
    k.row_tiles = 1;
    const int tail = p.tail ? p.S - p.cut.n_main : 0;
    if (p.ids == 64) f(Q8Ids64{}, Q8Ids64{}, p.cut, 0, k);
    else if (p.ids == 128) f(Q8Ids128{}, Q8Ids64{}, p.cut, tail, k);
    else if (p.tail == 128) f(Q8Ids256{}, Q8Ids128{}, p.cut, tail, k);
    else f(Q8Ids256{}, Q8Ids64{}, p.cut, tail, k);
    return p.S;
  }
  const int S = (V + kSlab - 1) / kSlab;
  int64_t est = 0;
  const K1Plan plan = plan_k1(N, S, cus, &est, cost);
  const Q8Plan p = q8_tail_plan(N, V, cus, cost, est);
  if (p.rows) {
    k.row_tiles = 1;
    const int tail = p.S - p.cut.n_main;
    if (p.rows == 128 && p.ids == 64) f(Q8Rows<128>{}, Q8Tail<128, 64>{}, p.cut, tail, k);
    else if (p.rows == 128) f(Q8Rows<128>{}, Q8Tail<128, 128>{}, p.cut, tail, k);
    else if (p.rows == 192) f(Q8Rows<192>{}, Q8Tail<192, 64>{}, p.cut, tail, k);
    else f(Q8Rows<256>{}, Q8Tail<256, 64>{}, p.cut, tail, k);
    return p.S;
  }
  asv_k1_launch launches[2];
  const int n = k1_launches(N, S, cus, plan, launches);
  for (int q = 0; q < n; ++q) {
    const asv_k1_launch& l = launches[q];
    const SlabCut cut{l.n_slabs, kSlab, kSlab, l.slab0, l.slab0 * kSlab};
    switch (l.tile_rows) {
      case 128: f(Q8Rows<128>{}, Q8Tail<128, 64>{}, cut, 0, l); break;
      case 192: f(Q8Rows<192>{}, Q8Tail<192, 64>{}, cut, 0, l); break;
      default: f(Q8Rows<256>{}, Q8Tail<256, 64>{}, cut, 0, l); break;
    }
  }
  return S;
}

template <class E>
int verify_fp8(const asv_verify_args* a, char* ws, hipStream_t s, const E& e) {
  const Layout L = layout(a->B, a->N, a->V, q8_max_records(a->N, a->V));
  const int cus = cu_count();
  int64_t tiles = 0;
  const int S = q8_launches(a->N, a->V, cus, kQ8Records,
                            [&](auto, auto, const SlabCut& cut, int n_tail, const asv_k1_launch& k) {
                              tiles = std::max(tiles, (int64_t)cut.n_main * k.row_tiles + n_tail);
                            });
  if (!step_fits(a, tiles)) return ASV_EINVAL;
  (void)hipGetLastError();
  LmheadArgs g = lmhead_args(a, L, ws, S);
  if (int rc = round_rows(a->hidden, a->w_lm, a->N, a->H, a->V, ws + L.bytes, s, &g)) return rc;
  if (int rc = draft_conf(a, L, ws, a->N <= 64 ? S : 0, s, &g.conf)) return rc;
  q8_launches(a->N, a->V, cus, kQ8Records,
              [&](auto m, auto t, const SlabCut& cut, int n_tail, const asv_k1_launch& k) {
                launch_lmhead<decltype(m), decltype(t)>(g, cut, n_tail, k, s,
                                                        K1Events{nullptr, nullptr}, e);
              });
  if (int rc = launch_status("k_lmhead_partial")) return rc;
  return finish_verify<E::kRules>(a, L, ws, S, s);
}

// ---- rules

template <class... P>
bool aligned4(const P*... p) {
  return ((reinterpret_cast<uintptr_t>(p) | ...) & 3u) == 0;
}

bool rules_ok(const asv_logit_rules& r, int V) {
  if (!aligned4(r.counts, r.repetition, r.presence, r.frequency, r.bias, r.allowed)) return false;
  return !r.bias || r.bias_pitch == 0 || r.bias_pitch >= V;
}

bool any_rule(const asv_logit_rules& r) {
  return r.counts || r.repetition || r.presence || r.frequency || r.bias || r.allowed;
}

RuleArgs rule_args(const asv_logit_rules& r, int V) {
  return RuleArgs{r.counts, r.repetition, r.presence,    r.frequency,
                  r.bias,   r.bias_pitch, r.allowed, (V + 31) / 32};
}

template <class T, int PT>
void launch_adjust(const AdjustArgs& a, int64_t grid, hipStream_t s) {
  k_adjust<T, PT><<<(unsigned)grid, kAdjThreads, 0, s>>>(a);
}

size_t element_bytes(int type) { return type == ASV_F32 ? 4 : 2; }
bool type_ok(int type) { return type == ASV_F32 || type == ASV_BF16 || type == ASV_F16; }

}  // namespace
}  // namespace asv

using namespace asv;

extern "C" int asv_fp8_lm_head_bytes(int32_t V, int32_t H, uint64_t* bytes) {
  uint64_t codes = 0;
  return bytes && fp8_size(V, H, &codes, bytes) ? ASV_OK : ASV_EINVAL;
}

extern "C" int asv_quantize_lm_head(const uint16_t* w, int32_t V, int32_t H, void* packed,
                                    uint64_t packed_bytes, void* stream) {
  return pack_fp8<true>(w, nullptr, V, H, packed, packed_bytes, stream);
}

extern "C" int asv_pack_fp8_lm_head(const uint8_t* q, const uint8_t* scale, int32_t V, int32_t H,
                                    void* packed, uint64_t packed_bytes, void* stream) {
  return pack_fp8<false>(q, scale, V, H, packed, packed_bytes, stream);
}

extern "C" int asv_logits_workspace_bytes(int32_t N, int32_t H, int32_t V, uint64_t* bytes) {
  uint64_t codes = 0, total = 0;
  if (!bytes || N < 0 || !fp8_size(V, H, &codes, &total) || !grid_ok(N, V)) return ASV_EINVAL;
  *bytes = rounded_bytes(N, H);
  return ASV_OK;
}

extern "C" int asv_lm_head_logits(const asv_logits_args* a, void* workspace,
                                  uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  if (!a || asv_logits_workspace_bytes(a->N, a->H, a->V, &need) != ASV_OK || !type_ok(a->out_type))
    return ASV_EINVAL;
  if (a->N == 0) return ASV_OK;
  if (!a->hidden || !a->w || !a->out || a->out_pitch < a->V || !aligned16(a->hidden) ||
      !aligned16(a->w) || reinterpret_cast<uintptr_t>(a->out) % element_bytes(a->out_type))
    return ASV_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, need)) return ASV_EWORKSPACE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  LmheadArgs g{};
  g.N = a->N;
  g.V = a->V;
  if (int rc = round_rows(a->hidden, a->w, a->N, a->H, a->V, static_cast<char*>(workspace), s, &g))
    return rc;
  const StoreArgs st{a->out, a->out_pitch, a->out_type};
  q8_launches(a->N, a->V, cu_count(), kQ8Logits,
              [&](auto m, auto t, const SlabCut& cut, int n_tail, const asv_k1_launch& k) {
                using M = decltype(m);
                k_lmhead_logits<M, decltype(t)>
                    <<<cut.n_main * k.row_tiles + n_tail, M::C::kThreads, 0, s>>>(
                        g, cut, k.row_tiles, k.blk_slabs, k.blk_rows, st);
              });
  return launch_status("k_lmhead_logits");
}

extern "C" int asv_verify_ruled_workspace_bytes(int32_t B, int32_t N, int32_t H, int32_t V,
                                                int32_t w_lm_layout, uint64_t* bytes) {
  if (w_lm_layout != ASV_W_FP8) {
    if (w_lm_layout != ASV_W_ROW_MAJOR && w_lm_layout != ASV_W_PACKED) return ASV_EINVAL;
    return asv_workspace_bytes(B, N, H, V, bytes);
  }
  uint64_t codes = 0, total = 0;
  if (!bytes || !sizes_ok(B, N, H, V) || !fp8_size(V, H, &codes, &total)) return ASV_EINVAL;
  *bytes = layout(B, N, V, q8_max_records(N, V)).bytes + rounded_bytes(N, H);
  return ASV_OK;
}

extern "C" int asv_verify_ruled(const asv_verify_args* a, const asv_logit_rules* rules,
                                void* workspace, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0, packed_bytes = 0;
  if (!a || asv_verify_ruled_workspace_bytes(a->B, a->N, a->H, a->V, a->w_lm_layout, &need) != ASV_OK)
    return ASV_EINVAL;
  if (a->w_lm_layout == ASV_W_PACKED &&
      !packed_size(a->V, a->H, kPackRowsTarget, &packed_bytes))
    return ASV_EINVAL;
  if (rules && !rules_ok(*rules, a->V)) return ASV_EINVAL;
  if (a->B == 0) return ASV_OK;
  if (int rc = check_verify(a)) return rc;
  if (!workspace_ok(workspace, workspace_bytes, need)) return ASV_EWORKSPACE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const bool ruled = rules && any_rule(*rules), fp8 = a->w_lm_layout == ASV_W_FP8;
  if (!ruled && !fp8) return asv_verify(a, workspace, workspace_bytes, stream);
  if (!ruled) return verify_fp8(a, ws, s, NoRules{});
  if (a->N > kMaxRuledRows) return ASV_EINVAL;
  const RuleArgs r = rule_args(*rules, a->V);
  return fp8 ? verify_fp8(a, ws, s, r) : verify_bf16_ruled(a, ws, r, s);
}

extern "C" int asv_adjust_logits(const asv_adjust_args* a, void* stream) {
  if (!a || a->B < 0 || a->N < a->B || (a->B == 0) != (a->N == 0) || a->V <= 0 ||
      a->N >= (1 << 30) || a->V >= (1 << 30) || !type_ok(a->type) || !rules_ok(a->rules, a->V))
    return ASV_EINVAL;
  if (!a->req_offsets && (a->N != a->B || a->parent)) return ASV_EINVAL;
  if ((a->parent == nullptr) != (a->draft_tok == nullptr)) return ASV_EINVAL;
  if (a->B == 0) return ASV_OK;
  const size_t eb = element_bytes(a->type);
  if (!a->in || !a->out || a->in_pitch < a->V || a->out_pitch < a->V ||
      !aligned4(a->req_offsets, a->parent, a->draft_tok) ||
      (reinterpret_cast<uintptr_t>(a->in) | reinterpret_cast<uintptr_t>(a->out)) % eb)
    return ASV_EINVAL;
  const int ids = kAdjThreads * (int)(16 / eb);
  // fewer rows a workgroup where that takes more workgroups to fill the chip: eight of them a CU (64 bf16
  // rows of 151936 ids 24.6 us at 8 rows, 19.4 at the 2 this takes)
  const int64_t chunks = (a->V + ids - 1) / ids;
  int rows = kAdjRows;
  while (rows > 1 && chunks * ((a->N + rows - 1) / rows) < 8 * (int64_t)cu_count()) rows /= 2;
  const int64_t grid = chunks * ((a->N + rows - 1) / rows);
  if (!launch_fits(grid, kAdjThreads)) return ASV_EINVAL;
  // out is in (one row has no pitch), or apart from it
  if (a->in == a->out ? a->in_pitch != a->out_pitch && a->N > 1
                      : rows_overlap(a->in, a->in_pitch, a->out, a->out_pitch, a->N, a->V, eb))
    return ASV_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const AdjustArgs g{rule_args(a->rules, a->V), a->in,     a->out,       a->in_pitch, a->out_pitch,
                     a->req_offsets,            a->parent, a->draft_tok, a->B,        a->N,
                     a->V,                      rows};
  switch (a->type) {
    case ASV_F32: launch_adjust<float, 4>(g, grid, s); break;
    case ASV_BF16: launch_adjust<__bf16, 8>(g, grid, s); break;
    default: launch_adjust<_Float16, 8>(g, grid, s); break;
  }
  return launch_status("k_adjust");
}

extern "C" int asv_token_counts(const asv_counts_args* a, void* stream) {
  if (!a || a->B < 0 || a->T < 0 || a->V <= 0 || a->V >= (1 << 30) || (a->add != 0 && a->add != 1))
    return ASV_EINVAL;
  if (a->B == 0) return ASV_OK;
  // two workgroups a CU, of at least kCountLeast ids and at most what the LDS holds
  const int64_t want = std::max<int64_t>(1, 2 * (int64_t)cu_count() / a->B);
  const int64_t share = ((int64_t)a->V + want - 1) / want;
  const int ids = (int)std::min<int64_t>(kCountIds, std::max<int64_t>(kCountLeast, (share + 3) / 4 * 4));
  const int64_t grid = ((int64_t)a->V + ids - 1) / ids * a->B;
  if ((!a->tok && a->T > 0) || !a->tok_offsets || !a->counts || !a->req_status ||
      !launch_fits(grid, kCountThreads) || !aligned4(a->tok, a->tok_offsets, a->prompt_len, a->counts, a->req_status))
    return ASV_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const CountArgs g{a->tok, a->tok_offsets, a->prompt_len, a->T,     a->B,
                    a->V,   a->add,         ids,           a->counts, a->req_status};
  k_token_counts<<<(unsigned)grid, kCountThreads, 0, s>>>(g);
  return launch_status("k_token_counts");
}
