// Host side of the 8-bit LM head and of the sampling rules (include/asv.h): checks, workspace
// layouts and launches.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "asv.h"
#include "asv_host.h"
#include "asv_k1_host.h"
#include "asv_q8_host.h"
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
