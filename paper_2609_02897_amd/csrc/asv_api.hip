// Host side of libasv: argument checks, workspace layouts, tile selection and the launch
// sequences of one verification step, one draft step, the pruning of the draft trees, the
// tree-attention metadata and the commit. Every entry point is declared in include/asv.h.
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <mutex>

#include <cstdio>

#include "asv.h"
#include "asv_host.h"
#include "asv_k1_host.h"
#include "k_accept.h"
#include "k_draft.h"
#include "k_lmhead.h"
#include "k_reduce.h"
#include "k_tree.h"

namespace asv {
namespace {

// Text of the most recent failure on this host thread (see asv_last_error).
thread_local char g_last_error[256] = "";

}  // namespace

void set_error(const char* what, hipError_t e) {
  snprintf(g_last_error, sizeof(g_last_error), "%s: %s (%d)", what, hipGetErrorString(e),
           (int)e);
}

int launch_status(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return ASV_OK;
  set_error(what, e);
  return ASV_EHIP;
}

int cu_count() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n <= 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
        n <= 0)
      n = 256;
    cached[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

namespace {

// Pack w into tiles of PR rows (k_pack_tiles), after the checks both pack entry points share.
template <int PR>
int pack_tiles(const uint16_t* w, int V, int H, uint16_t* packed, uint64_t packed_bytes,
               void* stream) {
  constexpr int kAlign = PR > 128 ? PR : 128;
  uint64_t need = 0;
  if (!packed_size(V, H, kAlign, &need) || !w || !packed || !aligned16(w) ||
      !aligned16(packed) || packed_bytes < need)
    return ASV_EINVAL;
  const uintptr_t w0 = reinterpret_cast<uintptr_t>(w), p0 = reinterpret_cast<uintptr_t>(packed);
  if (w0 < p0 + need && p0 < w0 + (uint64_t)V * H * 2) return ASV_EINVAL;   // overlap
  (void)hipGetLastError();
  const int T = (int)((need / 2 / H) / PR);        // tiles per 64-column block
  const int tiles = T * (H / kPackDepth);
  k_pack_tiles<PR><<<tiles, kPackThreads, 0, reinterpret_cast<hipStream_t>(stream)>>>(
      reinterpret_cast<const uint4*>(w), reinterpret_cast<uint4*>(packed), V, H, T);
  return launch_status("k_pack_tiles");
}

// ---- draft side

// The draft LM head (K5) by draft rows R = 4B. Up to 64 rows it streams its weight like K1 and
// runs K1's cut and tiles (cut_rows64), except where the vocabulary leaves each CU one slab of 64
// ids: those run on a 64-id tile of 32 or 64 rows, which holds nothing that it doesn't read and
// fills its ring three stages ahead instead of two. Beyond, one workgroup per CU: an equal share of
// the ids where that fits a tile of 128, 192 or 256 ids (128 rows) or 128 ids (256 rows), else the
// rounds of the cheapest of these tiles.
enum class DraftTile {
  kRows32x64, kRows64x64, kRows64, kRows128x128, kRows128x192, kRows128x256, kRows256x128
};

struct DraftPlan {
  DraftTile tile;
  Cut64 cut;       // kRows64: all of it; else cut.cut and cut.S
  int row_tiles;
};

DraftPlan plan_draft(int R, int V, int cus) {
  auto slabs = [&](DraftTile tile, int width, int row_tiles) {
    const int S = (V + width - 1) / width;
    return DraftPlan{tile, Cut64{Stream64::kDeep128, SlabCut{S, width, width, 0, 0}, S, false},
                     row_tiles};
  };
  if (R <= 64) {
    // Whole draft steps at H = 4096, K1's cut against the 64-id tile: V = 16384 36.2 against 27.4 us
    // at 1 request, 39.2 against 30.8 at 16. Past one slab per CU some CUs run two: from 16640 ids
    // on 39.3 against 46.7 us at 16 requests, 36.4 against 37.5 at 4, but 36.5 against 35.1 at 1
    // and 36.3 against 35.9 at 2; 22000 ids are level there.
    if (V <= (int64_t)cus * (R <= 8 ? 80 : 64))
      return slabs(R <= 32 ? DraftTile::kRows32x64 : DraftTile::kRows64x64, 64, 1);
    return DraftPlan{DraftTile::kRows64, cut_rows64(V, cus), 1};
  }
  struct Family { DraftTile tile; int ids, rows, cost; };
  // cost of one round of tiles, in us at H = 4096 (MI355X)
  const Family families[4] = {{DraftTile::kRows128x128, 128, 128, 46},
                              {DraftTile::kRows128x192, 192, 128, 59},
                              {DraftTile::kRows128x256, 256, 128, 79},
                              {DraftTile::kRows256x128, 128, 256, 59}};
  DraftPlan best{};
  int64_t best_est = INT64_MAX;
  for (const Family& f : families) {
    const int RT = (R + f.rows - 1) / f.rows;
    const int64_t tiles = ((int64_t)V + f.ids - 1) / f.ids * RT, rounds = (tiles + cus - 1) / cus;
    const int64_t est = rounds * f.cost;
    if (est >= best_est) continue;
    best_est = est;
    // the slabs one round's row tiles leave room for, ids shared equally
    const int64_t n = std::max<int64_t>(1, rounds * cus / RT);
    const int width = (int)std::min<int64_t>(
        f.ids, std::max<int64_t>(128, ((V + n - 1) / n + 7) / 8 * 8));
    best = slabs(f.tile, width, RT);
  }
  return best;
}

struct DraftLayout {
  size_t off_k = 0, off_s = 0, bytes = 0;
};

// Most records that a draft step of up to R rows writes, whatever the device's CU count: never
// falling as R or V grow (see max_records).
size_t max_draft_records(int R, int V) {
  const size_t n = (size_t)std::min(R, 64) * max_records64(V);
  return R <= 64 ? n : std::max(n, (size_t)R * ((V + 127) / 128));
}

DraftLayout draft_layout(int B, int V) {
  DraftLayout L;
  const int R = B * kTopK;
  const size_t rec = max_draft_records(R, V);
  size_t at = 0;
  L.off_k = at; at += align_up(rec * kTopK * 8);
  L.off_s = at; at += align_up(rec * 4);
  L.bytes = at;
  return L;
}

bool draft_sizes_ok(int B, int H, int V) {
  if (B < 0 || H <= 0 || V < kTopK || V >= (1 << 30)) return false;
  if (H % kKAlign != 0 || H > (1 << 20)) return false;
  // 32-bit offsets inside a tile's buffer resource: all 4B rows of X and one slab of W
  if ((int64_t)B * kTopK * H * 2 >= (int64_t)1 << 31) return false;
  // the draft LM head's workgroup count stays an int: at most ceil(V / 64) slabs up to 64 rows
  // (or one per CU of a small V), ceil(V / 128) slabs of 128-row tiles beyond
  const int64_t R = (int64_t)B * kTopK, ids = R <= 64 ? 64 : 128;
  const int64_t row_tiles = R <= 64 ? 1 : (R + 127) / 128;
  return (V + ids - 1) / ids * row_tiles < ((int64_t)1 << 31);
}

template <class M, class T = M>
void launch_draft(const asv_draft_args* a, const DraftLayout& L, char* ws, const DraftPlan& p,
                  hipStream_t s, const K1Events& ev) {
  static_assert(M::BK == kPackDepth, "a stage is one packed column block");
  DraftArgs g;
  g.X = a->hidden;
  g.W = a->w_draft;
  g.R = a->B * kTopK;
  g.H = a->H;
  g.V = a->V;
  g.S = p.cut.S;
  g.rec_k = reinterpret_cast<uint64_t*>(ws + L.off_k);
  g.rec_s = reinterpret_cast<float*>(ws + L.off_s);
  g.w_packed = a->w_draft_layout == ASV_W_PACKED ? 128 : 0;
  const int n_main = p.cut.cut.n_main;
  launch_timed(k_draft_partial<M, T>, n_main * p.row_tiles + p.cut.S - n_main, M::C::kThreads, s,
               ev.start, ev.stop, g, p.cut.cut, p.row_tiles);
}

// ---- static scratch of asv_verify_noalloc

// The workspace of asv_verify_noalloc. In host code `scratch` names a host-side stand-in, not
// the device array: the device address comes from hipGetSymbolAddress, once per device (each
// GPU holds its own copy at its own address).
__device__ __align__(256) char scratch[ASV_STATIC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;

// Device address of `scratch` on the current device, or nullptr (error recorded).
void* scratch_address() {
  static std::mutex mu;
  static void* addr[kMaxDevices] = {};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) {
    set_error("hipGetDevice", e);
    return nullptr;
  }
  if (dev < 0 || dev >= kMaxDevices) {
    set_error("asv_verify_noalloc: device ordinal out of range", hipErrorInvalidDevice);
    return nullptr;
  }
  std::lock_guard<std::mutex> lock(mu);
  if (!addr[dev]) {
    void* p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess || !p) {
      set_error("hipGetSymbolAddress(scratch)", e != hipSuccess ? e : hipErrorInvalidSymbol);
      return nullptr;
    }
    addr[dev] = p;
  }
  return addr[dev];
}

}  // namespace
}  // namespace asv

using namespace asv;

extern "C" int asv_version(void) { return ASV_VERSION; }

extern "C" const char* asv_last_error(void) { return g_last_error; }

extern "C" const char* asv_status_string(int code) {
  switch (code) {
    case ASV_OK: return "ok";
    case ASV_EINVAL: return "invalid argument (size, null or misaligned pointer, parameter)";
    case ASV_EWORKSPACE: return "workspace too small or not 256-byte aligned";
    case ASV_EHIP: return "HIP runtime error or kernel launch failure";
    case ASV_ESCRATCH:
      return "the sizes need more workspace than the static scratch of asv_verify_noalloc";
    default: return "unknown asv status code";
  }
}

extern "C" int asv_workspace_bytes(int32_t B, int32_t N, int32_t H, int32_t V,
                                   uint64_t* bytes) {
  if (!bytes || !sizes_ok(B, N, H, V)) return ASV_EINVAL;
  *bytes = layout(B, N, V).bytes;
  return ASV_OK;
}

extern "C" int asv_state_init(asv_req_state* state, int32_t B, const asv_params* p,
                              void* stream) {
  if (B < 0 || !p || (B > 0 && !state) || !params_ok(*p)) return ASV_EINVAL;
  if (B == 0) return ASV_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  k_state_init<<<(B + 255) / 256, 256, 0, s>>>(state, B, *p);
  return launch_status("k_state_init");
}

extern "C" int asv_tree_policy(const float* conf, asv_req_state* state, int32_t B,
                               const asv_params* p, void* stream) {
  if (B < 0 || !p || (B > 0 && !state) || !params_ok(*p)) return ASV_EINVAL;
  if (B == 0) return ASV_OK;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  k_tree_policy<<<(B + 255) / 256, 256, 0, s>>>(conf, state, B, *p);
  return launch_status("k_tree_policy");
}

extern "C" int asv_verify_tuned(const asv_verify_args* a, const asv_tuning* tuning,
                                void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!a || !sizes_ok(a->B, a->N, a->H, a->V)) return ASV_EINVAL;
  const asv_tuning tu = tuning ? *tuning : asv_tuning{nullptr, nullptr, 0};
  Tile forced = Tile::kRows64;
  if (tu.tile_rows != 0 && !forced_tile(tu.tile_rows, &forced)) return ASV_EINVAL;
  if (a->w_lm_layout != ASV_W_ROW_MAJOR && a->w_lm_layout != ASV_W_PACKED) return ASV_EINVAL;
  uint64_t packed_bytes = 0;
  if (a->w_lm_layout == ASV_W_PACKED &&
      !packed_size(a->V, a->H, kPackRowsTarget, &packed_bytes))
    return ASV_EINVAL;
  if (a->B == 0) return ASV_OK;
  if (int rc = check_verify(a)) return rc;
  if (!workspace_ok(workspace, workspace_bytes, layout(a->B, a->N, a->V).bytes))
    return ASV_EWORKSPACE;
  return verify_bf16(a, static_cast<char*>(workspace), tu.tile_rows != 0 ? &forced : nullptr,
                     reinterpret_cast<hipEvent_t>(tu.begin_event),
                     reinterpret_cast<hipEvent_t>(tu.end_event),
                     reinterpret_cast<hipStream_t>(stream), NoRules{});
}

// The step of asv_k1_plan and asv_k1_cut; ASV_EINVAL for sizes asv_verify would reject.
static int checked_step(int N, int V, int cus, int tile_rows, K1Step* step) {
  if (N < 1 || V < 1 || cus < 1 || !grid_ok(N, V)) return ASV_EINVAL;
  Tile forced = Tile::kRows64;
  if (tile_rows != 0 && !forced_tile(tile_rows, &forced)) return ASV_EINVAL;
  *step = k1_step(N, V, cus, tile_rows != 0 ? &forced : nullptr);
  return ASV_OK;
}

extern "C" int asv_k1_plan(int32_t N, int32_t V, int32_t cus, int32_t tile_rows,
                           asv_k1_launch* launches, int32_t* n_launches) {
  K1Step step;
  if (!launches || !n_launches) return ASV_EINVAL;
  if (int rc = checked_step(N, V, cus, tile_rows, &step)) return rc;
  for (int q = 0; q < step.n_plan; ++q) launches[q] = step.plan[q];
  *n_launches = step.n_plan;
  return ASV_OK;
}

extern "C" int asv_k1_cut(int32_t N, int32_t V, int32_t cus, int32_t tile_rows,
                          asv_lmhead_cut* cut) {
  K1Step step;
  if (!cut) return ASV_EINVAL;
  if (int rc = checked_step(N, V, cus, tile_rows, &step)) return rc;
  const CutWide& w = step.wide;
  *cut = step.rows64 ? describe(step.cut64, tile_ids_of(step.cut64.kind), 64)
         : w.rows    ? describe(w.cut, w.S, kSlab, w.rows, w.tail_ids, w.tail_rows)
                     : asv_lmhead_cut{};
  return ASV_OK;
}

extern "C" int asv_draft_cut(int32_t B, int32_t V, int32_t cus, asv_lmhead_cut* cut) {
  if (B < 1 || cus < 1 || !cut || !draft_sizes_ok(B, kKAlign, V)) return ASV_EINVAL;
  const DraftPlan p = plan_draft(B * kTopK, V, cus);
  switch (p.tile) {
    case DraftTile::kRows32x64: *cut = describe(p.cut, 64, 32); break;
    case DraftTile::kRows64x64: *cut = describe(p.cut, 64, 64); break;
    case DraftTile::kRows64: *cut = describe(p.cut, tile_ids_of(p.cut.kind), 64); break;
    case DraftTile::kRows128x128: *cut = describe(p.cut, 128, 128); break;
    case DraftTile::kRows128x192: *cut = describe(p.cut, 192, 128); break;
    case DraftTile::kRows128x256: *cut = describe(p.cut, 256, 128); break;
    case DraftTile::kRows256x128: *cut = describe(p.cut, 128, 256); break;
  }
  return ASV_OK;
}

extern "C" int asv_verify(const asv_verify_args* a, void* workspace, uint64_t workspace_bytes,
                          void* stream) {
  return asv_verify_tuned(a, nullptr, workspace, workspace_bytes, stream);
}

extern "C" int asv_verify_noalloc(const asv_verify_args* a, void* stream) {
  if (!a || !sizes_ok(a->B, a->N, a->H, a->V)) return ASV_EINVAL;
  if (a->B == 0) return asv_verify_tuned(a, nullptr, nullptr, 0, stream);
  const size_t need = layout(a->B, a->N, a->V).bytes;
  if (need > ASV_STATIC_SCRATCH_BYTES) {
    snprintf(g_last_error, sizeof(g_last_error),
             "asv_verify_noalloc: %zu workspace bytes needed, the static scratch holds %u",
             need, ASV_STATIC_SCRATCH_BYTES);
    return ASV_ESCRATCH;
  }
  void* ws = scratch_address();
  if (!ws) return ASV_EHIP;
  return asv_verify_tuned(a, nullptr, ws, ASV_STATIC_SCRATCH_BYTES, stream);
}

extern "C" int asv_packed_lm_head_bytes(int32_t V, int32_t H, uint64_t* bytes) {
  if (!bytes || !packed_size(V, H, kPackRowsTarget, bytes)) return ASV_EINVAL;
  return ASV_OK;
}

extern "C" int asv_pack_lm_head(const uint16_t* w, int32_t V, int32_t H, uint16_t* packed,
                                uint64_t packed_bytes, void* stream) {
  return pack_tiles<kPackRowsTarget>(w, V, H, packed, packed_bytes, stream);
}

extern "C" int asv_packed_draft_head_bytes(int32_t V, int32_t H, uint64_t* bytes) {
  if (!bytes || V < kTopK || !packed_size(V, H, 128, bytes)) return ASV_EINVAL;
  return ASV_OK;
}

extern "C" int asv_pack_draft_head(const uint16_t* w, int32_t V, int32_t H, uint16_t* packed,
                                   uint64_t packed_bytes, void* stream) {
  if (V < kTopK) return ASV_EINVAL;
  return pack_tiles<kPackRowsDraft>(w, V, H, packed, packed_bytes, stream);
}

extern "C" int asv_draft_workspace_bytes(int32_t B, int32_t H, int32_t V, uint64_t* bytes) {
  if (!bytes || !draft_sizes_ok(B, H, V)) return ASV_EINVAL;
  *bytes = draft_layout(B, V).bytes;
  return ASV_OK;
}

extern "C" int asv_draft_step_tuned(const asv_draft_args* a, const asv_tuning* tuning,
                                    void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!a || !draft_sizes_ok(a->B, a->H, a->V) || a->step < 0) return ASV_EINVAL;
  const asv_tuning tu = tuning ? *tuning : asv_tuning{nullptr, nullptr, 0};
  if (tu.tile_rows != 0) return ASV_EINVAL;
  if (a->w_draft_layout != ASV_W_ROW_MAJOR && a->w_draft_layout != ASV_W_PACKED)
    return ASV_EINVAL;
  uint64_t packed_bytes = 0;
  if (a->w_draft_layout == ASV_W_PACKED && !packed_size(a->V, a->H, 128, &packed_bytes))
    return ASV_EINVAL;
  if (a->B == 0) return ASV_OK;
  if (!a->hidden || !a->w_draft || !a->tree || !a->topk_id || !a->topk_logp || !a->row_lse ||
      !a->front_tok)
    return ASV_EINVAL;
  if (!aligned16(a->hidden) || !aligned16(a->w_draft)) return ASV_EINVAL;
  if (!a->state && a->step == 0) {
    const int ns = a->shape[0], tk = a->shape[1], nd = a->shape[2];
    if (!(ns >= 1 && tk >= 1 && tk <= kTopK && nd >= 1 && ns <= kPoolMax &&
          tk + (ns - 1) * tk * tk <= kPoolMax))
      return ASV_EINVAL;
  }
  const DraftLayout L = draft_layout(a->B, a->V);
  if (!workspace || workspace_bytes < L.bytes ||
      (reinterpret_cast<uintptr_t>(workspace) % kAlign) != 0)
    return ASV_EWORKSPACE;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  (void)hipGetLastError();
  // timing events (measurement only): the start and the end of the draft LM head's launch
  const K1Events ev{reinterpret_cast<hipEvent_t>(tu.begin_event),
                    reinterpret_cast<hipEvent_t>(tu.end_event)};
  const DraftPlan p = plan_draft(a->B * kTopK, a->V, cu_count());
  // four waves a workgroup up to 64 rows, eight beyond
  if (!launch_fits((int64_t)p.cut.S * p.row_tiles, (a->B * kTopK <= 64 ? 4 : 8) * kWave))
    return ASV_EINVAL;
  switch (p.tile) {
    case DraftTile::kRows32x64:
      launch_draft<TileFamily<64, 32, 2, 1, 4, 0, true, Mfma32>>(a, L, ws, p, s, ev);
      break;
    case DraftTile::kRows64x64:
      launch_draft<TileFamily<64, 64, 2, 2, 4, 0, true, Mfma32>>(a, L, ws, p, s, ev);
      break;
    case DraftTile::kRows64:
      switch (p.cut.kind) {
        case Stream64::kDeep128:
          if (p.cut.tail64)
            launch_draft<Deep128, Deep64>(a, L, ws, p, s, ev);
          else
            launch_draft<Deep128>(a, L, ws, p, s, ev);
          break;
        case Stream64::kSpread256: launch_draft<Spread256>(a, L, ws, p, s, ev); break;
        case Stream64::kWide256: launch_draft<Wide256>(a, L, ws, p, s, ev); break;
      }
      break;
    // <ids, draft rows, waves along ids, waves along rows, ring depth, K loop, non-temporal W
    // copies, MFMA shape>. Eight waves: one workgroup per CU needs them to keep copies and MFMAs
    // in flight. The spread loop on the wider tiles (128 ids x 256 rows: 59 us a round against
    // 72 us with the burst ring); the 128x128 tile is MFMA-light and 2-5% faster on the burst
    // ring (32000 ids, 80 and 128 rows), where the 32x32 shape's cheaper epilogue (one lane
    // merge instead of two, on half as many row blocks) is worth another 1-3%. The hint pays on
    // the others (64000 ids, 128 rows: 294 -> 284 us for three steps; 256 rows: 450 -> 432).
    case DraftTile::kRows128x128:
      launch_draft<TileFamily<128, 128, 2, 4, 3, 0, false, Mfma32>>(a, L, ws, p, s, ev);
      break;
    case DraftTile::kRows128x192:
      launch_draft<TileFamily<192, 128, 2, 4, 3, 3, true>>(a, L, ws, p, s, ev);
      break;
    case DraftTile::kRows128x256:
      launch_draft<TileFamily<256, 128, 2, 4, 3, 3, true>>(a, L, ws, p, s, ev);
      break;
    case DraftTile::kRows256x128:
      launch_draft<TileFamily<128, 256, 2, 4, 3, 3, true>>(a, L, ws, p, s, ev);
      break;
  }
  if (int rc = launch_status("k_draft_partial")) return rc;
  DraftGrowArgs g;
  g.B = a->B;
  g.S = p.cut.S;
  g.step = a->step;
  g.rec_k = reinterpret_cast<const uint64_t*>(ws + L.off_k);
  g.rec_s = reinterpret_cast<const float*>(ws + L.off_s);
  g.vocab_map = a->vocab_map;
  g.state = a->state;
  for (int k = 0; k < 3; ++k) g.shape[k] = a->shape[k];
  g.tree = a->tree;
  g.topk_id = a->topk_id;
  g.topk_logp = a->topk_logp;
  g.row_lse = a->row_lse;
  g.front_tok = a->front_tok;
  g.draft_conf = a->draft_conf;
  // the records of a row in one round of loads: four a lane up to 256 of them, else eight
  if (g.S <= 4 * kWave)
    k_draft_grow<4><<<a->B, kDraftThreads, 0, s>>>(g);
  else
    k_draft_grow<8><<<a->B, kDraftThreads, 0, s>>>(g);
  return launch_status("k_draft_grow");
}

extern "C" int asv_draft_step(const asv_draft_args* a, void* workspace, uint64_t workspace_bytes,
                              void* stream) {
  return asv_draft_step_tuned(a, nullptr, workspace, workspace_bytes, stream);
}

extern "C" int asv_draft_prune(const asv_draft_tree* tree, int32_t B, const int32_t* root_tok,
                               int32_t n_cap, int32_t* parent, int32_t* draft_tok,
                               int32_t* req_offsets, int32_t* req_status, void* stream) {
  if (B < 0 || n_cap < 0 || !launch_fits(B, kPruneThreads)) return ASV_EINVAL;
  if (B == 0) return ASV_OK;
  if (!tree || !parent || !draft_tok || !req_offsets || !req_status) return ASV_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  k_draft_prune<<<B, kPruneThreads, 0, s>>>(tree, root_tok, n_cap, parent, draft_tok,
                                            req_offsets, req_status);
  return launch_status("k_draft_prune");
}

extern "C" int asv_tree_meta(const int32_t* parent, const int32_t* req_offsets, int32_t B,
                             int32_t N, const int32_t* pos_base, int32_t mask_words,
                             int32_t* pos, uint32_t* mask, int32_t* req_status, void* stream) {
  if (B < 0 || N < B || (B == 0) != (N == 0) || !launch_fits(B, kMetaThreads)) return ASV_EINVAL;
  if (B == 0) return ASV_OK;
  if (!parent || !req_offsets || !req_status || (mask && mask_words < 1)) return ASV_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  k_tree_meta<<<B, kMetaThreads, 0, s>>>(parent, req_offsets, B, N, pos_base, mask_words, pos,
                                         mask, req_status);
  return launch_status("k_tree_meta");
}

extern "C" int asv_commit(const asv_commit_args* a, void* stream) {
  if (!a || a->B < 0 || a->N < a->B || (a->B == 0) != (a->N == 0) ||
      !launch_fits(a->B, kCommitThreads))
    return ASV_EINVAL;
  if (a->B == 0) return ASV_OK;
  if (!a->req_offsets || !a->draft_tok || !a->accepted_len || !a->accepted_path ||
      !a->bonus_token || !a->commit_off || !a->commit_tok || !a->commit_row || !a->req_status)
    return ASV_EINVAL;
  if (a->row_src) {
    if (!a->row_dst || a->row_bytes <= 0 || a->row_bytes % 4 != 0) return ASV_EINVAL;
    if ((reinterpret_cast<uintptr_t>(a->row_src) | reinterpret_cast<uintptr_t>(a->row_dst)) & 3)
      return ASV_EINVAL;
  }
  CommitArgs c;
  c.B = a->B;
  c.N = a->N;
  c.off = a->req_offsets;
  c.tok = a->draft_tok;
  c.acc_len = a->accepted_len;
  c.path = a->accepted_path;
  c.bonus = a->bonus_token;
  c.c_off = a->commit_off;
  c.c_tok = a->commit_tok;
  c.c_row = a->commit_row;
  c.src = static_cast<const char*>(a->row_src);
  c.dst = static_cast<char*>(a->row_dst);
  c.row_bytes = a->row_bytes;
  c.status = a->req_status;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  k_commit<<<dim3(a->B, c.src ? kCommitSplit : 1), kCommitThreads, 0, s>>>(c);
  return launch_status("k_commit");
}
