// Launches of the 8-bit LM head: how its plans cut the ids and the rows.
#pragma once

#include <algorithm>

#include "asv.h"
#include "asv_k1_host.h"
#include "k_fp8.h"

namespace asv {
namespace {

// Up to 64 rows: the tiles of 64, 128 and 256 ids by what share of the ids a CU has.
using Q8Ids64 = Q8Family<64, 64, 4, false>;
using Q8Ids128 = Q8Family<128, 64, 3, false>;
using Q8Ids256 = Q8Family<256, 64, 2, false>;
// Beyond: tiles of 256 ids, and what the tail of a launch runs (of 128 rows; of 256 where it is alone).
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

// In one row tile, where that is estimated to be faster than the best plan over whole slabs: up to 128 rows whole
// rounds of 256-id tiles and a tail of one narrower tile a CU; up to 256 rows, where 64 ids a CU hold the
// vocabulary, that tail alone. us of bf16 logits at H = 4096 on weights that are not in the caches,
// whole slabs -> with the tail: 100 rows, V = 16000 55 -> 40, 32000 58 -> 55, 70003 119 -> 101; 128 rows, 32000
// 56 -> 49, 75003 127 -> 110, 90003 129 -> 125; 256 rows, 14000 56 -> 48. Behind whole rounds of the taller
// tiles a tail (60 and 68 us) is never estimated below a launch of 128-row tiles over the slabs that are
// left (56). Tails of 128 ids lose at 190 rows (20000: 56 -> 65), and any behind two row tiles (333 rows, 40003:
// 124 -> 137; 480 rows level).
Q8Plan q8_tail_plan(int N, int V, int cus, const int* cost, int64_t plan_est) {
  // a tail of 64 and of 128 ids (0: not taken)
  struct Family { int rows, tail64, tail128; };
  const Family families[2] = {{128, 40, 50}, {256, 48, 0}};
  constexpr int kBehind = 3;      // what a tail takes more behind whole rounds
  Q8Plan best{};
  best.est = plan_est;
  for (const Family& f : families) {
    if (N > f.rows) continue;
    const int64_t rounds = V / ((int64_t)kSlab * cus);
    const int n_main = (int)(rounds * cus), rest = V - n_main * kSlab;
    const int width = q8_share(rest, cus), n_tail = (rest + width - 1) / width;
    const int tail = width <= 64 ? f.tail64 : width <= 128 ? f.tail128 : 0;
    const int64_t est = rounds * cost[0] + tail + (rounds > 0 ? kBehind : 0);
    if (rest == 0 || tail == 0 || n_tail > kMaxCutTail || est >= best.est ||
        (rounds > 0 && f.rows != 128))
      continue;
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
      case 192: f(Q8Rows<192>{}, Q8Rows<192>{}, cut, 0, l); break;
      default: f(Q8Rows<256>{}, Q8Tail<256, 64>{}, cut, 0, l); break;
    }
  }
  return S;
}

}  // namespace
}  // namespace asv
