// Host check of the launches of the 8-bit LM head (q8_launches, from the library's header): over row counts,
// vocabularies and CU counts, with records and with stored logits, every id and row is in exactly one tile, no
// slab is wider than its tile or starts off a multiple of 16 ids, the records of a step are as many as said and
// no more than the workspace holds, and every form of launch that the code can make is made. Exit 0 and
// "ok <launches>".
#include <cstdio>
#include <map>
#include <string>

#include "asv_q8_host.h"

using namespace asv;

int main() {
  std::map<std::string, long> seen;
  long launches = 0;
  for (int cus : {64, 228, 256, 304})
    for (const int* cost : {kQ8Records, kQ8Logits})
      for (int N : {1, 64, 65, 128, 129, 192, 193, 256, 257, 333, 512, 640, 2048})
        for (int V = 1; V < 300000; V += V < 3000 ? 13 : 211) {
          int64_t next = 0, records = 0;
          bool bad = false;
          const int S = q8_launches(N, V, cus, cost, [&](auto m, auto t, const SlabCut& c, int n_tail,
                                                         const asv_k1_launch& k) {
            using M = decltype(m);
            using T = decltype(t);
            ++launches;
            bad |= M::TR != T::TR || k.row_tiles != (N + M::TR - 1) / M::TR;
            bad |= (c.n_main > 0 && (c.width > M::TV || c.width % 16 != 0)) || c.v_first % 16 != 0;
            bad |= n_tail % k.row_tiles != 0 || c.slab0 != records;
            const int tails = n_tail / k.row_tiles;
            // the ids: main slabs, the tail's (of the main family without a tail of its own)
            const bool tailed = n_tail > 0;
            bad |= tailed && (c.tail_width > T::TV || c.tail_width % 16 != 0);
            bad |= c.v_first != next;
            const int64_t main_end = c.v_first + (int64_t)c.n_main * c.width;
            bad |= c.n_main > 0 && main_end - c.width >= V;      // a slab without ids
            bad |= tailed && main_end + (int64_t)(tails - 1) * c.tail_width >= V;
            next = main_end + (int64_t)tails * c.tail_width;
            records += c.n_main + tails;
            char form[64];
            std::snprintf(form, sizeof form, "%dx%d%s", c.n_main > 0 ? M::TV : 0, M::TR,
                          tailed ? ("+" + std::to_string(T::TV)).c_str() : "");
            ++seen[form];
          });
          bad |= next < V || records != S || (size_t)S * N > q8_max_records(N, V);
          if (bad) {
            std::printf("N %d, V %d, %d CUs: ids up to %lld, %lld records of %d\n", N, V, cus,
                        (long long)next, (long long)records, S);
            return 1;
          }
        }
  // up to 64 rows; 128-row tiles; taller ones
  for (const char* form : {"64x64", "128x64", "128x64+64", "256x64", "256x64+64", "256x64+128", "256x128",
                           "256x128+64", "256x128+128", "0x128+64", "0x128+128", "256x192", "256x256",
                           "0x256+64"})
    if (seen.erase(form) == 0) {
      std::printf("%s: never\n", form);
      return 1;
    }
  if (!seen.empty()) {
    std::printf("%s: unknown\n", seen.begin()->first.c_str());
    return 1;
  }
  std::printf("ok %ld\n", launches);
  return 0;
}
