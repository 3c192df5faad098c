// Host check of the 8-bit weight's LDS layout (q8_swz, from the library's header): it takes the 16-byte
// chunks of a tile to distinct places, and under the ds_read_b128 model of lds_swizzle_check.cpp (four
// passes of 16 lanes: equal lane bit 5 and equal parity of lane bits 2, 3 and 4) every fragment read,
// lane l at id base + 16 b + l % 16, chunk l / 16, puts each pass on 16 distinct bank groups. The
// workgroups' tiles begin at multiples of 16 ids, the waves' within them too. Exit 0 and "ok <reads>".
#include <cstdio>

#include "k_fp8.h"

int main() {
  static bool used[256 * 4];
  for (int r = 0; r < 256; ++r)
    for (int c = 0; c < 4; ++c) {
      const int u = asv::q8_swz(r, c);
      if (u < 0 || u >= 256 * 4 || used[u] || u / 4 != r) {
        std::printf("id %d, chunk %d: place %d\n", r, c, u);
        return 1;
      }
      used[u] = true;
    }
  int reads = 0;
  for (int base = 0; base < 256; base += 16) {
    int seen[4] = {0, 0, 0, 0};
    for (int l = 0; l < 64; ++l) {
      const int pass = ((l >> 5) & 1) * 2 + (((l >> 2) ^ (l >> 3) ^ (l >> 4)) & 1);
      const int grp = asv::q8_swz(base + l % 16, l / 16) & 15;
      if (seen[pass] & (1 << grp)) {
        std::printf("ids from %d: lane %d repeats group %d\n", base, l, grp);
        return 1;
      }
      seen[pass] |= 1 << grp;
    }
    ++reads;
  }
  std::printf("ok %d\n", reads);
  return 0;
}
