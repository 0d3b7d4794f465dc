// The bucket lookups of the relative position bias for every number of buckets and both kinds of directions, built with the array bounds checked.  The starts
// are laid down here as the library holds them: two to a word, 0xFFFF past the last.
#define __host__
#define __device__
#define __forceinline__ inline
#include "../paper_2405_01248_amd/csrc/dp_relbias_buckets.h"

#include <cstdio>
#include <cstring>

int main() {
  for (int both = 0; both < 2; ++both)
    for (int n = both ? 4 : 2; n <= dp::REL_MAX_BUCKETS; n += both ? 2 : 1) {
      dp::RelBucketsK r{};
      r.n_buckets = n; r.bidirectional = both; r.per_side = both ? n / 2 : n; r.half = r.per_side / 2;
      dp::RelStarts st;
      memset(&st, 0xFF, sizeof(st));
      const int rest = r.per_side - r.half;
      auto start = [&](int k) { return k < r.half ? k : r.half + 2 * (k - r.half); };      // (rising; up to 768)
      for (int k = 0; k < rest; ++k) {
        uint32_t& two = st.of[k / 2];
        two = k % 2 ? (two & 0xFFFFu) | (uint32_t)start(r.half + k) << 16 : (two & 0xFFFF0000u) | (uint32_t)start(r.half + k);
      }
      for (int k = 0; k <= r.per_side; ++k) {
        const int want = k == r.per_side ? 0x7FFF : start(k);
        if ((int)dp::rel_start(r, st, k) != want) { printf("start of bucket %d of %d (%d): %d, not %d\n", k, n, both, (int)dp::rel_start(r, st, k), want); return 1; }
      }
      for (int dist = -1200; dist <= 1200; ++dist) {
        const int d = both ? (dist < 0 ? -dist : dist) : (dist < 0 ? -dist : 0);
        int k = 0;
        while (k + 1 < r.per_side && start(k + 1) <= d) ++k;
        const int want = k + (both && dist > 0 ? r.per_side : 0);
        if (dp::rel_bucket(r, st, dist) != want) { printf("bucket of %d of %d (%d): %d, not %d\n", dist, n, both, dp::rel_bucket(r, st, dist), want); return 1; }
      }
    }
  printf("relative bias buckets: ok\n");
  return 0;
}
