// Buckets of the relative position bias, as the kernels look them up.  Plain C++ apart from the attributes, so that the indexing is also built and run without a GPU.
#pragma once
#include <stdint.h>

namespace dp {

constexpr int REL_MAX_BUCKETS = 512, REL_MAX_DISTANCE = 1024;

struct RelBucketsK {
  int n_buckets, per_side, half;      // buckets in all, of one direction, of one distance each
  int bidirectional;
  int lo, hi;                         // the bucket of every distance <= lo is lo's, of every one >= hi is hi's
};
// Least distance of bucket half + k, two to a word; past the last 0xFFFF.  A kernel argument of its own: indexed inside the other arguments, it would send
// all of them through scratch memory.
struct RelStarts { uint32_t of[REL_MAX_BUCKETS / 4]; };

// Counts the starts that are not above the distance, sixteen (eight scalar registers) at a time: no lane waits for a memory access of its own.
__host__ __device__ __forceinline__ int rel_bucket(const RelBucketsK& r, const RelStarts& st, int dist) {
  const int far = dist < 0 ? -dist : dist, n = r.bidirectional || dist < 0 ? far : 0, side = r.bidirectional && dist > 0 ? r.per_side : 0;
  int k = r.half - 1;
  for (int w = 0; w < (r.per_side - r.half + 1) / 2; w += 8) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const uint32_t two = st.of[w + u];
      k += (int)(two & 0xFFFFu) <= n;
      k += (int)(two >> 16) <= n;
    }
  }
  return side + (n < r.half ? n : k);
}

// Least distance of bucket k of a direction, and for k = per_side, where no start is held (512 buckets of one direction fill the array), more than any in the sums' reach.
__host__ __device__ __forceinline__ uint32_t rel_start(const RelBucketsK& r, const RelStarts& st, int k) {
  if (k >= r.per_side) return 0x7FFFu;
  if (k < r.half) return (uint32_t)k;
  const uint32_t two = st.of[(k - r.half) / 2];
  return (k - r.half) & 1 ? two >> 16 : two & 0xFFFFu;
}

}  // namespace dp
