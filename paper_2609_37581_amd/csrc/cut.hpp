// How the steps of a cut attention call are dealt to its workgroups.
#pragma once

namespace trevs {

// `total` steps, those of all tiles one after the other, in n equal pieces.
// The launch's workgroups are counted from the longest that the sequences may
// be, `total` from what they are: n is the smaller of the two, so that every
// one of the first n has a step and the workgroups between a tile's first and
// its last have all left their sums; the others do nothing.  (Fewer and longer
// pieces, 4 steps for the 4 waves of a workgroup, end more often in a second
// tile: a token of 4 sequences of 1187 under a table of 16 times that, 15.1 us,
// and 12.2 this way.)
struct Cut {
  int total, n;
  __host__ __device__ __forceinline__ Cut(int total_, int workgroups)
      : total(total_), n(total_ < workgroups ? total_ : workgroups) {}
  // The first step of workgroup w (total for w = n).
  __host__ __device__ __forceinline__ int start(int w) const { return (int)((long long)w * total / n); }
  // The workgroup that holds a step.
  __host__ __device__ __forceinline__ int owner(int step) const {
    int w = (int)((long long)step * n / total);
    while (start(w + 1) <= step) ++w;
    return w;
  }
};

}  // namespace trevs
