// The cut of an attention call's steps, on the host (test_cache_cut.py).
#define __host__
#define __device__
#define __forceinline__ inline
#include "../paper_2609_37581_amd/csrc/cut.hpp"

extern "C" {
int cut_n(int total, int workgroups, int side) { return trevs::Cut(total, workgroups, side).n; }
int cut_start(int total, int workgroups, int side, int w) { return trevs::Cut(total, workgroups, side).start(w); }
int cut_owner(int total, int workgroups, int side, int step) { return trevs::Cut(total, workgroups, side).owner(step); }
}
