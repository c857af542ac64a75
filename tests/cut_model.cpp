// The cut of an attention call's steps, on the host (test_cache_cut.py).
#define __host__
#define __device__
#define __forceinline__ inline
#include "../paper_2609_37581_amd/csrc/cut.hpp"

extern "C" {
int cut_n(int total, int workgroups) { return trevs::Cut(total, workgroups).n; }
int cut_start(int total, int workgroups, int w) { return trevs::Cut(total, workgroups).start(w); }
int cut_owner(int total, int workgroups, int step) { return trevs::Cut(total, workgroups).owner(step); }
}
