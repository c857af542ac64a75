// Which tokens of a cached sequence stay: the first and last ones, and of those
// between the highest scores.
//
// One workgroup to a sequence: the choice is a stable top-K over keys held in
// registers, E of them a thread, in which the tokens that always stay have the largest
// key and NaN the smallest.  Bound by latency: a count and a barrier for each bit of the
// key.  Sequences of more than 32,768 tokens read the scores again for each bit (four of
// 20 k to 32 k tokens 35 us, of 34 k to 60 k 280).
#include "cache.hpp"
#include "select.hpp"

namespace trevs {
namespace {

__device__ __forceinline__ uint32_t score_key(float s) { return s != s ? 0u : f2key(s); }

// Calls emit(j, kept, kept tokens before j) for every token j < L, n < L of which are kept.
// The n-th largest key is found bit by bit (few keys a thread: two bits), counting with
// ballots: the scores of a sequence share few exponents, so a histogram's atomics would
// meet in few bins (up to 16,547 tokens: the selection of select.hpp 25 us, this way 22.5;
// up to 700 tokens 10, which the loads that wait for each other take).
template <int E, class Emit>
__device__ __forceinline__ void select_held(const float* score, int L, int n, int first, int last, Emit emit,
                                            SelectShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t key[E];
#pragma unroll
  for (int e = 0; e < E; ++e) key[e] = score_key(score[min(e * kSelThreads + tid, L - 1)]);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int j = e * kSelThreads + tid;
    if (j < first || j >= L - last) key[e] = 0xffffffffu;
    if (j >= L) key[e] = 0u;  // (as NaN, but never emitted; nothing is counted by a bound of 0)
  }
  // BITS bits of the threshold at a time: the keys that reach each of the values that they can have
  constexpr int BITS = E <= 4 ? 2 : 1, kSteps = 32 / BITS, kValues = (1 << BITS) - 1;
  for (int i = tid; i < kSteps * kValues; i += kSelThreads) sh.hist[i] = 0u;
  __syncthreads();
  uint32_t thr = 0;
  for (int step = 0; step < kSteps; ++step) {
    const int shift = 32 - BITS * (step + 1);
    int count[kValues] = {};
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int v = 0; v < kValues; ++v) count[v] += __popcll(__ballot(key[e] >= (thr | ((v + 1u) << shift))));
    uint32_t* counts = sh.hist + step * kValues;
#pragma unroll
    for (int v = 0; v < kValues; ++v)
      if (lane == v) atomicAdd(&counts[v], (uint32_t)count[v]);
    __syncthreads();
    uint32_t digit = 0;
    bool exact = false;
#pragma unroll
    for (int v = 0; v < kValues; ++v) {
      const int total = __builtin_amdgcn_readfirstlane((int)counts[v]);
      if (total >= n) {
        digit = v + 1;
        exact = total == n;
      }
    }
    thr |= digit << shift;
    if (exact) break;
  }
  __syncthreads();  // the counts are read before the words below are written
  // above the threshold, and equal to it, before each token
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const bool in = e * kSelThreads + tid < L;
    const uint64_t above = __ballot(in && key[e] > thr), ties = __ballot(in && key[e] == thr);
    if (lane == 0) sh.wcnt[e * kSelWaves + wave] = (uint32_t)__popcll(above) | ((uint32_t)__popcll(ties) << 16);
  }
  __syncthreads();
  // (packed sums of up to 65,536 of either: each half's exclusive ones fit it, the sum of all `above` is n at most)
  if (wave == 0) {
    constexpr int kPer = (E * kSelWaves + 63) / 64;
    uint32_t c[kPer], sum = 0;
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const int i = lane * kPer + q;
      c[q] = i < E * kSelWaves ? sh.wcnt[i] : 0u;
      sum += c[q];
    }
    uint32_t run = wave_incl_scan_u32(sum) - sum;
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const int i = lane * kPer + q;
      if (i < E * kSelWaves) sh.wcnt[i] = run;
      run += c[q];
    }
    if (lane == 63) sh.total = (int)(run & 0xffffu);
  }
  __syncthreads();
  const int need = n - sh.total;  // ties kept, lowest index first
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int j = e * kSelThreads + tid;
    const bool in = j < L, over = in && key[e] > thr, tie = in && key[e] == thr;
    const uint64_t below = (1ull << lane) - 1;
    const uint32_t base = sh.wcnt[e * kSelWaves + wave];
    const int na = (int)(base & 0xffffu) + __popcll(__ballot(over) & below);
    const int nt = (int)(base >> 16) + __popcll(__ballot(tie) & below);
    if (in) emit(j, over || (tie && nt < need), na + min(nt, need));
  }
}

// The same for any length: a thread owns `per` tokens in a row.
template <class Emit>
__device__ void select_streamed(const float* score, int L, int n, int first, int last, Emit emit, SelectShared& sh) {
  const int per = (L + kSelThreads - 1) / kSelThreads;
  const int j0 = (int)min((long long)threadIdx.x * per, (long long)L), j1 = min(j0 + per, L);
  auto key = [&](int j) { return j < first || j >= L - last ? 0xffffffffu : score_key(score[j]); };
  uint32_t thr = 0;  // the n-th largest key
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t least = thr | (1u << bit);
    int c = 0, total;
#pragma unroll 8
    for (int j = threadIdx.x; j < L; j += kSelThreads) c += key(j) >= least;
    block_excl_scan(c, sh, total);
    if (total >= n) thr = least;
    if (total == n) break;
  }
  int above = 0, ties = 0, n_above, n_ties;
  for (int j = j0; j < j1; ++j) {
    const uint32_t k = key(j);
    above += k > thr;
    ties += k == thr;
  }
  above = block_excl_scan(above, sh, n_above);
  ties = block_excl_scan(ties, sh, n_ties);
  const int need = n - n_above;
  for (int j = j0; j < j1; ++j) {
    const uint32_t k = key(j);
    emit(j, k > thr || (k == thr && ties < need), above + min(ties, need));
    above += k > thr;
    ties += k == thr;
  }
}

__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(EvictArgs a) {
  __shared__ SelectShared sh;
  __shared__ int s_first;
  const int b = blockIdx.x, tid = threadIdx.x;
  const int slot = slot_of(a.slots, b, a.c.n_slots);
  bool bad = slot < 0;
  if (a.slots)
    for (int j = tid; j < b; j += kSelThreads) bad = bad || a.slots[j] == slot;
  if (tid == 0) s_first = INT32_MAX;
  int32_t* kept = a.kept_idx + (size_t)b * a.n_keep;
  const int L = slot_len(a.c.len, slot, a.c.max_pages << a.page_shift);
  const int least = max(a.n_first + a.n_last, 1);
  const int n = a.keep ? min(max(a.keep[b], least), a.n_keep) : a.n_keep;
  if (__syncthreads_or(bad) || L <= n) {
    for (int i = tid; i < a.n_keep; i += kSelThreads) kept[i] = -1;
    if (tid == 0) a.info[b] = EvictInfo{-1, 0, 0, 0, 0};
    return;
  }
  const float* score = a.score + ((size_t)slot * a.c.max_pages << a.page_shift);
  int gone = INT32_MAX;  // this thread's first evicted token
  auto emit = [&](int j, bool keep, int before) {
    if (!keep)
      gone = min(gone, j);
    else if (before < n)  // (exactly n are kept; the bound guards memory)
      kept[before] = j;
  };
  if (L <= 1 * kSelThreads)
    select_held<1>(score, L, n, a.n_first, a.n_last, emit, sh);
  else if (L <= 4 * kSelThreads)
    select_held<4>(score, L, n, a.n_first, a.n_last, emit, sh);
  else if (L <= 12 * kSelThreads)
    select_held<12>(score, L, n, a.n_first, a.n_last, emit, sh);
  else if (L <= 20 * kSelThreads)
    select_held<20>(score, L, n, a.n_first, a.n_last, emit, sh);
  else if (L <= 32 * kSelThreads)
    select_held<32>(score, L, n, a.n_first, a.n_last, emit, sh);
  else
    select_streamed(score, L, n, a.n_first, a.n_last, emit, sh);
  if (gone != INT32_MAX) atomicMin(&s_first, gone);
  for (int i = n + tid; i < a.n_keep; i += kSelThreads) kept[i] = -1;
  __syncthreads();
  // tokens before the first evicted one stay where they are: kept[i] = i below it, and above i from there on
  const int moved = min(s_first, n);
  const int page = 1 << a.page_shift, want = (n + page - 1) >> a.page_shift;
  const int from = moved < n ? moved >> a.page_shift : want;
  for (int j = from + tid; j < (L + page - 1) >> a.page_shift; j += kSelThreads)
    a.old[(size_t)b * a.c.max_pages + j] = a.c.table[(size_t)slot * a.c.max_pages + j];
  if (tid == 0) a.info[b] = EvictInfo{slot, L, n, moved, from};
}

}  // namespace

hipError_t launch_evict_select(const EvictArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(evict_select_kernel, dim3(a.B), dim3(kSelThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace trevs
