// The page table of the 8-bit cache: room reserved, sequences forked, pages
// given up.  Integers only; results are those of serving the requests in
// order, whatever order the waves run in.
//
// A page is free when no slot holds it (ref 0), so giving up and sharing pages
// is counting, which atomics do in any order with one result; a list of free
// pages would have to be kept in order instead.  Reserving takes the lowest
// free pages: one workgroup scans the counts, which is latency-bound (32 KB of
// counts a step).
#include "cache.hpp"

namespace trevs {
namespace {

constexpr int kListThreads = 256;
constexpr int kReserveThreads = 1024;
static_assert(kReserveThreads == TREVS_MAX_PAGE_REQUESTS, "a thread to a request");

__device__ __forceinline__ int request_slot(const PagesArgs& a, const int32_t* slots, int i) {
  return slot_of(slots, i, a.n_slots);
}
__device__ __forceinline__ int pages_of(const PagesArgs& a, long long tokens) {
  return (int)((tokens + (1 << a.page_shift) - 1) >> a.page_shift);
}

__global__ __launch_bounds__(kListThreads) void fork_kernel(PagesArgs a, const int32_t* src, const int32_t* dst,
                                                            const int32_t* n_tokens, int32_t* done) {
  const int i = blockIdx.x, tid = threadIdx.x;
  const int from = src[i], to = dst[i];
  bool bad = from < 0 || from >= a.n_slots || to < 0 || to >= a.n_slots;
  const int to_len = bad ? 0 : a.len[to];
  bad = bad || to_len != 0;
  for (int j = tid; j < a.n; j += kListThreads) {
    const int d = dst[j];
    bad = bad || d == from || (j < i && d == to);
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) done[i] = 0;
    return;
  }
  const int len = slot_len(a.len, from, a.max_pages << a.page_shift);
  const int n = n_tokens ? min(max(n_tokens[i], 0), len) : len;
  const int pages = pages_of(a, n);
  for (int j = tid; j < pages; j += kListThreads) {
    const int p = a.table[(size_t)from * a.max_pages + j];
    a.table[(size_t)to * a.max_pages + j] = p;
    if (p >= 0 && p < a.n_pages) atomicAdd(&a.ref[p], 1);
  }
  if (tid == 0) {
    a.len[to] = n;
    done[i] = 1;
  }
}

__global__ __launch_bounds__(kListThreads) void free_kernel(PagesArgs a, const int32_t* slots, const int32_t* keep) {
  const int i = blockIdx.x, tid = threadIdx.x;
  const int slot = request_slot(a, slots, i);
  bool bad = slot < 0;
  if (slots)
    for (int j = tid; j < i; j += kListThreads) bad = bad || slots[j] == slot;
  const int len = slot_len(a.len, slot, a.max_pages << a.page_shift);
  if (__syncthreads_or(bad)) return;  // (every thread has read len)
  const int k = keep ? min(max(keep[i], 0), len) : 0;
  for (int j = pages_of(a, k) + tid; j < pages_of(a, len); j += kListThreads) {
    int32_t* entry = a.table + (size_t)slot * a.max_pages + j;
    const int p = *entry;
    *entry = -1;
    if (p >= 0 && p < a.n_pages && atomicSub(&a.ref[p], 1) <= 0) atomicAdd(&a.ref[p], 1);  // never below 0
  }
  if (tid == 0) a.len[slot] = k;
}

// Sum over the workgroup before this thread, and the workgroup's total.
__device__ __forceinline__ int block_excl_scan(int v, int* lds, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int incl = wave_incl_scan(v, lane);
  if (lane == 63) lds[w] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int k = 0; k < kReserveThreads / 64; ++k) {
    before += k < w ? lds[k] : 0;
    total += lds[k];
  }
  __syncthreads();
  return before + incl - v;
}

// Which of the 8 pages from p on are free, as bits.
__device__ __forceinline__ uint32_t free_bits(const PagesArgs& a, long long p) {
  uint32_t bits = 0;
  if (p + 8 <= a.n_pages && (reinterpret_cast<uintptr_t>(a.ref) & 15) == 0) {
    const u32x4 x = ldg16(a.ref + p), y = ldg16(a.ref + p + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) bits |= ((int)x[k] <= 0 ? 1u << k : 0u) | ((int)y[k] <= 0 ? 16u << k : 0u);
  } else {
    for (int k = 0; k < 8; ++k)
      if (p + k < a.n_pages && a.ref[p + k] <= 0) bits |= 1u << k;
  }
  return bits;
}

__global__ __launch_bounds__(kReserveThreads) void reserve_kernel(PagesArgs a, const int32_t* slots,
                                                                  const int32_t* n_new, int32_t* granted,
                                                                  int32_t* copy_src, int32_t* copy_dst) {
  __shared__ __align__(16) int l_slot[kReserveThreads], l_last[kReserveThreads];
  __shared__ int l_off[kReserveThreads + 1], l_col[kReserveThreads];
  __shared__ int l_need[kReserveThreads], l_ref[kReserveThreads], l_first[kReserveThreads], l_cow[kReserveThreads];
  __shared__ int red[kReserveThreads / 64];
  __shared__ unsigned long long l_sum;
  __shared__ int l_total;
  const int i = threadIdx.x, wave0 = i & ~63;
  const int max_tokens = a.max_pages << a.page_shift;
  // the first pages' counts are on their way while the requests are read
  const uint32_t bits0 = free_bits(a, 8 * i);
  int slot = -1, want_new = 0, len = 0;
  if (i < a.n) {
    slot = request_slot(a, slots, i);
    want_new = n_new[i];
    len = slot_len(a.len, slot, max_tokens);
  }
  l_slot[i] = slot;
  if (i == 0) l_sum = 0;
  __syncthreads();
  bool ok = slot >= 0 && want_new >= 1 && want_new <= max_tokens - len;
  // (waves without requests pass by the loops over the earlier ones; four entries a read)
  const int4* slots4 = reinterpret_cast<const int4*>(l_slot);
  if (slots && wave0 < a.n) {
    bool same = false;
    for (int j = 0; j < min(a.n, wave0 + 64); j += 4) {
      const int4 x = slots4[j >> 2];
      same = same || (j < i && x.x == slot) || (j + 1 < i && x.y == slot) || (j + 2 < i && x.z == slot) ||
             (j + 3 < i && x.w == slot);
    }
    ok = ok && !same;
  }
  // the last page, if rows would be appended to it
  const int have = pages_of(a, len), want = ok ? pages_of(a, (long long)len + want_new) : have;
  int last = -1;
  if (ok && (len & ((1 << a.page_shift) - 1))) {
    const int p = a.table[(size_t)slot * a.max_pages + have - 1];
    last = p >= 0 && p < a.n_pages ? p : -1;
  }
  const int refs = last >= 0 ? a.ref[last] : 0;
  l_last[i] = last;
  l_ref[i] = refs;
  __syncthreads();
  // of the requests that end in one shared page, each takes a copy until one holder is left
  int rank = 0, first = i;
  const int4* last4 = reinterpret_cast<const int4*>(l_last);
  if (__any(last >= 0)) {
    auto earlier = [&](int j, int x) {
      const bool same = j < i && last >= 0 && x == last;
      rank += same;
      first = same ? min(first, j) : first;
    };
    for (int j = 0; j < min(a.n, wave0 + 64); j += 4) {
      const int4 x = last4[j >> 2];
      earlier(j, x.x);
      earlier(j + 1, x.y);
      earlier(j + 2, x.z);
      earlier(j + 3, x.w);
    }
  }
  bool cow = last >= 0 && rank < refs - 1;
  int need = ok ? want - have + cow : 0;
  l_need[i] = ok ? want - have : -1;  // without the copy; -1: refused already
  l_first[i] = first;
  // all needs, which may pass 32 bits: their halves are summed by the wave, the waves' sums by 64-bit adds
  // (one such add a thread took 3.8 us)
  const uint32_t low = __builtin_amdgcn_readlane(wave_incl_scan(need & 0xffff, 0), 63);
  const uint32_t high = __builtin_amdgcn_readlane(wave_incl_scan(need >> 16, 0), 63);
  if ((i & 63) == 0 && (low | high)) atomicAdd(&l_sum, ((unsigned long long)high << 16) + low);
  __syncthreads();
  const unsigned long long sum = l_sum;
  // free pages, until they cover the requests
  long long n_free = 0;
  for (long long p0 = 0; p0 < a.n_pages && (unsigned long long)n_free < sum; p0 += 8 * kReserveThreads) {
    int total;
    block_excl_scan(__popc(p0 ? free_bits(a, p0 + 8 * i) : bits0), red, total);
    n_free += total;
  }
  if (sum > (unsigned long long)n_free) {
    // a shortage: in order, each request that still fits is served
    l_cow[i] = 0;  // copies taken so far of the page of which i is the first request
    __syncthreads();
    if (i == 0) {
      long long left = n_free;
      int at = 0;
      for (int j = 0; j < a.n; ++j) {
        l_off[j] = at;
        if (l_need[j] < 0) continue;
        const bool c = l_last[j] >= 0 && l_cow[l_first[j]] < l_ref[j] - 1;
        const int nj = l_need[j] + c;
        if (nj > left) {
          l_need[j] = -1;
          continue;
        }
        if (c) ++l_cow[l_first[j]];
        l_last[j] = c ? l_last[j] : -1;  // from here on: the page copied
        left -= nj;
        at += nj;
      }
      l_total = at;
    }
    __syncthreads();
    ok = i < a.n && l_need[i] >= 0;
    cow = ok && l_last[i] >= 0;
    need = ok ? l_need[i] + cow : 0;
    if (i >= a.n) l_off[i] = l_total;
    if (i == 0) l_off[kReserveThreads] = l_total;
  } else {
    int total;
    l_off[i] = block_excl_scan(need, red, total);
    if (i == 0) l_off[kReserveThreads] = l_total = total;
  }
  l_cow[i] = cow;
  l_col[i] = have - cow;
  __syncthreads();
  const int total = l_total;
  const int reach = a.n > 1 ? 1 << (31 - __builtin_clz(a.n - 1)) : 0;  // largest power of two below n
  // the r-th lowest free page goes to the request whose range holds r
  int base = 0;
  for (long long p0 = 0; p0 < a.n_pages && base < total; p0 += 8 * kReserveThreads) {
    const long long p = p0 + 8 * i;
    uint32_t bits = p0 ? free_bits(a, p) : bits0;
    int sum_step;
    int r = base + block_excl_scan(__popc(bits), red, sum_step);
    base += sum_step;
    if (bits && r < total) {
      int at = 0;  // the last request whose range begins at or before r
      for (int step = reach; step > 0; step >>= 1) at += l_off[at + step] <= r ? step : 0;
      while (bits && r < total) {
        while (l_off[at + 1] <= r) ++at;  // (l_off[n] = total)
        const int k = __builtin_ctz(bits), o = r - l_off[at];
        bits &= bits - 1;
        a.table[(size_t)l_slot[at] * a.max_pages + l_col[at] + o] = (int)(p + k);
        a.ref[p + k] = 1;
        if (o == 0 && l_cow[at]) copy_dst[at] = (int)(p + k);
        ++r;
      }
    }
  }
  if (i >= a.n) return;
  granted[i] = ok ? want_new : 0;
  copy_src[i] = cow ? last : -1;
  if (!cow) copy_dst[i] = -1;
  if (ok) a.len[slot] = len + want_new;
  if (cow) atomicSub(&a.ref[last], 1);
}

// Pages for what evict_select_kernel chose to keep, from those that are free before
// the call; a thread to a request.  Bound by latency, as reserving is (4 requests or 64:
// 6 us).
__global__ __launch_bounds__(kReserveThreads) void evict_pages_kernel(EvictArgs e, PagesArgs a) {
  __shared__ int l_slot[kReserveThreads], l_off[kReserveThreads + 1], l_col[kReserveThreads], l_need[kReserveThreads];
  __shared__ int red[kReserveThreads / 64];
  __shared__ int l_total;
  const int i = threadIdx.x;
  const uint32_t bits0 = free_bits(a, 8 * i);
  EvictInfo x = {-1, 0, 0, 0, 0};
  if (i < a.n) x = e.info[i];
  bool ok = x.slot >= 0;
  int need = ok && x.moved < x.n ? pages_of(a, x.n) - x.first_page : 0;
  l_slot[i] = x.slot;
  l_col[i] = x.first_page;
  l_need[i] = ok ? need : -1;
  // all needs, which may pass 32 bits, by halves
  int low, high;
  block_excl_scan(need & 0xffff, red, low);
  block_excl_scan(need >> 16, red, high);
  const long long sum = ((long long)high << 16) + low;
  long long n_free = 0;
  for (long long p0 = 0; p0 < a.n_pages && n_free < sum; p0 += 8 * kReserveThreads) {
    int total;
    block_excl_scan(__popc(p0 ? free_bits(a, p0 + 8 * i) : bits0), red, total);
    n_free += total;
  }
  if (sum > n_free) {
    // a shortage: in order, each request that still fits is served
    if (i == 0) {
      int at = 0;
      for (int j = 0; j < a.n; ++j) {
        l_off[j] = at;
        if (l_need[j] < 0) continue;
        if (l_need[j] > n_free - at)
          l_need[j] = -1;
        else
          at += l_need[j];
      }
      l_total = at;
    }
    __syncthreads();
    ok = l_need[i] >= 0;
    if (i >= a.n) l_off[i] = l_total;
    if (i == 0) l_off[kReserveThreads] = l_total;
  } else {
    int total;
    l_off[i] = block_excl_scan(need, red, total);
    if (i == 0) l_off[kReserveThreads] = l_total = total;
  }
  __syncthreads();
  const int total = l_total;
  const int reach = a.n > 1 ? 1 << (31 - __builtin_clz(a.n - 1)) : 0;  // largest power of two below n
  int base = 0;
  for (long long p0 = 0; p0 < a.n_pages && base < total; p0 += 8 * kReserveThreads) {
    const long long p = p0 + 8 * i;
    uint32_t bits = p0 ? free_bits(a, p) : bits0;
    int sum_step;
    int r = base + block_excl_scan(__popc(bits), red, sum_step);
    base += sum_step;
    int at = 0;  // the last request whose range begins at or before r
    if (bits && r < total)
      for (int step = reach; step > 0; step >>= 1) at += l_off[at + step] <= r ? step : 0;
    while (bits && r < total) {
      while (l_off[at + 1] <= r) ++at;  // (l_off[n] = total)
      const int k = __builtin_ctz(bits);
      bits &= bits - 1;
      a.table[(size_t)l_slot[at] * a.max_pages + l_col[at] + r - l_off[at]] = (int)(p + k);
      a.ref[p + k] = 1;
      ++r;
    }
  }
  if (i >= a.n) return;
  e.n_evicted[i] = ok ? x.len - x.n : 0;
  if (x.slot >= 0 && !ok) e.info[i].slot = -1;
}

// A group's entries: the slot of each (-1: the entry does nothing) and the entry
// whose sequence it takes over (its own: it keeps what it has).
struct Group {
  int slot[TREVS_MAX_BEAMS], src[TREVS_MAX_BEAMS], len[TREVS_MAX_BEAMS];
};
__device__ __forceinline__ void read_group(const PagesArgs& a, int g, int width, const int32_t* slots,
                                           const int32_t* parent, Group& s) {
  const int tid = threadIdx.x;
  for (int w = tid; w < width; w += blockDim.x) {
    const int i = g * width + w, slot = request_slot(a, slots, i);
    s.slot[w] = slot;
    s.len[w] = slot_len(a.len, slot, a.max_pages << a.page_shift);
  }
  __syncthreads();
  if (slots) {  // an earlier entry's slot
    const int n = (g + 1) * width;
    for (int e = tid; e < n * width; e += blockDim.x) {
      const int w = e / n, j = e - w * n;
      if (j < g * width + w && slots[j] == slots[g * width + w]) s.slot[w] = -1, s.len[w] = 0;
    }
    __syncthreads();
  }
  for (int w = tid; w < width; w += blockDim.x) {
    const int p = parent[g * width + w];
    s.src[w] = s.slot[w] >= 0 && p >= 0 && p < width && s.slot[p] >= 0 ? p : w;
  }
  __syncthreads();
}

constexpr int kReorderThreads = 128;
constexpr int kReorderHeld = TREVS_MAX_BEAMS * kReorderThreads;  // entries that a workgroup holds

// A thread holds a column of the group, so reads are done before writes.  (The columns lie
// in as much LDS as the beams need, or too few workgroups fit a CU: 16 x 8 beams of 1.3 k to
// 16.6 k tokens 7.6 us, 12.6 with room for 64.)
__global__ __launch_bounds__(kReorderThreads) void reorder_scores_kernel(PagesArgs a, int width, const int32_t* slots,
                                                                         const int32_t* parent, float* score) {
  __shared__ Group s;
  extern __shared__ float held_scores[];
  const int tid = threadIdx.x, g = blockIdx.y;
  read_group(a, g, width, slots, parent, s);
  int longest = 0;
  for (int w = 0; w < width; ++w) longest = max(longest, s.len[w]);
  const size_t row = (size_t)a.max_pages << a.page_shift;
  float* held = held_scores + tid;
  for (int j = blockIdx.x * kReorderThreads + tid; j < longest; j += gridDim.x * kReorderThreads) {
#pragma unroll 8
    for (int w = 0; w < width; ++w) held[w * kReorderThreads] = s.slot[w] >= 0 ? score[s.slot[w] * row + j] : 0.f;
    for (int w = 0; w < width; ++w) {
      const int p = s.src[w];
      if (p != w && j < max(s.len[w], s.len[p]))
        score[s.slot[w] * row + j] = j < s.len[p] ? held[p * kReorderThreads] : 0.f;
    }
  }
}

// One workgroup to a group, since the lengths that it reads are written at the end: with
// fewer beams it has more threads, so that it goes over the pages at once (16 x 8 beams
// of 22 to 261 pages: 13.8 us with 128 threads, 8 so, 6.3 with the counts of eight beams
// awaited together).
__global__ __launch_bounds__(1024) void reorder_kernel(PagesArgs a, int width, const int32_t* slots,
                                                       const int32_t* parent) {
  __shared__ Group s;
  __shared__ int held[kReorderHeld];
  const int tid = threadIdx.x, g = blockIdx.x, n = blockDim.x;
  read_group(a, g, width, slots, parent, s);
  int longest = 0;
  for (int w = 0; w < width; ++w) longest = max(longest, s.len[w]);
  for (int j = tid; j < pages_of(a, longest); j += n) {
#pragma unroll 8
    for (int w = 0; w < width; ++w)
      held[w * n + tid] = s.slot[w] >= 0 ? a.table[(size_t)s.slot[w] * a.max_pages + j] : -1;
    // (eight beams at a time: their counts come back together)
    for (int w0 = 0; w0 < width; w0 += 8) {
      int old[8], left[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int w = w0 + i;
        old[i] = -1;
        left[i] = 1;
        if (w >= width) continue;
        const int p = s.src[w], w_pages = pages_of(a, s.len[w]), p_pages = pages_of(a, s.len[p]);
        if (p == w || j >= max(w_pages, p_pages)) continue;
        const int was = j < w_pages ? held[w * n + tid] : -1, now = j < p_pages ? held[p * n + tid] : -1;
        if (was == now) continue;
        a.table[(size_t)s.slot[w] * a.max_pages + j] = now;
        if (now >= 0 && now < a.n_pages) atomicAdd(&a.ref[now], 1);
        if (was >= 0 && was < a.n_pages) old[i] = was;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (old[i] >= 0) left[i] = atomicSub(&a.ref[old[i]], 1);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (left[i] <= 0) atomicAdd(&a.ref[old[i]], 1);  // never below 0
    }
  }
  for (int w = tid; w < width; w += n)
    if (s.src[w] != w) a.len[s.slot[w]] = s.len[s.src[w]];
}

}  // namespace

hipError_t launch_evict_pages(const EvictArgs& e, hipStream_t s) {
  PagesArgs a;
  a.table = const_cast<int32_t*>(e.c.table);
  a.len = const_cast<int32_t*>(e.c.len);
  a.ref = e.ref;
  a.n_pages = e.c.n_pages;
  a.n_slots = e.c.n_slots;
  a.max_pages = e.c.max_pages;
  a.page_shift = e.page_shift;
  a.n = e.B;
  hipLaunchKernelGGL(evict_pages_kernel, dim3(1), dim3(kReserveThreads), 0, s, e, a);
  return hipGetLastError();
}

hipError_t launch_pages_reorder(const PagesArgs& a, int groups, int width, const int32_t* slots, const int32_t* parent,
                                float* score, hipStream_t s) {
  if (score) {
    const long long tokens = (long long)a.max_pages << a.page_shift;
    const int blocks = (int)min((tokens + kReorderThreads - 1) / kReorderThreads, 4096LL / groups + 1);
    hipLaunchKernelGGL(reorder_scores_kernel, dim3(blocks, groups), dim3(kReorderThreads),
                       width * kReorderThreads * sizeof(float), s, a, width, slots, parent, score);
  }
  int threads = 1024;
  while (threads * width > kReorderHeld || (threads > 64 && threads >= 2 * a.max_pages)) threads >>= 1;
  hipLaunchKernelGGL(reorder_kernel, dim3(groups), dim3(threads), 0, s, a, width, slots, parent);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const PagesArgs& a, const int32_t* slots, const int32_t* n_new, int32_t* granted,
                                int32_t* copy_src, int32_t* copy_dst, hipStream_t s) {
  hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kReserveThreads), 0, s, a, slots, n_new, granted, copy_src,
                     copy_dst);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesArgs& a, const int32_t* src, const int32_t* dst, const int32_t* n_tokens,
                             int32_t* done, hipStream_t s) {
  hipLaunchKernelGGL(fork_kernel, dim3(a.n), dim3(kListThreads), 0, s, a, src, dst, n_tokens, done);
  return hipGetLastError();
}

hipError_t launch_pages_free(const PagesArgs& a, const int32_t* slots, const int32_t* keep, hipStream_t s) {
  hipLaunchKernelGGL(free_kernel, dim3(a.n), dim3(kListThreads), 0, s, a, slots, keep);
  return hipGetLastError();
}

}  // namespace trevs
