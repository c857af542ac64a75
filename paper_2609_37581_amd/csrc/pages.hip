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

}  // namespace

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
