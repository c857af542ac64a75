// Beam search's selection over beams and vocabulary.
//
// Within a beam continuations rank as their logits do, so the n best of a sequence
// are among the n best of each chunk of each beam's logits.  The first kernel reads
// every logit once: a workgroup holds a chunk in registers, forms its maximum and sum
// of exponentials and lists its n best; bound by bytes, with the exponentials close
// behind.  The second joins a sequence's chunks: its log-sum-exps, then the scores of
// the listed continuations, in 64 bits, since continuations of different beams can lie
// closer together than 32 bits tell apart.
//
// The n best of many values are found by a bound: the n-th largest of the maxima of 64
// groups of them.  At least n values reach it, and hardly more do; those are listed in
// LDS and ranked by comparing each with each.  Lists that overflow (ties: banned
// tokens, all -inf) are cut exactly, by bisection over the bits and in index order.
#include "beam.hpp"
#include "common.hpp"

namespace trevs {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = kBeamChunk / kThreads;  // logits of a thread
constexpr int kVec = 8;                      // logits next to each other
constexpr int kRounds = kPer / kVec;
constexpr int kList = 512;
static_assert(TREVS_MAX_BEAM_OUT <= 64, "a group of threads to a continuation at least");

// Eight logits from any element on: rows need not be aligned.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void load_logits(const void* p, size_t i, float* x, BF16) {
  const u32x4 w = *reinterpret_cast<const u32x4_any*>(reinterpret_cast<const uint16_t*>(p) + i);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = bf16_lo(w[j]);
    x[2 * j + 1] = bf16_hi(w[j]);
  }
}
typedef uint32_t u32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void load_logits(const void* p, size_t i, float* x, F32) {
  const u32x4_any4* f = reinterpret_cast<const u32x4_any4*>(reinterpret_cast<const float*>(p) + i);
  const u32x4 a = f[0], b = f[1];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = __uint_as_float(a[j]);
    x[4 + j] = __uint_as_float(b[j]);
  }
}

// The value of rank n - 1 (from the largest; ties in lane order) among the lanes' values.
template <class T>
__device__ __forceinline__ T nth_largest(T v, int n) {
  const int lane = threadIdx.x & 63;
  int rank = 0;
  for (int l = 0; l < 64; ++l) {
    const T o = __shfl(v, l, 64);
    rank += o > v || (o == v && l < lane);
  }
  return __shfl(v, (int)__builtin_ctzll(__ballot(rank == n - 1)), 64);
}

struct ChunkShared {
  uint64_t list[kList];
  float top[64], sum[4];
  float bound;
  int count;
  int counts[2][4];
};

// Sum of v over the workgroup (`turn` alternates between calls).
__device__ __forceinline__ int block_count(int v, int turn, ChunkShared& sh) {
  v = wave_reduce_bits(v, 0, [](int a, int b) { return a + b; });
  if ((threadIdx.x & 63) == 0) sh.counts[turn][threadIdx.x >> 6] = v;
  __syncthreads();
  return sh.counts[turn][0] + sh.counts[turn][1] + sh.counts[turn][2] + sh.counts[turn][3];
}

// The list cut to exactly the chunk's n best (all of fewer): the n-th largest key by
// bisection, what lies above it, and the first of those that equal it.
__device__ __forceinline__ void exact_list(const float (&x)[kPer], int first, int V, int n, ChunkShared& sh) {
  const int tid = threadIdx.x;
  auto index = [&](int e) { return first + e / kVec * (kThreads * kVec) + tid * kVec + e % kVec; };
  // (0 for places past the vocabulary)
  auto key = [&](int e) { return index(e) < V ? f2key(x[e]) : 0u; };
  uint32_t thr = 0;
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t least = thr | (1u << bit);
    int c = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) c += key(e) >= least;
    if (block_count(c, bit & 1, sh) >= n) thr = least;
  }
  int above = 0;
#pragma unroll
  for (int e = 0; e < kPer; ++e) above += key(e) > thr;
  int before = block_count(above, 1, sh);  // (the bisection ends with turn 0)
  if (tid == 0) sh.count = 0;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < kPer; ++e)
    if (key(e) > thr) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < kList) sh.list[at] = (uint64_t)key(e) << 32 | ~(uint32_t)index(e);
    }
  if (thr > 0) {
    const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      int c = 0;
#pragma unroll
      for (int e = 0; e < kVec; ++e) c += key(k * kVec + e) == thr;
      const int incl = wave_incl_scan(c, lane);
      if (lane == 63) sh.counts[k & 1][wave] = incl;
      __syncthreads();
      int at = before + incl - c;
      for (int w = 0; w < 4; ++w) {
        at += w < wave ? sh.counts[k & 1][w] : 0;
        before += sh.counts[k & 1][w];
      }
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (key(k * kVec + e) == thr) {
          if (at < n) sh.list[at] = (uint64_t)thr << 32 | ~(uint32_t)index(k * kVec + e);
          ++at;
        }
    }
  }
  __syncthreads();
  if (tid == 0) sh.count = min(before, n);
  __syncthreads();
}

template <class E>
__global__ __launch_bounds__(kThreads) void beam_chunk_kernel(BeamArgs a) {
  __shared__ ChunkShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x / a.chunks, chunk = blockIdx.x - row * a.chunks;
  if (a.done && a.done[row] != 0) return;
  const int first = chunk * kBeamChunk;
  const size_t at = (size_t)row * a.ld;
  float x[kPer], m = -INFINITY;
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const int i = first + k * (kThreads * kVec) + tid * kVec;
    if (i + kVec <= a.V) {
      load_logits(a.logits, at + i, x + k * kVec, E());
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[k * kVec + e] = i + e < a.V ? load_scalar(a.logits, at + i + e, E()) : -INFINITY;
    }
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e) m = fmaxf(m, x[e]);
  m = fmaxf(m, __shfl_xor(m, 1, 64));
  m = fmaxf(m, __shfl_xor(m, 2, 64));
  if ((tid & 3) == 0) sh.top[tid >> 2] = m;
  if (tid == 0) sh.count = 0;
  __syncthreads();
  const float group = sh.top[lane], top = wave_max(group);
  if (wave == 0) {
    const float bound = nth_largest(group, a.n);
    if (lane == 0) sh.bound = bound;
  }
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) sum += __builtin_amdgcn_exp2f((x[e] - base) * kLog2e);
  sum = wave_sum(sum);
  if (lane == 0) sh.sum[wave] = sum;
  __syncthreads();
  const float bound = sh.bound;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int i = first + e / kVec * (kThreads * kVec) + tid * kVec + e % kVec;
    if (x[e] >= bound && i < a.V) {
      const int to = atomicAdd(&sh.count, 1);
      if (to < kList) sh.list[to] = (uint64_t)f2key(x[e]) << 32 | ~(uint32_t)i;
    }
  }
  __syncthreads();
  if (sh.count > kList) exact_list(x, first, a.V, a.n, sh);
  const int count = sh.count;
  uint64_t* out = a.cand + (size_t)blockIdx.x * a.n;
  for (int i = tid; i < count; i += kThreads) {
    const uint64_t mine = sh.list[i];
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += sh.list[j] > mine;
    if (rank < a.n) out[rank] = mine;
  }
  for (int i = count + tid; i < a.n; i += kThreads) out[i] = 0;
  if (tid == 0) a.part[blockIdx.x] = make_float2(top, sh.sum[0] + sh.sum[1] + sh.sum[2] + sh.sum[3]);
}

// ---------------------------------------------------------------------- join
constexpr int kJoinThreads = 1024;
constexpr int kJoinList = 1024;

// Order-preserving map from fp64 (no NaN) to integers above 0.
__device__ __forceinline__ uint64_t order_of(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
  return u ^ ((uint64_t)((int64_t)u >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double value_of(uint64_t k) {
  return __longlong_as_double((long long)(k >> 63 ? k & 0x7fffffffffffffffull : ~k));
}

enum RowKind { kNormal, kDone, kNothing };
struct JoinShared {
  double base[TREVS_MAX_BEAMS];   // score minus log of the sum
  float top[TREVS_MAX_BEAMS];
  int kind[TREVS_MAX_BEAMS];
  uint64_t group[64];
  uint64_t order[kJoinList];
  int index[kJoinList];
  uint64_t bound;
  int count;
  uint64_t wave_order[kJoinThreads / 64];
  int wave_index[kJoinThreads / 64];
};

// Continuation q of the sequence's lists: its order (0: there is none) and beam * V + token.
__device__ __forceinline__ uint64_t continuation(const BeamArgs& a, const JoinShared& sh, int b, long long q,
                                                 int& index) {
  const int per = a.chunks * a.n, w = (int)(q / per), i = (int)(q - (long long)w * per);
  if (sh.kind[w] == kNormal) {
    const uint64_t c = a.cand[(size_t)b * a.W * per + q];
    if (c == 0) return 0;
    index = w * a.V + (int)~(uint32_t)c;
    return order_of(sh.base[w] + ((double)key2f((uint32_t)(c >> 32)) - (double)sh.top[w]));
  }
  if (i >= (sh.kind[w] == kDone ? 1 : min(a.n, a.V))) return 0;
  index = w * a.V + (sh.kind[w] == kDone ? a.eos : i);
  return order_of(sh.kind[w] == kDone ? sh.base[w] : (double)-INFINITY);
}

__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(BeamArgs a) {
  __shared__ JoinShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
  for (int w = wave; w < a.W; w += kJoinThreads / 64) {
    const int row = b * a.W + w;
    float score = a.score[row];
    if (!(score < INFINITY)) score = -INFINITY;  // (NaN too)
    if (a.done && a.done[row] != 0) {
      if (lane == 0) {
        sh.base[w] = score;
        sh.kind[w] = kDone;
      }
      continue;
    }
    float m = -INFINITY;
    for (int c = lane; c < a.chunks; c += 64) m = fmaxf(m, a.part[(size_t)row * a.chunks + c].x);
    m = wave_max(m);
    double sum = 0.0;
    for (int c = lane; c < a.chunks; c += 64) {
      const float2 p = a.part[(size_t)row * a.chunks + c];
      sum += p.x == -INFINITY && p.y == 0.f ? 0.0 : (double)p.y * exp((double)p.x - (double)m);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
    if (lane == 0) {
      sh.base[w] = (double)score - log(sum);
      sh.top[w] = m;
      sh.kind[w] = isfinite(score) && isfinite(m) && isfinite(sum) ? kNormal : kNothing;
    }
  }
  if (tid == 0) sh.count = 0;
  __syncthreads();
  const long long total = (long long)a.W * a.chunks * a.n;
  uint64_t best = 0;
  for (long long q = tid; q < total; q += kJoinThreads) {
    int index;
    best = max(best, continuation(a, sh, b, q, index));
  }
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, d, 64));
  if ((tid & 15) == 0) sh.group[tid >> 4] = best;
  __syncthreads();
  if (wave == 0) {
    const uint64_t bound = nth_largest((unsigned long long)sh.group[lane], a.n);
    if (lane == 0) sh.bound = bound;
  }
  __syncthreads();
  const uint64_t bound = max(sh.bound, (uint64_t)1);
  for (long long q = tid; q < total; q += kJoinThreads) {
    int index;
    const uint64_t order = continuation(a, sh, b, q, index);
    if (order < bound) continue;
    const int at = atomicAdd(&sh.count, 1);
    if (at < kJoinList) {
      sh.order[at] = order;
      sh.index[at] = index;
    }
  }
  __syncthreads();
  const int count = sh.count;
  auto write = [&](int rank, uint64_t order, int index) {
    const size_t to = (size_t)b * a.n + rank;
    a.score_out[to] = order ? (float)value_of(order) : -INFINITY;
    a.parent[to] = order ? index / a.V : -1;
    a.token[to] = order ? index % a.V : -1;
  };
  if (count <= kJoinList) {
    for (int i = tid; i < count; i += kJoinThreads) {
      const uint64_t order = sh.order[i];
      const int index = sh.index[i];
      int rank = 0;
      for (int j = 0; j < count; ++j) rank += sh.order[j] > order || (sh.order[j] == order && sh.index[j] < index);
      if (rank < a.n) write(rank, order, index);
    }
    for (int i = count + tid; i < a.n; i += kJoinThreads) write(i, 0, 0);
    return;
  }
  // more than the list holds: one after the other, each the first after the one before
  uint64_t last = ~0ull;
  int last_index = -1;
  for (int r = 0; r < a.n; ++r) {
    uint64_t order = 0;
    int index = INT32_MAX;
    for (long long q = tid; q < total; q += kJoinThreads) {
      int i = 0;
      const uint64_t o = continuation(a, sh, b, q, i);
      if (o == 0 || o > last || (o == last && i <= last_index)) continue;
      if (o > order || (o == order && i < index)) {
        order = o;
        index = i;
      }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint64_t o = __shfl_xor((unsigned long long)order, d, 64);
      const int i = __shfl_xor(index, d, 64);
      if (o > order || (o == order && i < index)) {
        order = o;
        index = i;
      }
    }
    if (lane == 0) {
      sh.wave_order[wave] = order;
      sh.wave_index[wave] = index;
    }
    __syncthreads();
    for (int w = 0; w < kJoinThreads / 64; ++w) {
      const uint64_t o = sh.wave_order[w];
      const int i = sh.wave_index[w];
      if (o > order || (o == order && i < index)) {
        order = o;
        index = i;
      }
    }
    __syncthreads();
    if (tid == 0) write(r, order, index);
    last = order;
    last_index = index;
  }
}

}  // namespace

hipError_t launch_beam_select(const BeamArgs& a, int dtype, hipStream_t s) {
  const dim3 grid((unsigned)((long long)a.B * a.W * a.chunks));
  if (dtype == TREVS_BF16)
    hipLaunchKernelGGL(beam_chunk_kernel<BF16>, grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(beam_chunk_kernel<F32>, grid, dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL(beam_join_kernel, dim3(a.B), dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace trevs
