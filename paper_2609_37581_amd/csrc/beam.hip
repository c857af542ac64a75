// Beam search's selection over beams and vocabulary.
//
// Within a beam continuations rank as their logits do, so the n best of a sequence
// are among the n best of each chunk of each beam's logits.  The first kernel reads
// every logit once: a wave holds a chunk in registers, forms its maximum and sum of
// exponentials and lists its best.  The second joins a sequence's chunks: its log-sum-
// exps, then the scores of the listed continuations, in 64 bits, since continuations of
// different beams can lie closer together than 32 bits tell apart.
//
// The n best of many values are found by a bound: the n-th largest of the maxima of 64
// groups of them (of the lanes).  At least n values reach it, and hardly more do; those
// are the list.  Lists that overflow (ties: banned tokens, all -inf) are cut exactly, by
// bisection over the bits and in index order.
#include <type_traits>

#include "beam.hpp"
#include "common.hpp"

namespace trevs {
namespace {

constexpr int kVec = 8;  // logits next to each other
static_assert(TREVS_MAX_BEAM_OUT <= 64, "a lane to a continuation at least");

typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_4 __attribute__((ext_vector_type(4), aligned(4)));

// Eight logits from any element on (rows need not be aligned), as they lie.
template <class E>
struct Eight {
  static constexpr int kWords = 2 * E::kBytes;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void* p, size_t i) {
    using any = typename std::conditional<E::kBytes == 2, u32x4_2, u32x4_4>::type;
    const any* f = reinterpret_cast<const any*>(reinterpret_cast<const uint8_t*>(p) + i * E::kBytes);
#pragma unroll
    for (int j = 0; j < kWords / 4; ++j) {
      const u32x4 v = f[j];
#pragma unroll
      for (int q = 0; q < 4; ++q) w[4 * j + q] = v[q];
    }
  }
  // the first n of them (n < 8), -inf behind
  __device__ __forceinline__ void load_some(const void* p, size_t i, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = j < n ? load_scalar(p, i + j, E()) : -INFINITY;
      const uint32_t u = __float_as_uint(x);
      if constexpr (E::kBytes == 4)
        w[j] = u;
      else
        w[j >> 1] = j & 1 ? (w[j >> 1] & 0xffffu) | (u & 0xffff0000u) : u >> 16;
    }
  }
  __device__ __forceinline__ float operator[](int j) const {
    if constexpr (E::kBytes == 4) return __uint_as_float(w[j]);
    return j & 1 ? bf16_hi(w[j >> 1]) : bf16_lo(w[j >> 1]);
  }
};

// A bound that at least n of the lanes' values reach, and hardly more: the n-th largest of
// them cut to its high BITS bits, found bit by bit (comparing each with each takes four
// times as many instructions).
template <int BITS>
__device__ __forceinline__ uint32_t nth_bound(uint32_t v, int n) {
  uint32_t bound = 0;
#pragma unroll
  for (int bit = 31; bit >= 32 - BITS; --bit) {
    const uint32_t least = bound | (1u << bit);
    bound = __popcll(__ballot(v >= least)) >= n ? least : bound;
  }
  return bound;
}

// Exponentials are taken to base 2, as exp2(x L - base(m)) with L = log2 e in 32 bits and
// m the chunk's maximum: one instruction to an argument.  What L lacks of log2 e makes
// all of them too small by a factor of about 2^(kRest m), which the join puts back (the
// terms far from m, where it is another, hardly count), so that continuations of different
// beams compare as if it were not there.  Far from 0 base(m) would be off by whole powers of
// two: there they are exp2((x - m) L).
constexpr float kFar = 65536.f;
constexpr double kRest = 1.4426950408889634073599 - (double)kLog2e;
__device__ __forceinline__ float chunk_base(float m) { return m * kLog2e; }

// A wave's chunk: logit e of round k of a lane is number k 512 + lane 8 + e.
template <class E>
struct Chunk {
  static constexpr int kRounds = kBeamChunk<E::kBytes> / (64 * kVec);
  Eight<E> x[kRounds];
  __device__ __forceinline__ void load(const BeamArgs& a, size_t row, int first) {
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      const int i = first + (k * 64 + (threadIdx.x & 63)) * kVec;
      if (i + kVec <= a.V)
        x[k].load(a.logits, row + i);
      else
        x[k].load_some(a.logits, row + i, max(a.V - i, 0));
    }
  }
  // The floats of bf16 logits are not kept from one pass to the next (they take twice the
  // registers; unpacked again, 8 waves of a SIMD hide each other's loads instead of 3).
  __device__ __forceinline__ void forget() {
    if constexpr (E::kBytes == 2) {
#pragma unroll
      for (int k = 0; k < kRounds; ++k)
#pragma unroll
        for (int j = 0; j < Eight<E>::kWords; ++j) x[k].w[j] = (uint32_t)opaque((int)x[k].w[j]);
    }
  }
};

// The best of the chunk, exactly n (all of fewer), to out[0, n): the n-th largest key by
// bisection, what lies above it, and the first of those that equal it.  Returns their number.
template <class E>
__device__ __forceinline__ int exact_list(Chunk<E>& c, int first, int V, int n, uint64_t* out) {
  const int lane = threadIdx.x & 63;
  // (0 for places past the vocabulary)
  auto key = [&](int k, int e) { return first + (k * 64 + lane) * kVec + e < V ? f2key(c.x[k][e]) : 0u; };
  auto entry = [&](int k, int e) {
    return (uint64_t)key(k, e) << 32 | ~(uint32_t)(first + (k * 64 + lane) * kVec + e);
  };
  uint32_t thr = 0;
#pragma unroll 1
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t least = thr | (1u << bit);
    int count = 0;
    c.forget();
#pragma unroll
    for (int k = 0; k < Chunk<E>::kRounds; ++k)
#pragma unroll
      for (int e = 0; e < kVec; ++e) count += __popcll(__ballot(key(k, e) >= least));
    if (count >= n) thr = least;
  }
  int at = 0;
  c.forget();
#pragma unroll
  for (int k = 0; k < Chunk<E>::kRounds; ++k)
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const uint64_t hits = __ballot(key(k, e) > thr);
      if (key(k, e) > thr) out[at + __popcll(hits & ((1ull << lane) - 1))] = entry(k, e);
      at += __popcll(hits);
    }
  if (thr == 0) return at;
  c.forget();
#pragma unroll
  for (int k = 0; k < Chunk<E>::kRounds; ++k) {
    if (at >= n) break;
    int ties = 0;
#pragma unroll
    for (int e = 0; e < kVec; ++e) ties += key(k, e) == thr;
    const int incl = wave_incl_scan(ties, lane);
    int to = at + incl - ties;
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (key(k, e) == thr) {
        if (to < n) out[to] = entry(k, e);
        ++to;
      }
    at += __builtin_amdgcn_readlane(incl, 63);
  }
  return min(at, n);
}

// Bound by bytes, with the vector instructions close behind; the waves of a workgroup have
// nothing to do with each other (64 x 8 beams of 152,064 tokens, a fifth of them finished:
// 28 us, 4.4 TB/s; as workgroups of 8192 logits with barriers between the steps 41 us).
template <class E>
__global__ __launch_bounds__(256, E::kBytes == 2 ? 8 : 4) void beam_chunk_kernel(BeamArgs a) {
  constexpr int kRounds = Chunk<E>::kRounds;
  __shared__ int s_list[4][kBeamList];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long id = (long long)blockIdx.x * 4 + wave;
  const int row = (int)(id / a.chunks), chunk = (int)(id - (long long)row * a.chunks);
  if (row >= a.B * a.W) return;
  if (a.done && a.done[row] != 0) return;
  const int first = chunk * kBeamChunk<E::kBytes>;
  const size_t at = (size_t)row * a.ld;
  Chunk<E> c;
  c.load(a, at, first);
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < kRounds; ++k)
#pragma unroll
    for (int e = 0; e < kVec; ++e) m = fmaxf(m, c.x[k][e]);
  const float top = wave_max(m);
  const uint32_t least = nth_bound<16>(f2key(m), a.n);
  const float bound = fmaxf(key2f(least), -INFINITY);  // (NaN below -inf's key)
  const float base = top == -INFINITY ? 0.f : chunk_base(top);
  c.forget();
  // the logits that reach the bound: their places
  const int V = opaque(a.V);  // (else the bounds of the loads are kept, a pair of registers to each)
  int* list = s_list[wave];
  float sum[2] = {0.f, 0.f};
  int count = 0;
#pragma unroll
  for (int k = 0; k < kRounds; ++k)
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const float y = c.x[k][e];
      sum[e & 1] += __builtin_amdgcn_exp2f(fmaf(y, kLog2e, -base));
      const uint64_t hits = __ballot(y >= bound);
      if (hits) {
        const int to = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(hits >> 32),
                                                      __builtin_amdgcn_mbcnt_lo((uint32_t)hits, (uint32_t)count));
        if (y >= bound && to < kBeamList) list[to] = first + (k * 64 + lane) * kVec + e;
        count += __popcll(hits);
      }
    }
  if (fabsf(top) >= kFar && top != -INFINITY) {
    sum[0] = sum[1] = 0.f;
    c.forget();
#pragma unroll
    for (int k = 0; k < kRounds; ++k)
#pragma unroll
      for (int e = 0; e < kVec; ++e) sum[e & 1] += __builtin_amdgcn_exp2f((c.x[k][e] - top) * kLog2e);
  }
  const float total = wave_sum(sum[0] + sum[1]);
  uint64_t* out = a.cand + (size_t)id * a.stride;
  if (count <= a.stride) {
    __builtin_amdgcn_wave_barrier();
    for (int i = lane; i < a.stride; i += 64) {
      const int v = i < count ? list[i] : V;
      // (places past the vocabulary are listed when the bound is -inf)
      out[i] = v < V ? (uint64_t)f2key(load_scalar(a.logits, at + v, E())) << 32 | ~(uint32_t)v : 0;
    }
  } else {
    const int n = exact_list(c, first, V, a.n, out);
    for (int i = n + lane; i < a.stride; i += 64) out[i] = 0;
  }
  if (lane == 0) a.part[id] = make_float2(top, total);
}

// ---------------------------------------------------------------------- join
constexpr int kJoinThreads = 512;
constexpr int kJoinList = 1024;
constexpr int kJoinChunks = 1024;

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
  uint64_t best[kJoinThreads / 64][64];
  uint64_t order[kJoinList];
  int index[kJoinList];
  uint64_t bound;
  int count, chunks;
  int chunk[kJoinChunks];
  uint64_t wave_order[kJoinThreads / 64];
  int wave_index[kJoinThreads / 64];
};

// The best that chunk j = w chunks + c of the sequence can have (0: it has none).  A
// finished beam's one continuation, and those of a beam without scores, count as its first
// chunk's.
__device__ __forceinline__ uint64_t chunk_top(const BeamArgs& a, const JoinShared& sh, int b, int j) {
  const int w = j / a.chunks;
  if (sh.kind[w] != kNormal && j != w * a.chunks) return 0;
  if (sh.kind[w] == kNothing) return order_of(-INFINITY);
  if (sh.kind[w] == kDone) return order_of(sh.base[w]);
  const float x = a.part[(size_t)b * a.W * a.chunks + j].x;
  return order_of(sh.base[w] + ((double)x - (double)sh.top[w]));
}
// Entry i of chunk j's list: its order (0: there is none) and beam * V + token.
__device__ __forceinline__ uint64_t continuation(const BeamArgs& a, const JoinShared& sh, int b, int j, int i,
                                                 int& index) {
  const int w = j / a.chunks;
  if (sh.kind[w] == kNormal) {
    const uint64_t c = a.cand[((size_t)b * a.W * a.chunks + j) * a.stride + i];
    if (c == 0) return 0;
    index = w * a.V + (int)~(uint32_t)c;
    return order_of(sh.base[w] + ((double)key2f((uint32_t)(c >> 32)) - (double)sh.top[w]));
  }
  if (j != w * a.chunks || i >= (sh.kind[w] == kDone ? 1 : min(a.n, a.V))) return 0;
  index = w * a.V + (sh.kind[w] == kDone ? a.eos : i);
  return order_of(sh.kind[w] == kDone ? sh.base[w] : (double)-INFINITY);
}

// The n-th largest (about) of the workgroup's values, a group being a lane of all waves
// (values next to each other, which a list's are, belong to different ones); 1 at least.
__device__ __forceinline__ uint64_t group_bound(uint64_t best, int n, JoinShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  sh.best[wave][lane] = best;
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 1; w < kJoinThreads / 64; ++w) best = max(best, sh.best[w][lane]);
    const uint32_t bound = nth_bound<32>((uint32_t)(best >> 32), n);
    if (lane == 0) sh.bound = max((uint64_t)bound << 32, (uint64_t)1);
  }
  __syncthreads();
  return sh.bound;
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
      const double to = m * (kLog2e + kRest);
      const double from = fabsf(p.x) >= kFar ? p.x * (kLog2e + kRest) : chunk_base(p.x) + kRest * p.x;
      sum += p.x == -INFINITY && p.y == 0.f ? 0.0 : p.y * exp2(from - to);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
    if (lane == 0) {
      sh.base[w] = (double)score - log(sum);
      sh.top[w] = m;
      sh.kind[w] = isfinite(score) && isfinite(m) && isfinite(sum) ? kNormal : kNothing;
    }
  }
  if (tid == 0) sh.count = sh.chunks = 0;
  __syncthreads();
  // chunks whose best reaches a bound that n chunks' best reach
  const int all = a.W * a.chunks;
  uint64_t best = 0;
  for (int j = tid; j < all; j += kJoinThreads) best = max(best, chunk_top(a, sh, b, j));
  const uint64_t least = group_bound(best, a.n, sh);
  for (int j = tid; j < all; j += kJoinThreads)
    if (chunk_top(a, sh, b, j) >= least) {
      const int at = atomicAdd(&sh.chunks, 1);
      if (at < kJoinChunks) sh.chunk[at] = j;
    }
  __syncthreads();
  // (more than the list holds: all of them)
  const bool listed = sh.chunks <= kJoinChunks;
  const int total = (listed ? sh.chunks : all) * a.stride;
  auto entry = [&](int q, int& index) {
    const int c = q / a.stride;
    return continuation(a, sh, b, listed ? sh.chunk[c] : c, q - c * a.stride, index);
  };
  // of their entries, those that reach a bound that n of them reach
  best = 0;
  for (int q = tid; q < total; q += kJoinThreads) {
    int index;
    best = max(best, entry(q, index));
  }
  const uint64_t bound = max(group_bound(best, a.n, sh), least);
  for (int q = tid; q < total; q += kJoinThreads) {
    int index;
    const uint64_t order = entry(q, index);
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
    for (int q = tid; q < total; q += kJoinThreads) {
      int i = 0;
      const uint64_t o = entry(q, i);
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
  const dim3 grid((unsigned)(((long long)a.B * a.W * a.chunks + 3) / 4));
  if (dtype == TREVS_BF16)
    hipLaunchKernelGGL(beam_chunk_kernel<BF16>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(beam_chunk_kernel<F32>, grid, dim3(256), 0, s, a);
  hipLaunchKernelGGL(beam_join_kernel, dim3(a.B), dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace trevs
