// Rotary positions of query and key rows, alone or after the norms of their heads.
//
// A pair (a, b) turns by 2 pi pos f: the turns pos * f lose what matters in
// 32 bits (position 10^6 of a pair that turns once in 6 positions has 2^-7 of
// a turn left), so they are reduced to a fraction of a turn in 64 bits.  For
// fp32 rows sine and cosine are formed in 64 too and rounded once, with
// attn_factor: the rotated values are then off by 3.7e-8, with 32-bit ones by
// 5.6e-8 (a token of 64 sequences 4.85 us, 4.65 with those).  The rounding of
// bf16 rows, 1.7e-3, hides either, and they take the 32-bit ones.
//
// Bound by bytes: every value is read and written once.  A workgroup takes a
// few rows (tokens), forms each pair's sine and cosine once in LDS and turns
// all heads of q and k with them, 16 bytes of either side of VE pairs per
// lane and step.
#include <type_traits>

#include "cache.hpp"

namespace trevs {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kMaxRows = 8;  // rows of one workgroup

template <class E>
struct Vec;
template <>
struct Vec<BF16> {
  static constexpr int VE = 8;
  static __device__ __forceinline__ void load(const uint8_t* p, float (&x)[8]) {
    const u32x4 w = ldg16(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = bf16_lo(w[j]);
      x[2 * j + 1] = bf16_hi(w[j]);
    }
  }
  static __device__ __forceinline__ void store(uint8_t* p, const float (&x)[8]) {
    typedef __bf16 bf16v __attribute__((ext_vector_type(8)));
    bf16v y;
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = (__bf16)x[j];
    *reinterpret_cast<bf16v*>(p) = y;
  }
};
template <>
struct Vec<F32> {
  static constexpr int VE = 4;
  static __device__ __forceinline__ void load(const uint8_t* p, float (&x)[4]) {
    const u32x4 w = ldg16(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(w[j]);
  }
  static __device__ __forceinline__ void store(uint8_t* p, const float (&x)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  }
};

// Sine and cosine of every pair of the workgroup's rows.
template <class E>
__device__ __forceinline__ void fill_turns(const RopeArgs& a, long long row0, int rows, int half, float2* turn) {
  for (int e = threadIdx.x; e < rows * half; e += kThreads) {
    const int r = e / half, i = e - r * half;
    int p = 0;
    while (p < a.n_pos - 1 && i >= a.bound[p]) ++p;
    const double at = (double)a.pos[p * a.rows + row0 + r], f = a.freqs[i];
    const double turns = fma(at, f, -rint(at * f));  // (the product is not rounded)
    if constexpr (E::kBytes == 4) {
      double sn, cs;
      sincospi(2.0 * turns, &sn, &cs);
      turn[e] = make_float2((float)(cs * a.attn_factor), (float)(sn * a.attn_factor * a.sign));
    } else {
      float sn, cs;
      sincospif(2.f * (float)turns, &sn, &cs);
      turn[e] = make_float2(cs * a.attn_factor, sn * a.attn_factor * a.sign);
    }
  }
}

// Two vectors of pairs turned: of pairs (i, i + R/2) those of x with those of y,
// of interleaved ones those within x, then those within y.
template <class E, bool INTER>
__device__ __forceinline__ void turn_pairs(float (&x)[Vec<E>::VE], float (&y)[Vec<E>::VE], const float2* w) {
  constexpr int VE = Vec<E>::VE;
  if constexpr (INTER) {
#pragma unroll
    for (int j = 0; j < VE / 2; ++j) {
      const float2 u = w[j], z = w[VE / 2 + j];
      const float a0 = x[2 * j], b0 = x[2 * j + 1], a1 = y[2 * j], b1 = y[2 * j + 1];
      x[2 * j] = a0 * u.x - b0 * u.y;
      x[2 * j + 1] = b0 * u.x + a0 * u.y;
      y[2 * j] = a1 * z.x - b1 * z.y;
      y[2 * j + 1] = b1 * z.x + a1 * z.y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float2 u = w[j];
      const float a0 = x[j], b0 = y[j];
      x[j] = a0 * u.x - b0 * u.y;
      y[j] = b0 * u.x + a0 * u.y;
    }
  }
}

template <class E, bool INTER>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, int rows_per_block) {
  constexpr int VE = Vec<E>::VE;
  __shared__ float2 turn[kMaxRows * kMaxPairs];
  const int tid = threadIdx.x;
  const long long row0 = (long long)blockIdx.x * rows_per_block;
  const int rows = (int)min((long long)rows_per_block, a.rows - row0);
  const int half = a.rot_dim >> 1;
  fill_turns<E>(a, row0, rows, half, turn);
  __syncthreads();
  // items of a row: VE pairs of one head, then (out of place) the vectors past rot_dim
  const int heads = a.t[0].H + a.t[1].H, chunks = half / VE;
  const int tail = a.copy_tail ? (a.d_head - a.rot_dim) / VE : 0;
  const int per_head = chunks + tail, per_row = heads * per_head;
  const int n_items = rows * per_row;
  for (int e = blockIdx.y * kThreads + tid; e < n_items; e += gridDim.y * kThreads) {
    const int r = e / per_row, in_row = e - r * per_row;
    int h = in_row / per_head;
    const int c = in_row - h * per_head;
    const bool is_k = h >= a.t[0].H;
    const RopeTensor& t = is_k ? a.t[1] : a.t[0];
    h -= is_k ? a.t[0].H : 0;
    const uint8_t* in = t.in + (row0 + r) * t.in_ld + (size_t)h * a.d_head * E::kBytes;
    uint8_t* out = t.out + (row0 + r) * t.out_ld + (size_t)h * a.d_head * E::kBytes;
    if (c >= chunks) {
      const int o = a.rot_dim * E::kBytes + (c - chunks) * 16;
      *reinterpret_cast<u32x4*>(out + o) = ldg16(in + o);
      continue;
    }
    const int o0 = INTER ? c * 32 : c * 16, o1 = INTER ? c * 32 + 16 : half * E::kBytes + c * 16;
    float x[VE], y[VE];
    Vec<E>::load(in + o0, x);
    Vec<E>::load(in + o1, y);
    turn_pairs<E, INTER>(x, y, turn + r * half + c * VE);
    Vec<E>::store(out + o0, x);
    Vec<E>::store(out + o1, y);
  }
}

// ------------------------------------------------- norms of the heads before it
// VE weights from element i on, as floats; ones without weights.
template <int VE>
__device__ __forceinline__ void load_weights(const void* w, int bf16, size_t i, float offset, float (&y)[VE]) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < VE; ++j) y[j] = 1.f;
    return;
  }
  if (bf16) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(w) + i;
    u32x2 a[VE / 4];
#pragma unroll
    for (int j = 0; j < VE / 4; ++j) a[j] = reinterpret_cast<const u32x2*>(p)[j];
#pragma unroll
    for (int j = 0; j < VE / 2; ++j) {
      y[2 * j] = bf16_lo(a[j >> 1][j & 1]);
      y[2 * j + 1] = bf16_hi(a[j >> 1][j & 1]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < VE / 4; ++j) {
      const u32x4 a = ldg16(reinterpret_cast<const float*>(w) + i + 4 * j);
#pragma unroll
      for (int q = 0; q < 4; ++q) y[4 * j + q] = __uint_as_float(a[q]);
    }
  }
#pragma unroll
  for (int j = 0; j < VE; ++j) y[j] += offset;
}

// Sum over the LANES lanes next to each other that hold one head.
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int d = 1; d < LANES; d <<= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// A head's LANES lanes hold two vectors of it each (of the rotated part those whose
// pairs meet), so the norm's sum of squares is theirs, and every value is read and
// written once: bound by bytes, as the rotation alone (4 x 4259 rows of 32 heads of 128 in
// bf16 58.7 us, 4.8 TB/s, the rotation 56.5; a copy of the bytes 54).
template <class E, bool INTER, int D>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(NormRopeArgs n, int rows_per_block) {
  constexpr int VE = Vec<E>::VE, LANES = D / (2 * VE);
  const RopeArgs& a = n.rope;
  __shared__ float2 turn[kMaxRows * kMaxPairs];
  const int tid = threadIdx.x;
  const long long row0 = (long long)blockIdx.x * rows_per_block;
  const int rows = (int)min((long long)rows_per_block, a.rows - row0);
  const int half = a.rot_dim >> 1;
  fill_turns<E>(a, row0, rows, half, turn);
  __syncthreads();
  const int heads = a.t[0].H + a.t[1].H, per_row = heads * LANES, n_items = rows * per_row;
  const int c = tid % LANES, pairs = half / VE;
  const bool turned = c < pairs;
  // this lane's two vectors in a head (whole heads are skipped at the end, so a head's lanes stay together)
  const int o0 = !turned ? a.rot_dim + (c - pairs) * 2 * VE : INTER ? c * 2 * VE : c * VE;
  const int o1 = turned && !INTER ? half + c * VE : o0 + VE;
  for (int e = blockIdx.y * kThreads + tid; e < n_items; e += gridDim.y * kThreads) {
    const int r = e / per_row;
    int h = (e - r * per_row) / LANES;
    const bool is_k = h >= a.t[0].H;
    const RopeTensor& t = is_k ? a.t[1] : a.t[0];
    h -= is_k ? a.t[0].H : 0;
    const uint8_t* in = t.in + (row0 + r) * t.in_ld + (size_t)h * D * E::kBytes;
    uint8_t* out = t.out + (row0 + r) * t.out_ld + (size_t)h * D * E::kBytes;
    float x[VE], y[VE], wx[VE], wy[VE];
    Vec<E>::load(in + o0 * E::kBytes, x);
    Vec<E>::load(in + o1 * E::kBytes, y);
    const void* w = is_k ? n.k_weight : n.q_weight;
    const size_t w0 = n.per_head ? (size_t)h * D : 0;
    load_weights<VE>(w, n.weight_bf16, w0 + o0, n.weight_offset, wx);
    load_weights<VE>(w, n.weight_bf16, w0 + o1, n.weight_offset, wy);
    auto squares = [&] {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < VE; ++j) s = fmaf(x[j], x[j], fmaf(y[j], y[j], s));
      return head_sum<LANES>(s) * (1.f / D);
    };
    float mean = squares(), eps = n.eps;
    // squares beyond fp32, or so small that their bits are lost: those of the values times a power of two
    const bool big = !(mean < 0x1p120f);
    if (big || mean + eps < 0x1p-80f) {
      const float by = big ? 0x1p-70f : 0x1p70f;
#pragma unroll
      for (int j = 0; j < VE; ++j) x[j] *= by, y[j] *= by;
      eps = eps * by * by;
      mean = squares();
    }
    const float inv = rsqrtf(mean + eps);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      x[j] = x[j] * inv * wx[j];
      y[j] = y[j] * inv * wy[j];
    }
    if (turned) turn_pairs<E, INTER>(x, y, turn + r * half + c * VE);
    Vec<E>::store(out + o0 * E::kBytes, x);
    Vec<E>::store(out + o1 * E::kBytes, y);
  }
}

}  // namespace

int rope_rows(long long rows, int rot_dim) {
  // one sine and cosine a thread; fewer rows when the rows would not give every CU a workgroup
  int n = min(kMaxRows, max(1, 2 * kThreads / rot_dim));
  while (n > 1 && (rows + n - 1) / n < 512) n >>= 1;
  return n;
}

hipError_t launch_rope(const RopeArgs& a, int interleaved, int dtype, hipStream_t s) {
  const int half = a.rot_dim / 2;
  const int rows = rope_rows(a.rows, a.rot_dim);
  const long long blocks = (a.rows + rows - 1) / rows;
  // a few rows split their heads over workgroups
  const int ve = 16 / (dtype == TREVS_BF16 ? 2 : 4);
  const int items = rows * (a.t[0].H + a.t[1].H) * (half / ve + (a.copy_tail ? (a.d_head - a.rot_dim) / ve : 0));
  const int split = blocks >= 512 ? 1 : (int)min((long long)(items + kThreads - 1) / kThreads, 512 / blocks + 1);
  const dim3 grid((unsigned)blocks, split);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a, rows); };
  if (dtype == TREVS_BF16)
    interleaved ? go(rope_kernel<BF16, true>) : go(rope_kernel<BF16, false>);
  else
    interleaved ? go(rope_kernel<F32, true>) : go(rope_kernel<F32, false>);
  return hipGetLastError();
}

hipError_t launch_norm_rope(const NormRopeArgs& n, int interleaved, int dtype, hipStream_t s) {
  const RopeArgs& a = n.rope;
  const int rows = rope_rows(a.rows, a.rot_dim);
  const long long blocks = (a.rows + rows - 1) / rows;
  const int items = rows * (a.t[0].H + a.t[1].H) * (a.d_head / (32 / (dtype == TREVS_BF16 ? 2 : 4)));
  const int split = blocks >= 512 ? 1 : (int)min((long long)(items + kThreads - 1) / kThreads, 512 / blocks + 1);
  const dim3 grid((unsigned)blocks, split);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, n, rows); };
  auto by_head = [&](auto e, auto inter) {
    using E = decltype(e);
    constexpr bool INTER = decltype(inter)::value;
    if (a.d_head == 64) go(norm_rope_kernel<E, INTER, 64>);
    if (a.d_head == 128) go(norm_rope_kernel<E, INTER, 128>);
    if (a.d_head == 256) go(norm_rope_kernel<E, INTER, 256>);
  };
  auto by_pairs = [&](auto e) { interleaved ? by_head(e, std::true_type()) : by_head(e, std::false_type()); };
  dtype == TREVS_BF16 ? by_pairs(BF16()) : by_pairs(F32());
  return hipGetLastError();
}

}  // namespace trevs
