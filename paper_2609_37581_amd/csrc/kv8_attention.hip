// Attention of query rows over the 8-bit paged cache: one pass over the keys
// with the running maximum and sum of the softmax.
//
// A wave takes one query row: lanes hold a token each for the logits, then
// D/64 channels each for the weighted values.
#include "cache.hpp"

namespace trevs {
namespace {

template <class E, int D, int PAGE>
__global__ __launch_bounds__(64) void row_kernel(AttnArgs a) {
  __shared__ float q[D];
  __shared__ float w[64];
  const int lane = threadIdx.x;
  int id = blockIdx.x;
  const int h = id % a.H_q;
  id /= a.H_q;
  const int t = id % a.T_max, b = id / a.T_max;
  const int rows = a.q_len ? min(max(a.q_len[b], 0), a.T_max) : a.T_max;
  if (t >= rows) return;
  const int slot = slot_of(a.slots, b, a.c.n_slots);
  const int L = slot_len(a.c.len, slot, a.kv_max);
  const int n = a.causal ? min(L - rows + t + 1, L) : L;
  const size_t row = (size_t)b * a.T_max + t;
  for (int c = lane; c < D; c += 64) q[c] = load_scalar(a.q, row * a.q_ld + (size_t)h * D + c, E()) * a.scale_log2e;
  __syncthreads();
  float m = -INFINITY, sum = 0.f, acc[D / 64];
#pragma unroll
  for (int k = 0; k < D / 64; ++k) acc[k] = 0.f;
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    const int page = j < n ? page_at(a.c, slot, j / PAGE) : -1;
    const size_t block = (size_t)max(page, 0) * a.c.H_kv + h / a.G;
    float s = -INFINITY;
    if (page >= 0) {
      const uint32_t* k = reinterpret_cast<const uint32_t*>(a.c.k + block * (PAGE * D) + (j % PAGE) * D);
      float x = 0.f, y[4];
      for (int c = 0; c < D / 4; ++c) {
        from_e4m3(k[c], y);
#pragma unroll
        for (int i = 0; i < 4; ++i) x = fmaf(q[4 * c + i], y[i], x);
      }
      s = x * a.c.k_scale[block];
    }
    const float top = fmaxf(m, wave_max(s));
    if (top == -INFINITY) continue;
    const float old = exp2f(m - top), p = exp2f(s - top);
    m = top;
    sum = sum * old + wave_sum(p);
    __syncthreads();
    w[lane] = page >= 0 ? p * a.c.v_scale[block] : 0.f;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < D / 64; ++k) acc[k] *= old;
    for (int i = 0; i < min(64, n - j0); ++i) {
      const int pg = page_at(a.c, slot, (j0 + i) / PAGE);
      if (pg < 0) continue;
      const uint8_t* v = a.c.v + ((size_t)pg * a.c.H_kv + h / a.G) * (PAGE * D) + (j0 + i) % PAGE;
#pragma unroll
      for (int k = 0; k < D / 64; ++k) {
        float y[4];
        from_e4m3(v[(lane + 64 * k) * PAGE], y);
        acc[k] = fmaf(w[i], y[0], acc[k]);
      }
    }
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int k = 0; k < D / 64; ++k) {
    const size_t o = (row * a.H_q + h) * D + lane + 64 * k;
    if (E::kBytes == 2)
      reinterpret_cast<__bf16*>(a.out)[o] = (__bf16)(acc[k] * inv);
    else
      reinterpret_cast<float*>(a.out)[o] = acc[k] * inv;
  }
  if (a.lse && lane == 0)
    a.lse[((size_t)b * a.H_q + h) * a.T_max + t] = sum > 0.f ? (m + log2f(sum)) * kLn2 : -INFINITY;
}

template <class E, int D>
void by_page(const AttnArgs& a, int page, hipStream_t s) {
  const dim3 grid((unsigned)((long long)a.B * a.T_max * a.H_q));
  if (page == 16) hipLaunchKernelGGL((row_kernel<E, D, 16>), grid, dim3(64), 0, s, a);
  if (page == 32) hipLaunchKernelGGL((row_kernel<E, D, 32>), grid, dim3(64), 0, s, a);
  if (page == 64) hipLaunchKernelGGL((row_kernel<E, D, 64>), grid, dim3(64), 0, s, a);
}

template <class E>
void by_head(const AttnArgs& a, int d_head, int page, hipStream_t s) {
  if (d_head == 64) by_page<E, 64>(a, page, s);
  if (d_head == 128) by_page<E, 128>(a, page, s);
  if (d_head == 256) by_page<E, 256>(a, page, s);
}

}  // namespace

hipError_t launch_kv8_attention(const AttnArgs& a, int dtype, int d_head, int page, hipStream_t s) {
  if (dtype == TREVS_BF16)
    by_head<BF16>(a, d_head, page, s);
  else
    by_head<F32>(a, d_head, page, s);
  return hipGetLastError();
}

}  // namespace trevs
