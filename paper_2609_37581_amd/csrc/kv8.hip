// Rows into the 8-bit paged cache, kept rows moved inside it, pages copied.
//
// A workgroup owns one destination block: one page of one KV head, keys or
// values.  Its largest magnitude gives the block's scale, a power of two, so
// dividing by it is exact and each value is rounded once, by the e4m3
// conversion.  Lanes hold units of 4 tokens x 8 channels: keys are stored 8
// channels at a time, values (token last) are turned in LDS, four tokens to a
// word.
#include <float.h>

#include "cache.hpp"

namespace trevs {
namespace {

template <int D, int PAGE>
struct Block {
  static constexpr int kUnits = PAGE / 4 * (D / 8);
  static constexpr int kThreads = kUnits < 64 ? 64 : kUnits > 256 ? 256 : kUnits;
  static constexpr int kPer = (kUnits + kThreads - 1) / kThreads;  // units of a thread
  static constexpr int kRow = PAGE / 4 + 1;                        // words of a channel's tokens in LDS, padded
};

// Largest value of a workgroup, in every thread.
template <int NT>
__device__ __forceinline__ float block_max(float m, float* lds) {
  m = wave_max(m);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) m = fmaxf(m, lds[w]);
  }
  return m;
}

__device__ __forceinline__ void load8(const void* p, size_t i, float (&x)[8], BF16) {
  const u32x4 w = ldg16(reinterpret_cast<const uint16_t*>(p) + i);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = bf16_lo(w[j]);
    x[2 * j + 1] = bf16_hi(w[j]);
  }
}
__device__ __forceinline__ void load8(const void* p, size_t i, float (&x)[8], F32) {
  const float* f = reinterpret_cast<const float*>(p) + i;
  const u32x4 a = ldg16(f), b = ldg16(f + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = __uint_as_float(a[j]);
    x[4 + j] = __uint_as_float(b[j]);
  }
}

// Stores tokens [lo, hi) of a block from the units' values.  Earlier tokens
// of the block (t < lo) are moved to the new scale when `ratio` < 1.
template <int D, int PAGE>
__device__ __forceinline__ void store_block(uint8_t* dst, bool values, int lo, int hi, float inv, float ratio,
                                            const float (&x)[Block<D, PAGE>::kPer][4][8], uint32_t* lds) {
  using B = Block<D, PAGE>;
  const int tid = threadIdx.x;
  if (!values) {
#pragma unroll
    for (int u = 0; u < B::kPer; ++u) {
      const int e = tid + u * B::kThreads;
      if (B::kUnits < B::kThreads && e >= B::kUnits) break;
      const int c = e % (D / 8) * 8, t0 = e / (D / 8) * 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = t0 + i;
        u32x2* to = reinterpret_cast<u32x2*>(dst + t * D + c);
        const float(&y)[8] = x[u][i];
        if (t >= lo && t < hi) {
          *to = u32x2{to_e4m3(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv),
                      to_e4m3(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)};
        } else if (t < lo && ratio < 1.f) {
          const u32x2 w = *to;
          *to = u32x2{rescale_e4m3(w[0], ratio), rescale_e4m3(w[1], ratio)};
        }
      }
    }
    return;
  }
#pragma unroll
  for (int u = 0; u < B::kPer; ++u) {
    const int e = tid + u * B::kThreads;
    if (B::kUnits < B::kThreads && e >= B::kUnits) break;
    const int c = e % (D / 8) * 8, tq = e / (D / 8);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      lds[(c + j) * B::kRow + tq] = to_e4m3(x[u][0][j] * inv, x[u][1][j] * inv, x[u][2][j] * inv, x[u][3][j] * inv);
  }
  __syncthreads();
  // a channel's words: whole ones stored as they are, the others merged with what is held
  for (int e = tid; e < D * (PAGE / 4); e += B::kThreads) {
    const int c = e / (PAGE / 4), tq = e % (PAGE / 4), t0 = tq * 4;
    if (t0 >= hi) continue;
    uint32_t* to = reinterpret_cast<uint32_t*>(dst + c * PAGE + t0);
    uint32_t w = lds[c * B::kRow + tq];
    if (t0 < lo || t0 + 4 > hi) {
      if (t0 + 4 <= lo && !(ratio < 1.f)) continue;
      uint32_t held = *to, mask = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) mask |= t0 + i >= lo && t0 + i < hi ? 0xffu << (8 * i) : 0u;
      if (ratio < 1.f && t0 < lo) {
        uint32_t before = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) before |= t0 + i < lo ? 0xffu << (8 * i) : 0u;
        held = (rescale_e4m3(held, ratio) & before) | (held & ~before);
      }
      w = (w & mask) | (held & ~mask);
    }
    *to = w;
  }
}

// Rows [0, n_new) of a sequence to tokens len - n_new + t: workgroup (b, f, h)
// writes what falls into the f-th page from the first new token's on.
template <class E, int D, int PAGE>
__global__ __launch_bounds__((Block<D, PAGE>::kThreads)) void write_kernel(WriteArgs a) {
  using B = Block<D, PAGE>;
  __shared__ uint32_t lds[D * B::kRow];
  __shared__ float red[4];
  const bool values = blockIdx.y != 0;
  int id = blockIdx.x;
  const int h = id % a.c.H_kv;
  id /= a.c.H_kv;
  const int f = id % a.frames, b = id / a.frames;
  const int slot = slot_of(a.slots, b, a.c.n_slots);
  const int len = slot_len(a.c.len, slot, a.c.max_pages * PAGE);
  const int n_new = min(min(a.n_new ? max(a.n_new[b], 0) : a.T_max, a.T_max), len);
  const int start = len - n_new;
  const int j = start / PAGE + f;
  if (n_new == 0 || j * PAGE >= len) return;
  const int page = page_at(a.c, slot, j);  // (on its way while the rows are)
  const int lo = max(start - j * PAGE, 0), hi = min(len - j * PAGE, PAGE);
  const void* src = values ? a.v : a.k;
  const size_t ld = values ? a.v_ld : a.k_ld;
  const size_t row0 = (size_t)b * a.T_max + (j * PAGE - start);  // row of the page's token 0 (may wrap; added to below)
  float x[B::kPer][4][8];
#pragma unroll
  for (int u = 0; u < B::kPer; ++u) {
    const int e = threadIdx.x + u * B::kThreads;
    const int c = e % (D / 8) * 8, t0 = e / (D / 8) * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + i;
#pragma unroll
      for (int q = 0; q < 8; ++q) x[u][i][q] = 0.f;
      if (t >= lo && t < hi) load8(src, (row0 + t) * ld + (size_t)h * D + c, x[u][i], E());
    }
  }
  if (page < 0) return;
  const size_t block = (size_t)page * a.c.H_kv + h;
  float* scale = (values ? a.c.v_scale : a.c.k_scale) + block;
  const float held = lo > 0 ? *scale : 0.f;
  // The block's largest magnitude: fmaxf passes NaN by, and infinities, if it finds one, are left out in a second
  // try.  (Both are stored as NaN by the conversion, the other values with the scale that these need.)
  auto largest = [&](float below) {
    float m = 0.f;
#pragma unroll
    for (int u = 0; u < B::kPer; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) m = fabsf(x[u][i][q]) > below ? m : fmaxf(m, fabsf(x[u][i][q]));
    return block_max<B::kThreads>(m, red);
  };
  float m = largest(INFINITY);
  if (m == INFINITY) {
    __syncthreads();  // (every thread has the same m)
    m = largest(FLT_MAX);
  }
  float s = block_scale(m), ratio = 1.f;
  if (lo > 0) {
    if (held >= s) {
      s = held;
    } else {
      ratio = held * pow2_inverse(s);
    }
  }
  store_block<D, PAGE>((values ? a.c.v : a.c.k) + block * (PAGE * D), values, lo, hi, pow2_inverse(s), ratio, x, lds);
  if (threadIdx.x == 0) *scale = s;
}

// A destination block's tokens: source block and place of each, -1 for none.
template <int PAGE>
struct TokenMap {
  int block[PAGE];
  float scale[PAGE];
  u32x4 at[PAGE / 16];  // a byte a token
};

// Block (layer, b, f, h) of a destination, gathered from the source's rows.
// Values lie token last, a byte of each channel apart: a workgroup brings each
// source block that its tokens name into LDS whole, 16 bytes a lane, and takes
// the bytes from there (single bytes from memory, a line each: 37.5 us for 4
// layers of 4 x 1187 of 4259 tokens, this way 20).
//
// With TURNS a workgroup goes on to every frames-th block after its first; without, the launch has one for every
// block that the table can hold.  (4 and 28 layers of 4 sequences, 1187 of 4259 tokens of 4 heads of 128, the table
// 4 and 20 times as long as they are: without 48, 206 and 291, 1432 us, with 32, 32 and 151, 147; as long as they
// are, without: 20 and 109.)
template <int D, int PAGE, bool TURNS>
__global__ __launch_bounds__((Block<D, PAGE>::kThreads)) void compact_kernel(CompactArgs a) {
  using B = Block<D, PAGE>;
  __shared__ uint32_t lds[D * B::kRow];
  __shared__ float red[4];
  __shared__ TokenMap<PAGE> map;
  __shared__ uint64_t s_runs;
  const bool values = blockIdx.y != 0;
  const int tid = threadIdx.x;
  unsigned id = blockIdx.x;
  const int h = (int)(id % a.c.H_kv);
  id /= a.c.H_kv;
  int f = (int)(id % a.frames);
  id /= a.frames;
  const int b = (int)(id % a.B), layer = (int)(id / a.B);
  // the loads that depend on each other go out in three steps: slots and kept rows, lengths and pages,
  // scales and data (the bounds are checked on what came back)
  const int src = slot_of(a.src, b, a.c.n_slots), dst = slot_of(a.dst, b, a.c.n_slots);
  while (true) {
    int r = f * PAGE + min(tid, PAGE - 1);
    const int kept = a.kept[(size_t)b * a.n_kept + min(max(r - a.P, 0), a.n_kept - 1)];
    r = r >= a.P + a.n_kept ? r + a.K_in - a.n_kept : r >= a.P ? a.P + min(max(kept, 0), a.K_in - 1) : r;
    const int L = slot_len(a.c.len, src, a.c.max_pages * PAGE), room = slot_len(a.c.len, dst, a.c.max_pages * PAGE);
    const int page = dst < 0 ? -1 : page_at(a.c, dst, min(f, a.c.max_pages - 1));
    int from = src < 0 ? -1 : page_at(a.c, src, min(r / PAGE, a.c.max_pages - 1));
    const int n = L < a.P + a.K_in || src == dst ? 0 : min(L - a.K_in + a.n_kept, room);
    if (f * PAGE >= n) return;
    if (page >= 0) {
      const int hi = min(n - f * PAGE, PAGE), at = r % PAGE;
      if (tid >= hi) from = -1;
      const size_t layer_blocks = (size_t)layer * a.c.n_pages * a.c.H_kv;
      const uint8_t* data = (values ? a.c.v : a.c.k) + (layer_blocks + h) * (PAGE * D);
      const float* scales = (values ? a.c.v_scale : a.c.k_scale) + layer_blocks + h;
      if (tid < 64) {
        if (tid < PAGE) {
          map.block[tid] = from;
          reinterpret_cast<uint8_t*>(map.at)[tid] = (uint8_t)at;
          map.scale[tid] = from >= 0 ? scales[(size_t)from * a.c.H_kv] : 0.f;
        }
        const int before = __shfl_up(from, 1, 64);
        const uint64_t starts = __ballot(tid < hi && (tid == 0 || from != before));
        if (tid == 0) s_runs = starts;  // tokens whose page is not the one before's
      }
      __syncthreads();
      const size_t block = layer_blocks + (size_t)page * a.c.H_kv + h;
      if (!values) {
        float x[B::kPer][4][8], m = 0.f;
#pragma unroll
        for (int u = 0; u < B::kPer; ++u) {
          const int e = tid + u * B::kThreads;
          const int c = e % (D / 8) * 8, t0 = e / (D / 8) * 4;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int t = t0 + i;
            const int from = t < hi ? map.block[t] : -1;
            const int row = reinterpret_cast<const uint8_t*>(map.at)[t];
            const u32x2 w = from >= 0 ? *reinterpret_cast<const u32x2*>(data + (size_t)from * a.c.H_kv * (PAGE * D) +
                                                                        row * D + c)
                                      : u32x2{0u, 0u};
            float y[2][4];
            from_e4m3(w[0], y[0]);
            from_e4m3(w[1], y[1]);
            const float s = from >= 0 ? map.scale[t] : 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              x[u][i][q] = y[q >> 2][q & 3] * s;
              m = fmaxf(m, fabsf(x[u][i][q]));
            }
          }
        }
        const float s = block_scale(block_max<B::kThreads>(m, red));
        store_block<D, PAGE>(a.c.k + block * (PAGE * D), false, 0, hi, pow2_inverse(s), 1.f, x, lds);
        if (tid == 0) a.c.k_scale[block] = s;
      } else {
        // a thread's items: 16 tokens of a channel, as bytes
        constexpr int kGroups = PAGE / 16, kItems = D * kGroups / B::kThreads;
        static_assert(kItems * B::kThreads == D * kGroups, "whole items");
        u32x4 w[kItems], next[kItems], at16[kItems];
        uint64_t runs = s_runs;
        auto fetch = [&](int t) {
          const int from = map.block[t];
#pragma unroll
          for (int i = 0; i < kItems; ++i)
            next[i] = from >= 0 ? ldg16(data + (size_t)from * a.c.H_kv * (PAGE * D) + (tid + i * B::kThreads) * 16)
                                : zero4();
        };
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
          w[i] = zero4();
          at16[i] = map.at[(tid + i * B::kThreads) % kGroups];
        }
        int r0 = 0;
        fetch(0);
        while (r0 < hi) {
          runs &= runs - 1;
          const int r1 = runs ? __builtin_ctzll(runs) : hi;
#pragma unroll
          for (int i = 0; i < kItems; ++i) {
            const int e = tid + i * B::kThreads;
#pragma unroll
            for (int j = 0; j < 4; ++j) lds[e / kGroups * B::kRow + e % kGroups * 4 + j] = next[i][j];
          }
          __syncthreads();
          if (r1 < hi) fetch(r1);
#pragma unroll
          for (int i = 0; i < kItems; ++i) {
            const int e = tid + i * B::kThreads, t0 = e % kGroups * 16;
            const uint8_t* row = reinterpret_cast<const uint8_t*>(lds + e / kGroups * B::kRow);
            // a byte for every token, those of other blocks dropped: the reads wait for nothing
            uint32_t byte[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) byte[j] = row[(at16[i][j >> 2] >> (8 * (j & 3))) & 0xff];
#pragma unroll
            for (int j = 0; j < 16; ++j)
              w[i][j >> 2] |= t0 + j >= r0 && t0 + j < r1 ? byte[j] << (8 * (j & 3)) : 0u;
          }
          __syncthreads();
          r0 = r1;
        }
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
          const int t0 = (tid + i * B::kThreads) % kGroups * 16;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float y[4];
            from_e4m3(w[i][j], y);
#pragma unroll
            for (int q = 0; q < 4; ++q) m = fmaxf(m, fabsf(y[q]) * map.scale[t0 + 4 * j + q]);
          }
        }
        const float s = block_scale(block_max<B::kThreads>(m, red)), inv = pow2_inverse(s);
        uint8_t* out = a.c.v + block * (PAGE * D);
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
          const int e = tid + i * B::kThreads, t0 = e % kGroups * 16;
          if (t0 >= hi) continue;
          u32x4* to = reinterpret_cast<u32x4*>(out + e * 16);
          u32x4 y = t0 + 16 > hi ? *to : zero4();  // tokens past the last are kept
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float x[4];
            from_e4m3(w[i][j], x);
#pragma unroll
            // (one factor after the other: a block of zeros has the smallest scale, and the product of the two
            // passes fp32's range)
            for (int q = 0; q < 4; ++q) x[q] = x[q] * map.scale[t0 + 4 * j + q] * inv;
            const int n_t = hi - t0 - 4 * j;  // tokens of this word
            const uint32_t mask = n_t >= 4 ? ~0u : n_t <= 0 ? 0u : (1u << (8 * n_t)) - 1u;
            y[j] = (to_e4m3(x[0], x[1], x[2], x[3]) & mask) | (y[j] & ~mask);
          }
          *to = y;
        }
        if (tid == 0) a.c.v_scale[block] = s;
      }
    }
    if (!TURNS || f + a.frames > (n - 1) / PAGE) return;
    f += a.frames;
    __syncthreads();  // the block's LDS is read before the next one's is written
  }
}

// Pair i's page in layer z, 16 bytes a lane and step.
constexpr int kCopyThreads = 256;
__global__ __launch_bounds__(kCopyThreads) void copy_kernel(CopyArgs a) {
  const int i = blockIdx.x, layer = blockIdx.y;
  const int src = a.src[i], dst = a.dst[i];
  if (src < 0 || src >= a.n_pages || dst < 0 || dst >= a.n_pages) return;
  const size_t from = (size_t)layer * a.n_pages + src, to = (size_t)layer * a.n_pages + dst;
  uint8_t* data = blockIdx.z & 1 ? a.v : a.k;
  const int step = gridDim.z / 2 * kCopyThreads * 16;
  for (int o = (blockIdx.z / 2 * kCopyThreads + threadIdx.x) * 16; o < a.page_bytes; o += step)
    *reinterpret_cast<u32x4*>(data + to * a.page_bytes + o) = ldg16(data + from * a.page_bytes + o);
  if (blockIdx.z < 2) {
    float* sc = blockIdx.z & 1 ? a.v_scale : a.k_scale;
    for (int h = threadIdx.x; h < a.H_kv; h += kCopyThreads) sc[to * a.H_kv + h] = sc[from * a.H_kv + h];
  }
}

// One instantiation for every head size and page length.
template <class F>
hipError_t by_shape(int d_head, int page, F f) {
  auto with_page = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (page == 16) f(std::integral_constant<int, D>(), std::integral_constant<int, 16>());
    if (page == 32) f(std::integral_constant<int, D>(), std::integral_constant<int, 32>());
    if (page == 64) f(std::integral_constant<int, D>(), std::integral_constant<int, 64>());
  };
  if (d_head == 64) with_page(std::integral_constant<int, 64>());
  if (d_head == 128) with_page(std::integral_constant<int, 128>());
  if (d_head == 256) with_page(std::integral_constant<int, 256>());
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv8_write(const WriteArgs& a, int dtype, int d_head, int page, hipStream_t s) {
  const dim3 grid((unsigned)((long long)a.B * a.frames * a.c.H_kv), 2);
  return by_shape(d_head, page, [&](auto d, auto p) {
    constexpr int D = decltype(d)::value, PAGE = decltype(p)::value;
    const dim3 block(Block<D, PAGE>::kThreads);
    if (dtype == TREVS_BF16)
      hipLaunchKernelGGL((write_kernel<BF16, D, PAGE>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((write_kernel<F32, D, PAGE>), grid, block, 0, s, a);
  });
}

hipError_t launch_kv8_compact(const CompactArgs& a, int d_head, int page, hipStream_t s) {
  const dim3 grid((unsigned)a.n_layers * a.B * a.frames * a.c.H_kv, 2);
  return by_shape(d_head, page, [&](auto d, auto p) {
    constexpr int D = decltype(d)::value, PAGE = decltype(p)::value;
    const dim3 block(Block<D, PAGE>::kThreads);
    if (a.turns)
      hipLaunchKernelGGL((compact_kernel<D, PAGE, true>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((compact_kernel<D, PAGE, false>), grid, block, 0, s, a);
  });
}

hipError_t launch_kv8_copy(const CopyArgs& a, hipStream_t s) {
  const int chunks = (a.page_bytes + kCopyThreads * 64 - 1) / (kCopyThreads * 64);
  hipLaunchKernelGGL(copy_kernel, dim3(a.n, a.n_layers, 2 * chunks), dim3(kCopyThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace trevs
