// The attention weights that query rows give to each cached token, summed over rows
// and heads and added to the tokens' scores: the weights are formed again from the
// log-sum-exp that the attention left, exp2(f q.k - lse log2 e), so no maximum and no
// value is needed.
//
// Logits are products C = Q K^T on the matrix cores (keys and bf16 queries exact in
// bf16, fp32 queries as three parts): a lane's column of C is one key, so the sum over
// query rows is a sum of its registers, and a key's sum stays in one register
// however many rows pass by.  Nothing is added by atomics: the order of every sum
// follows from the sizes.
#include "rows.hpp"

namespace trevs {
namespace {

constexpr int kKeys = 64;   // keys of a wave: two columns of 32 a lane
constexpr int kRows = 32;   // query rows of a product
constexpr int kMaxWaves = 16;

struct Span2 {
  int slot, rows, L;
};
__device__ __forceinline__ Span2 sequence(const WeightsArgs& a, int b) {
  Span2 s;
  s.slot = slot_of(a.slots, b, a.c.n_slots);
  s.rows = a.q_len ? min(max(a.q_len[b], 0), a.T_max) : a.T_max;
  s.L = slot_len(a.c.len, s.slot, a.kv_max);
  return s;
}

// -lse in base 2; -inf, whose weights are 0, for a row that sees nothing.
__device__ __forceinline__ float row_base(float lse) { return lse == -INFINITY ? -INFINITY : -lse * kLog2e; }

// A wave's 64 keys of KV head h from token j0 on: lane column c holds keys j0 + c and j0 + 32 + c, half of the
// channels each (16 in turn with the other half).  f is their scale, times the logits'; absent keys have `there` 0.
template <int D>
struct Keys {
  u32x4 w[2][D / 32];
  float f[2];
  bool there[2];
  __device__ __forceinline__ void load(const WeightsArgs& a, const Span2& s, int hk, int j0) {
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int32_t* table = a.c.table + (size_t)max(s.slot, 0) * a.c.max_pages;
    int page[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int j = min(j0 + 32 * y + col, max(s.L - 1, 0));
      const int p = table[j >> a.page_shift];
      there[y] = p >= 0 && p < a.c.n_pages;
      page[y] = there[y] ? p : 0;
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int j = min(j0 + 32 * y + col, max(s.L - 1, 0));
      const size_t block = (size_t)page[y] * a.c.H_kv + hk;
      const uint8_t* k = a.c.k + ((block << a.page_shift) + (j & ((1 << a.page_shift) - 1))) * D + 16 * half;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) w[y][c] = ldg16(k + 32 * c);
      f[y] = a.c.k_scale[block] * a.scale_log2e;
    }
  }
};

// ------------------------------------------------------------------ few rows
// A workgroup takes 64 tokens of a sequence, its waves the KV heads in turn; up to 32
// rows a group, whose operand each lane loads for itself.  Bound by the keys' bytes.
template <class E, int D>
__global__ __launch_bounds__(64 * kMaxWaves) void few_rows_kernel(WeightsArgs a) {
  constexpr int NP = kParts<E>;
  __shared__ float sums[kMaxWaves][kKeys];
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), n_waves = blockDim.x >> 6;
  const int b = blockIdx.x / a.key_blocks, kb = blockIdx.x - b * a.key_blocks;
  const Span2 s = sequence(a, b);
  if (s.slot < 0) return;
  const int n_rows = s.rows * a.G, j0 = kb * kKeys;
  float* score = a.score + (size_t)s.slot * a.width;
  if (j0 < s.L) {
    float acc[2] = {0.f, 0.f};
    const int t = col / a.G, g = col - t * a.G;
    const bool live = col < n_rows;
    const int lim = a.causal ? s.L - s.rows + t + 1 : s.L;
    // (rows see more and more keys: the first one's limit is the least)
    const bool whole = !a.causal || s.L - s.rows + 1 >= min(j0 + kKeys, s.L);
    for (int hk = wave; hk < a.c.H_kv && n_rows > 0; hk += n_waves) {
      Keys<D> k;
      k.load(a, s, hk, j0);
      const int h = hk * a.G + g;
      const float nl = live ? row_base(a.lse[((size_t)b * a.H_q + h) * a.T_max + t]) : -INFINITY;
      const size_t at = ((size_t)b * a.T_max + t) * a.q_ld + (size_t)h * D + 16 * half;
      f32x16 x[2];
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[y][i] = 0.f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        float q[8] = {};
        if (live) load_row8(a.q, at + c / 2 * 32 + 8 * (c & 1), q, E());
        bf16x8 qp[NP];
        split_parts<NP>(q, qp);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const u32x4 w = k.w[y][c / 2];
          const bf16x8 kk = c & 1 ? widen(w[2], w[3], 1.f) : widen(w[0], w[1], 1.f);
#pragma unroll
          for (int p = NP - 1; p >= 0; --p) x[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qp[p], kk, x[y], 0, 0, 0);
        }
      }
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (8 * (i >> 2) >= n_rows) break;
        const int row = mfma_row(i, half);
        const float base = __shfl(nl, row, 64);
        const int n = __shfl(lim, row, 64);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const float e = __builtin_amdgcn_exp2f(fmaf(x[y][i], k.f[y], base));
          sum[y] += whole || j0 + 32 * y + col < n ? e : 0.f;
        }
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) acc[y] += k.there[y] ? sum[y] : 0.f;
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      acc[y] += __shfl_xor(acc[y], 32, 64);
      if (half == 0) sums[wave][32 * y + col] = acc[y];
    }
    __syncthreads();
    if (tid < kKeys && j0 + tid < a.width) {
      const int j = j0 + tid;
      float x = 0.f;
      for (int w = 0; w < n_waves; ++w) x += sums[w][tid];
      if (j < s.L)
        score[j] = a.decay == 0.f ? x : fmaf(a.decay, score[j], x);
      else if (a.decay == 0.f)
        score[j] = 0.f;
    }
  }
  if (a.decay != 0.f) return;
  // the blocks of the row past those that hold tokens
  const int held = (s.L + kKeys - 1) / kKeys;
  for (long long j = (kb < held ? (long long)kb + a.key_blocks : kb) * kKeys + tid; j < a.width;
       j += (long long)a.key_blocks * kKeys)
    if (tid < kKeys) score[j] = 0.f;
}

// ----------------------------------------------------------------- many rows
// A workgroup's four waves hold 64 keys each, widened once into registers, while the
// query rows of a group, r = t G + g, pass by 32 at a time, staged in LDS a step ahead.
// Its sums are one of the `splits` parts of its keys' scores, joined by sum_kernel.
template <int D>
__device__ __forceinline__ int query_swizzle(int row) {
  return D == 64 ? (row >> 1) & 7 : row & 15;
}

template <class E, int D>
struct QueryShared {
  static constexpr int kVecs = kRows * D / 8;  // 8 values each
  u32x4 q[2][kParts<E>][kVecs];
  float4 base[2][kRows / 4];
  int4 lim[2][kRows / 4];
};

template <class E, int D>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void many_rows_kernel(WeightsArgs a) {
  constexpr int NP = kParts<E>, kVecs = QueryShared<E, D>::kVecs / 256;
  __shared__ QueryShared<E, D> sh;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // sequences' groups next to each other, so that what reads the same rows meets on one XCD; early keys,
  // which most rows see, first
  const int groups = a.B * a.head_groups;
  const int group = blockIdx.x % groups, rest = blockIdx.x / groups;
  const int b = group / a.head_groups, hg = group - b * a.head_groups;
  const int piece = rest % a.pieces, kb = rest / a.pieces;
  const Span2 s = sequence(a, b);
  const int j0 = kb * 4 * kKeys, jw = j0 + wave * kKeys;
  if (s.slot < 0 || j0 >= s.L) return;
  const int n_rows = s.rows * a.G;
  // row tiles of which some row sees a key of this workgroup, and this piece of them
  const int t_first = a.causal ? max(j0 - (s.L - s.rows), 0) : 0;
  const int tile0 = t_first * a.G / kRows, n_tiles = max((n_rows + kRows - 1) / kRows - tile0, 0);
  const int first = tile0 + (int)((long long)piece * n_tiles / a.pieces);
  const int end = tile0 + (int)((long long)(piece + 1) * n_tiles / a.pieces);
  float acc[2] = {0.f, 0.f};
  for (int hk = hg * a.heads; hk < min((hg + 1) * a.heads, a.c.H_kv); ++hk) {
    if (first >= end) break;
    bf16x8 kk[2][D / 16];
    float f[2];
    bool there[2];
    {
      Keys<D> k;
      k.load(a, s, hk, jw);
#pragma unroll
      for (int y = 0; y < 2; ++y) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          kk[y][2 * c] = widen(k.w[y][c][0], k.w[y][c][1], 1.f);
          kk[y][2 * c + 1] = widen(k.w[y][c][2], k.w[y][c][3], 1.f);
        }
        f[y] = k.f[y];
        there[y] = k.there[y];
      }
    }
    float q[kVecs][8], base = 0.f;
    int lim = 0;
    auto load = [&](int tile) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int e = tid + 256 * i, r = tile * kRows + e / (D / 8), t = r / a.G, g = r - t * a.G;
#pragma unroll
        for (int j = 0; j < 8; ++j) q[i][j] = 0.f;
        if (r < n_rows)
          load_row8(a.q, ((size_t)b * a.T_max + t) * a.q_ld + (size_t)(hk * a.G + g) * D + e % (D / 8) * 8, q[i], E());
      }
      if (tid < kRows) {
        const int r = tile * kRows + tid, t = r / a.G, h = hk * a.G + r - t * a.G;
        base = r < n_rows ? row_base(a.lse[((size_t)b * a.H_q + h) * a.T_max + t]) : -INFINITY;
        lim = r >= n_rows ? 0 : a.causal ? s.L - s.rows + t + 1 : s.L;
      }
    };
    auto store = [&](int buf) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int e = tid + 256 * i, r = e / (D / 8), c = e % (D / 8);
        bf16x8 parts[NP];
        split_parts<NP>(q[i], parts);
#pragma unroll
        for (int p = 0; p < NP; ++p)
          sh.q[buf][p][r * (D / 8) + (c ^ query_swizzle<D>(r))] = __builtin_bit_cast(u32x4, parts[p]);
      }
      if (tid < kRows) {
        reinterpret_cast<float*>(sh.base[buf])[tid] = base;
        reinterpret_cast<int*>(sh.lim[buf])[tid] = lim;
      }
    };
    __syncthreads();  // (the head before has read its last tile)
    load(first);
    store(0);
    __syncthreads();
    for (int tile = first; tile < end; ++tile) {
      const int buf = (tile - first) & 1;
      load(min(tile + 1, end - 1));
      // rows see more and more keys: the tile's first and last rows' limits
      const int least = a.causal ? s.L - s.rows + tile * kRows / a.G + 1 : s.L;
      const int most = a.causal ? s.L - s.rows + min(tile * kRows + kRows - 1, n_rows - 1) / a.G + 1 : s.L;
      if (jw < most) {
        f32x16 x[2];
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int i = 0; i < 16; ++i) x[y][i] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
          for (int p = NP - 1; p >= 0; --p) {
            const int chunk = c / 2 * 4 + 2 * half + (c & 1);
            const bf16x8 qq =
                __builtin_bit_cast(bf16x8, sh.q[buf][p][col * (D / 8) + (chunk ^ query_swizzle<D>(col))]);
#pragma unroll
            for (int y = 0; y < 2; ++y)
              x[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qq, kk[y][c], x[y], 0, 0, 0);
          }
        float sum[2] = {0.f, 0.f};
        if (least >= min(jw + kKeys, s.L)) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 n = sh.base[buf][2 * i + half];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              sum[y] += __builtin_amdgcn_exp2f(fmaf(x[y][4 * i], f[y], n.x));
              sum[y] += __builtin_amdgcn_exp2f(fmaf(x[y][4 * i + 1], f[y], n.y));
              sum[y] += __builtin_amdgcn_exp2f(fmaf(x[y][4 * i + 2], f[y], n.z));
              sum[y] += __builtin_amdgcn_exp2f(fmaf(x[y][4 * i + 3], f[y], n.w));
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 n = sh.base[buf][2 * i + half];
            const int4 l = sh.lim[buf][2 * i + half];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int j = jw + 32 * y + col;
              const float e0 = __builtin_amdgcn_exp2f(fmaf(x[y][4 * i], f[y], n.x));
              const float e1 = __builtin_amdgcn_exp2f(fmaf(x[y][4 * i + 1], f[y], n.y));
              const float e2 = __builtin_amdgcn_exp2f(fmaf(x[y][4 * i + 2], f[y], n.z));
              const float e3 = __builtin_amdgcn_exp2f(fmaf(x[y][4 * i + 3], f[y], n.w));
              sum[y] += j < l.x ? e0 : 0.f;
              sum[y] += j < l.y ? e1 : 0.f;
              sum[y] += j < l.z ? e2 : 0.f;
              sum[y] += j < l.w ? e3 : 0.f;
            }
          }
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) acc[y] += there[y] ? sum[y] : 0.f;
      }
      store(buf ^ 1);
      __syncthreads();
    }
  }
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    acc[y] += __shfl_xor(acc[y], 32, 64);
    const int j = jw + 32 * y + col;
    if (half == 0 && j < s.L) a.part[((size_t)(b * a.head_groups + hg) * a.pieces + piece) * a.kv_max + j] = acc[y];
  }
}

// The parts of each token's sum, in their order.
constexpr int kSumThreads = 256;
__global__ __launch_bounds__(kSumThreads) void sum_kernel(WeightsArgs a) {
  const int b = blockIdx.y;
  const Span2 s = sequence(a, b);
  if (s.slot < 0) return;
  const int splits = a.head_groups * a.pieces;
  const float* part = a.part + (size_t)b * splits * a.kv_max;
  float* score = a.score + (size_t)s.slot * a.width;
  const int end = a.decay == 0.f ? a.width : s.L;
  for (long long j = (long long)blockIdx.x * kSumThreads + threadIdx.x; j < end; j += (long long)gridDim.x * kSumThreads) {
    float x = 0.f;
    if (j < s.L) {
#pragma unroll 8
      for (int i = 0; i < splits; ++i) x += part[(size_t)i * a.kv_max + j];
      if (a.decay != 0.f) x = fmaf(a.decay, score[j], x);
    }
    score[j] = x;
  }
}

template <class E, int D>
hipError_t launch(const WeightsArgs& a, const WeightsPlan& p, hipStream_t s) {
  if (p.few) {
    hipLaunchKernelGGL((few_rows_kernel<E, D>), dim3((unsigned)(a.B * (long long)a.key_blocks)),
                       dim3(64 * std::min(a.c.H_kv, kMaxWaves)), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((many_rows_kernel<E, D>),
                     dim3((unsigned)((long long)a.B * a.head_groups * a.pieces * a.key_blocks)), dim3(256), 0, s, a);
  const int tokens = a.decay == 0.f ? a.width : a.kv_max;
  const unsigned blocks = (unsigned)std::min((tokens + kSumThreads - 1LL) / kSumThreads, 65536LL / a.B + 1);
  hipLaunchKernelGGL(sum_kernel, dim3(blocks, a.B), dim3(kSumThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

WeightsPlan weights_plan(int B, int T_max, int H_kv, int G, int kv_max) {
  WeightsPlan p = {};
  const long long n_rows = (long long)T_max * G;
  p.few = n_rows <= kRows;
  p.key_blocks = p.few ? (kv_max + kKeys - 1) / kKeys : (kv_max + 4 * kKeys - 1) / (4 * kKeys);
  p.heads = 1;
  p.head_groups = H_kv;
  p.pieces = 1;
  if (p.few) return p;
  const long long row_tiles = (n_rows + kRows - 1) / kRows, want = 2048;
  // the parts' floats: 64 MB at most, where splitting the heads alone does not pass that
  const long long most = std::max((16LL << 20) / ((long long)B * kv_max), 1LL);
  if (most < H_kv) {
    p.heads = (int)((H_kv + most - 1) / most);
    p.head_groups = (H_kv + p.heads - 1) / p.heads;
  } else {
    const long long units = (long long)B * H_kv * p.key_blocks;
    p.pieces = (int)std::max(std::min({(want + units - 1) / units, row_tiles / 4, most / H_kv}), 1LL);
  }
  return p;
}

hipError_t launch_kv8_weights(const WeightsArgs& a, const WeightsPlan& p, int dtype, int d_head, hipStream_t s) {
  auto by_head = [&](auto e) {
    using E = decltype(e);
    if (d_head == 64) return launch<E, 64>(a, p, s);
    if (d_head == 128) return launch<E, 128>(a, p, s);
    return launch<E, 256>(a, p, s);
  };
  return dtype == TREVS_BF16 ? by_head(BF16()) : by_head(F32());
}

}  // namespace trevs
