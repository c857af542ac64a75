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
#include <type_traits>

#include "rows.hpp"
#include "cut.hpp"

namespace trevs {
namespace {

constexpr int kKeys = 64;   // keys of a wave: two columns of 32 a lane
constexpr int kRows = 32;   // query rows of a product

struct Seq {
  int slot, rows, L;
};
__device__ __forceinline__ Seq sequence(const WeightsArgs& a, int b) {
  Seq s;
  s.slot = slot_of(a.slots, b, a.c.n_slots);
  s.rows = a.q_len ? min(max(a.q_len[b], 0), a.T_max) : a.T_max;
  s.L = slot_len(a.c.len, s.slot, a.kv_max);
  return s;
}

// -lse in base 2; -inf, whose weights are 0, for a row that sees nothing.
__device__ __forceinline__ float row_base(float lse) { return lse == -INFINITY ? -INFINITY : -lse * kLog2e; }

// 8 values of a row as they lie, and their parts.
template <class E>
struct Raw {
  u32x4 w[E::kBytes / 2];
  __device__ __forceinline__ void load(const void* q, size_t i) {
    const u32x4* p = reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(q) + i * E::kBytes);
#pragma unroll
    for (int j = 0; j < E::kBytes / 2; ++j) w[j] = ldg16(p + j);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < E::kBytes / 2; ++j) w[j] = zero4();
  }
  __device__ __forceinline__ void parts(u32x4 (&out)[kParts<E>]) const {
    if constexpr (E::kBytes == 2) {
      out[0] = w[0];
    } else {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(w[j >> 2][j & 3]);
      bf16x8 y[kParts<E>];
      split_parts<kParts<E>>(x, y);
#pragma unroll
      for (int p = 0; p < kParts<E>; ++p) out[p] = __builtin_bit_cast(u32x4, y[p]);
    }
  }
};

// Where a wave's 64 keys lie, of every KV head: lane column c holds keys j0 + c and j0 + 32 + c, half of the
// channels each (16 in turn with the other half).
struct Places {
  size_t block[2];  // page, counted in KV heads' blocks
  int row[2];       // in the page
  bool there[2];
  __device__ __forceinline__ Places(const WeightsArgs& a, const Seq& s, int j0) {
    const int col = threadIdx.x & 31;
    const int32_t* table = a.c.table + (size_t)max(s.slot, 0) * a.c.max_pages;
    int page[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int j = min(j0 + 32 * y + col, max(s.L - 1, 0));
      page[y] = table[j >> a.page_shift];
      row[y] = j & ((1 << a.page_shift) - 1);
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      there[y] = page[y] >= 0 && page[y] < a.c.n_pages;
      block[y] = (size_t)(there[y] ? page[y] : 0) * a.c.H_kv;
    }
  }
};
// Channels [C0, C0 + C) of them in KV head hk, 16 bytes a vector.
template <int D, int C>
__device__ __forceinline__ void load_keys(const WeightsArgs& a, const Places& at, int hk, int c0, u32x4 (&w)[2][C / 32]) {
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const uint8_t* k = a.c.k + (((at.block[y] + hk) << a.page_shift) + at.row[y]) * D + c0 + 16 * half;
#pragma unroll
    for (int c = 0; c < C / 32; ++c) w[y][c] = ldg16(k + 32 * c);
  }
}

// ------------------------------------------------------------------ few rows
// Products of 16 x 16: a load takes 64 bytes of each of 16 keys.  A workgroup takes
// tokens of one sequence, its waves the KV heads in turn, the group's rows in NQ tiles
// of 16.  Bound by the keys' bytes: a wave's rows stay in its registers over the blocks
// of a sequence, pages are looked up two blocks ahead and keys loaded one, where there
// are registers for two (one token of 64 sequences of 1.2 k to 16.5 k tokens, 28/4
// heads of 128: 60 us, 4.9 TB/s; beside 62, with the keys of one block 66, streamed past
// the caches 68, as products of 32 x 32, 32 bytes of each of 32 keys, 83).  In fp32 two
// waves share a SIMD and wait for half of their time (32 sequences of 1 k to 8 k tokens:
// 22 us, 3.4 TB/s; matrix cores busy for 15 % of the cycles, vector units for 39 %).
// Two tiles of 256 channels spill 20 to 41 registers: 3 or 4 rows of 8 sequences of 8 k to
// 12 k tokens, 8/1 heads, take 18 us, with the kernel of many rows 14.5; of 2 sequences of
// 2 k to 3 k 4.2 (16 tokens a workgroup) and 8.1; one row of 8 of 4 k to 8 k, 320/10 heads,
// 43 and 50.
constexpr int kRun = 8;  // blocks whose sums are joined at once

// The calling wave's part of the sums of `run` blocks of 16 Y tokens from j0 on.
template <class E, int D, int Y, int NQ>
struct FewRows {
  Raw<E> q[NQ][D / 32];
  float nl[NQ];  // of row 16 m + lane % 16
  int lim[NQ];
  __device__ __forceinline__ void load(const WeightsArgs& a, const Seq& s, int b, int hk) {
    const int n16 = threadIdx.x & 15, g4 = (threadIdx.x & 63) >> 4, n_rows = s.rows * a.G;
#pragma unroll
    for (int m = 0; m < NQ; ++m) {
      // (a lane past the last row has the first one's: its weights come to nothing)
      const int r = 16 * m + n16;
      const bool live = r < n_rows;
      const int t = live ? r / a.G : 0, h = hk * a.G + (live ? r - t * a.G : 0);
      const size_t at = ((size_t)b * a.T_max + t) * a.q_ld + (size_t)h * D + 16 * g4;
      const float lse = a.lse[((size_t)b * a.H_q + h) * a.T_max + t];
#pragma unroll
      for (int c = 0; c < D / 32; ++c) q[m][c].load(a.q, at + c / 2 * 64 + 8 * (c & 1));
      nl[m] = live ? lse : -INFINITY;
      lim[m] = a.causal ? s.L - s.rows + t + 1 : s.L;
    }
  }
  __device__ __forceinline__ void add(const WeightsArgs& a, const Seq& s, int hk, int j0, int run, bool first,
                                      float* sums) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    constexpr int NP = kParts<E>;
    const int n16 = threadIdx.x & 15, g4 = (threadIdx.x & 63) >> 4;
    const int32_t* table = a.c.table + (size_t)s.slot * a.c.max_pages;
    int page[Y];
    auto look_up = [&](int u) {
#pragma unroll
      for (int y = 0; y < Y; ++y) page[y] = table[min(j0 + 16 * (u * Y + y) + n16, s.L - 1) >> a.page_shift];
    };
    // (registers for a second block's keys)
    constexpr bool kAhead = D <= 128 || (NQ == 1 && NP == 1);
    look_up(0);
    u32x4 w[Y][D / 64], next[Y][D / 64];
    float f[Y], next_f[Y];
    bool there[Y], next_there[Y];
    auto load = [&](int u) {
#pragma unroll
      for (int y = 0; y < Y; ++y) {
        next_there[y] = page[y] >= 0 && page[y] < a.c.n_pages;
        const size_t block = (size_t)(next_there[y] ? page[y] : 0) * a.c.H_kv + hk;
        const int row = min(j0 + 16 * (u * Y + y) + n16, s.L - 1) & ((1 << a.page_shift) - 1);
        const uint8_t* k = a.c.k + (block << a.page_shift) * D + row * D + 16 * g4;
#pragma unroll
        for (int c = 0; c < D / 64; ++c) next[y][c] = ldg16(k + 64 * c);
        next_f[y] = a.c.k_scale[block] * a.scale_log2e;
      }
    };
    if (kAhead) {
      load(0);
      look_up(1);
    }
    // rows that give nothing are zeros: exp2(NaN - inf) is NaN (here, not with their loads, which the keys'
    // would wait for)
#pragma unroll
    for (int m = 0; m < NQ; ++m) {
      const bool none = nl[m] == -INFINITY;
      if (__any(none)) {
        if (none) {
#pragma unroll
          for (int c = 0; c < D / 32; ++c) q[m][c].clear();
        }
      }
    }
#pragma unroll 1
    for (int u = 0; u < run; ++u) {
      const int j = j0 + 16 * u * Y;
      if (!kAhead) load(u);
#pragma unroll
      for (int y = 0; y < Y; ++y) {
        f[y] = next_f[y];
        there[y] = next_there[y];
#pragma unroll
        for (int c = 0; c < D / 64; ++c) w[y][c] = next[y][c];
      }
      if (kAhead && u + 1 < run) load(u + 1);
      look_up(u + (kAhead ? 2 : 1));
      // (rows see more and more keys: the first one's limit is the least)
      const bool whole = !a.causal || s.L - s.rows + 1 >= min(j + 16 * Y, s.L);
      float sum[Y];
#pragma unroll
      for (int y = 0; y < Y; ++y) sum[y] = 0.f;
#pragma unroll
      for (int m = 0; m < NQ; ++m) {
        f32x4 x[Y];
#pragma unroll
        for (int y = 0; y < Y; ++y) x[y] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          u32x4 qp[NP];
          q[m][c].parts(qp);
#pragma unroll
          for (int y = 0; y < Y; ++y) {
            const u32x4 v = w[y][c / 2];
            const bf16x8 kk = c & 1 ? widen(v[2], v[3], 1.f) : widen(v[0], v[1], 1.f);
#pragma unroll
            for (int p = NP - 1; p >= 0; --p)
              x[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, qp[p]), kk, x[y], 0, 0, 0);
          }
        }
        // register i of a lane is row 4 g4 + i of the 16
        const float nl_m = row_base(nl[m]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float base = __shfl(nl_m, 4 * g4 + i, 64);
          const int n = whole ? 0 : __shfl(lim[m], 4 * g4 + i, 64);
#pragma unroll
          for (int y = 0; y < Y; ++y) {
            const float e = __builtin_amdgcn_exp2f(fmaf(x[y][i], f[y], base));
            sum[y] += whole || j + 16 * y + n16 < n ? e : 0.f;
          }
        }
      }
#pragma unroll
      for (int y = 0; y < Y; ++y) {
        float e = there[y] ? sum[y] : 0.f;
        e += __shfl_xor(e, 16, 64);
        e += __shfl_xor(e, 32, 64);
        float* to = sums + 16 * (u * Y + y) + n16;
        if (g4 == 0) *to = first ? e : *to + e;
      }
    }
  }
};

// The waves' sums of tokens [j0, j1), in the waves' order, into the scores; a thread has PER of the old ones.
template <int PER>
__device__ __forceinline__ void old_scores(const WeightsArgs& a, const Seq& s, int j0, int j1, float (&was)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = j0 + threadIdx.x + i * blockDim.x;
    was[i] = a.decay != 0.f && j < j1 ? a.score[(size_t)s.slot * a.width + j] : 0.f;
  }
}
template <int PER>
__device__ __forceinline__ void join_waves(const WeightsArgs& a, const Seq& s, int j0, int j1, const float (&was)[PER],
                                           int n_waves, const float* sums, int stride) {
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = threadIdx.x + i * blockDim.x;
    if (j0 + e >= j1) return;
    float x = 0.f;
    for (int w = 0; w < n_waves; ++w) x += sums[w * stride + e];
    a.score[(size_t)s.slot * a.width + j0 + e] = a.decay == 0.f ? x : fmaf(a.decay, was[i], x);
  }
}

// Calls of few tokens: 16 to a workgroup, and a wave to each of up to 16 heads.
template <class E, int D, int NQ>
__global__ __launch_bounds__(1024) void short_kernel(WeightsArgs a) {
  __shared__ float sums[16][16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n_waves = blockDim.x >> 6;
  const int b = blockIdx.x / a.key_blocks, kb = blockIdx.x - b * a.key_blocks, j0 = kb * 16;
  const Seq s = sequence(a, b);
  if (s.slot < 0) return;
  if (j0 < s.L) {
    const int j1 = min(j0 + 16, s.L);
    float was[1];
    old_scores(a, s, j0, j1, was);
    if (s.rows == 0 && (threadIdx.x & 63) < 16) sums[wave][threadIdx.x & 15] = 0.f;
    for (int hk = wave; hk < a.c.H_kv && s.rows > 0; hk += n_waves) {
      FewRows<E, D, 1, NQ> rows;
      rows.load(a, s, b, hk);
      rows.add(a, s, hk, j0, 1, hk == wave, sums[wave]);
    }
    __syncthreads();
    join_waves(a, s, j0, j1, was, n_waves, &sums[0][0], 16);
  }
  if (a.decay != 0.f) return;
  // zeros behind the sequence
  float* score = a.score + (size_t)s.slot * a.width;
  if (threadIdx.x >= 16) return;
  for (long long j = kb * 16LL + threadIdx.x; j < a.width; j += a.key_blocks * 16LL)
    if (j >= s.L) score[j] = 0.f;
}

// The 64-token blocks of all sequences, one after the other, in equal pieces, a
// workgroup to a piece, as many as the GPU holds at once (kFewPerCu a CU, by the
// registers).  With a workgroup to every block or four the lengths of the sequences
// leave a last round that is mostly idle.  More than 8 KV heads take 8 waves (16
// sequences of 2 k to 8 k tokens, 32 heads: 69 us, 73 with 4; in fp32 51 and 101),
// fewer 4 (8 heads: 61 us, 62 with 8).
template <class E, int D, int WAVES, int NQ>
constexpr int kFewPerCu = WAVES == 8 || (D == 256 && E::kBytes == 4) ? 1 : NQ == 1 && D <= 128 && E::kBytes == 2 ? 3 : 2;
template <class E, int D, int WAVES, int NQ>
__global__ __launch_bounds__(64 * WAVES, (kFewPerCu<E, D, WAVES, NQ> * WAVES / 4)) void few_rows_kernel(WeightsArgs a) {
  constexpr int kPer = (kRun + WAVES - 1) / WAVES;  // tokens of a thread
  __shared__ float sums[WAVES][64 * kRun];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto blocks_of = [&](int b) { return b < a.B ? (sequence(a, b).L + 63) / 64 : 0; };
  auto scan = [&](int b0) { return wave_incl_scan(blocks_of(b0 + lane), lane); };
  int ends = scan(0), total = __builtin_amdgcn_readlane(ends, 63);
  for (int b0 = 64; b0 < a.B; b0 += 64) total += __builtin_amdgcn_readlane(scan(b0), 63);
  const Cut cut(total, gridDim.x);
  if ((int)blockIdx.x < cut.n) {
    int at = cut.start(blockIdx.x);
    const int end = cut.start(blockIdx.x + 1);
    int before = 0, b0 = 0;
    while (before + __builtin_amdgcn_readlane(ends, 63) <= at) {
      before += __builtin_amdgcn_readlane(ends, 63);
      b0 += 64;
      ends = scan(b0);
    }
    const int i = __builtin_ctzll(__ballot(before + ends > at));
    int b = b0 + i, block = at - before - (i ? __builtin_amdgcn_readlane(ends, i - 1) : 0);
    Seq s = sequence(a, b);
    FewRows<E, D, 4, NQ> rows;
    bool held = false;  // the rows of the wave's first head, if it has no other
    while (true) {
      const int left = (s.L + 63) / 64 - block, run = min(min(left, end - at), kRun);
      const int j0 = block * 64, j1 = min(j0 + 64 * run, s.L);
      float was[kPer];
      old_scores(a, s, j0, j1, was);
      if (s.rows == 0 || wave >= a.c.H_kv)
        for (int e = lane; e < 64 * kRun; e += 64) sums[wave][e] = 0.f;
      for (int hk = wave; hk < a.c.H_kv && s.rows > 0; hk += WAVES) {
        if (!held || a.c.H_kv > WAVES) rows.load(a, s, b, hk);
        rows.add(a, s, hk, j0, run, hk == wave, sums[wave]);
      }
      held = true;
      __syncthreads();
      join_waves(a, s, j0, j1, was, WAVES, &sums[0][0], 64 * kRun);
      at += run;
      block += run;
      if (at >= end) break;
      if (run == left) {  // to the next sequence that has tokens (there is one)
        do {
          s = sequence(a, ++b);
        } while (s.L == 0);
        block = 0;
        held = false;
      }
      __syncthreads();  // the sums are read before the next ones are written
    }
  }
  if (a.decay != 0.f) return;
  // zeros behind the sequences
  const int per = (a.width + 64 * WAVES - 1) / (64 * WAVES);
  for (long long e = blockIdx.x; e < (long long)a.B * per; e += gridDim.x) {
    const int b = (int)(e / per);
    const long long j = (e - (long long)b * per) * (64 * WAVES) + tid;
    const Seq s = sequence(a, b);
    if (s.slot >= 0 && j >= s.L && j < a.width) a.score[(size_t)s.slot * a.width + j] = 0.f;
  }
}

// ----------------------------------------------------------------- many rows
// A workgroup's four waves hold 64 keys each, widened once into registers, while the
// query rows of a group, r = t G + g, pass by, staged in LDS a step ahead.  Its sums are
// one of the parts of its keys' scores, joined by sum_kernel.  Bound by the vector units
// and the matrix cores, half of the time one after the other: of a pass over prompts of
// 4 x 4259 rows with 28/4 heads of 128 (303 us, 860 TFLOP/s) the former are busy for 57 %
// of the cycles, a third of that with exponentials, the latter for 41 %, and one or the
// other for 80 %.  (The exponentials of one product placed among the instructions of the
// next: 344 us beside 330.)

// Permutation of a staged row's 16-byte columns, by the row's low bits reversed: 16 lanes
// next to each other read one column of 16 rows, or write 4 or 8 columns of 4 or 2 rows,
// and meet 16 different ones modulo 256 bytes, the width of the banks, either way.
template <int D>
__device__ __forceinline__ int query_swizzle(int row) {
  return (int)(D == 64 ? __brev((uint32_t)row >> 1) >> 29 : __brev((uint32_t)row) >> 28);
}

// Rows staged at once: two products' for bf16 rows of up to 128 channels.
template <class E, int D>
constexpr int kStage = E::kBytes == 2 && D <= 128 ? 2 * kRows : kRows;

template <class E, int D>
struct QueryShared {
  static constexpr int kVecs = kStage<E, D> * D / 8;  // 8 values each
  u32x4 q[2][kParts<E>][kVecs];
  float4 base[2][kStage<E, D> / 4];
  int4 lim[2][kStage<E, D> / 4];
};

// The weights of a product's rows for a lane's two keys, summed.  MASKED: a row sees the tokens below its limit.
template <bool MASKED>
__device__ __forceinline__ void add_weights(const f32x16 (&x)[2], const float (&f)[2], int j, const float4* base,
                                            const int4* lim, float (&sum)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 n = base[2 * i];
    const float nn[4] = {n.x, n.y, n.z, n.w};
    int ll[4];
    if constexpr (MASKED) {
      const int4 l = lim[2 * i];
      ll[0] = l.x, ll[1] = l.y, ll[2] = l.z, ll[3] = l.w;
    }
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float e = __builtin_amdgcn_exp2f(fmaf(x[y][4 * i + q], f[y], nn[q]));
        if constexpr (MASKED)
          sum[y] += j + 32 * y < ll[q] ? e : 0.f;
        else
          sum[y] += e;
      }
  }
}

template <class E, int D>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void many_rows_kernel(WeightsArgs a) {
  constexpr int NP = kParts<E>, S = kStage<E, D>, kVecs = QueryShared<E, D>::kVecs / 256;
  __shared__ QueryShared<E, D> sh;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // sequences' groups next to each other, so that what reads the same rows meets on one XCD; early keys,
  // which most rows see, first
  const int groups = a.B * a.head_groups;
  const int group = blockIdx.x % groups, rest = blockIdx.x / groups;
  const int b = group / a.head_groups, hg = group - b * a.head_groups;
  const int piece = rest % a.pieces, kb = rest / a.pieces;
  const Seq s = sequence(a, b);
  const int j0 = kb * 4 * kKeys, jw = j0 + wave * kKeys;
  if (s.slot < 0 || j0 >= s.L) return;
  const int n_rows = s.rows * a.G;
  // stages of which some row sees a key of this workgroup, and this piece of them
  const int t_first = a.causal ? max(j0 - (s.L - s.rows), 0) : 0;
  const int stage0 = t_first * a.G / S, n_stages = max((n_rows + S - 1) / S - stage0, 0);
  const int first = stage0 + (int)((long long)piece * n_stages / a.pieces);
  const int end = stage0 + (int)((long long)(piece + 1) * n_stages / a.pieces);
  float acc[2] = {0.f, 0.f};
  const Places at_keys(a, s, jw);
  for (int hk = hg * a.heads; hk < min((hg + 1) * a.heads, a.c.H_kv); ++hk) {
    if (first >= end) break;
    // A thread stages parts of every S-th row: it follows the row's place.  (Dividing the row's number by G
    // takes as long as the exponentials; for the log-sum-exps alone it takes 8 of 308 us of 4 x 4259 rows.)
    constexpr int kPer = 256 / S;  // threads of a row, which has kPer * kVecs vectors
    static_assert(kPer * kVecs == D / 8, "whole rows");
    Raw<E> raw[kVecs];
    const long long step = (long long)(S / a.G) * a.q_ld + S % a.G * D, wrap = a.q_ld - (long long)a.G * D;
    const int in_row = tid / kPer, vec = tid % kPer;
    int row = first * S + in_row, g = row % a.G;
    const size_t head = (size_t)b * a.T_max * a.q_ld + (size_t)hk * a.G * D + vec * 8;
    const size_t head_lse = ((size_t)b * a.H_q + hk * a.G) * a.T_max;
    int t = row / a.G;
    size_t at = head + (size_t)t * a.q_ld + g * D, at_lse = head_lse + (size_t)g * a.T_max + t;
    float base = 0.f;
    int lim = 0;
    auto load = [&] {
      const bool live = row < n_rows;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) raw[i].load(a.q, (live ? at : head) + i * (kPer * 8));
      base = live ? a.lse[at_lse] : -INFINITY;
      lim = !live ? 0 : a.causal ? s.L - s.rows + t + 1 : s.L;
      row += S;
      at += step;
      g += S % a.G;
      const bool over = g >= a.G;
      at += over ? wrap : 0;
      g -= over ? a.G : 0;
      t += S / a.G + over;
      at_lse = head_lse + (size_t)g * a.T_max + t;
    };
    auto store = [&](int buf) {
      // places past the last row are zeros, as are rows that give nothing: products that take no limits drop
      // them by their base alone, and exp2(NaN - inf) is NaN
      const bool none = base == -INFINITY;
      if (__any(none)) {
        if (none) {
#pragma unroll
          for (int i = 0; i < kVecs; ++i) raw[i].clear();
        }
      }
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        u32x4 parts[NP];
        raw[i].parts(parts);
#pragma unroll
        for (int p = 0; p < NP; ++p)
          sh.q[buf][p][in_row * (D / 8) + ((vec + i * kPer) ^ query_swizzle<D>(in_row))] = parts[p];
      }
      if (vec == 0) {
        reinterpret_cast<float*>(sh.base[buf])[in_row] = row_base(base);
        reinterpret_cast<int*>(sh.lim[buf])[in_row] = lim;
      }
    };
    load();
    bf16x8 kk[2][D / 16];
    float f[2], sum[2] = {0.f, 0.f};
    {
      u32x4 w[2][D / 32];
      load_keys<D, D>(a, at_keys, hk, 0, w);
#pragma unroll
      for (int y = 0; y < 2; ++y) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          kk[y][2 * c] = widen(w[y][c][0], w[y][c][1], 1.f);
          kk[y][2 * c + 1] = widen(w[y][c][2], w[y][c][3], 1.f);
        }
        f[y] = a.c.k_scale[at_keys.block[y] + hk] * a.scale_log2e;
      }
    }
    store(0);  // (the head before ended with a barrier behind its last reads)
    __syncthreads();
    for (int stage = first; stage < end; ++stage) {
      const int buf = (stage - first) & 1;
      if (stage + 1 < end) load();
      // rows see more and more keys: the limits of the stage's first and last one
      const int least = a.causal ? s.L - s.rows + stage * S / a.G + 1 : s.L;
      const int most = a.causal ? s.L - s.rows + min(stage * S + S - 1, n_rows - 1) / a.G + 1 : s.L;
      if (jw < most) {
        f32x16 x[S / kRows][2];
        auto product = [&](int u) {
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[u][y][i] = 0.f;
#pragma unroll
          for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int p = NP - 1; p >= 0; --p) {
              const int chunk = c / 2 * 4 + 2 * half + (c & 1), r = u * kRows + col;
              const bf16x8 qq =
                  __builtin_bit_cast(bf16x8, sh.q[buf][p][r * (D / 8) + (chunk ^ query_swizzle<D>(r))]);
#pragma unroll
              for (int y = 0; y < 2; ++y)
                x[u][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qq, kk[y][c], x[u][y], 0, 0, 0);
            }
        };
        const float4* bases = sh.base[buf] + half;
        const int4* lims = sh.lim[buf] + half;
        float part[2] = {0.f, 0.f};
        if (least >= min(jw + kKeys, s.L)) {
#pragma unroll
          for (int u = 0; u < S / kRows; ++u) product(u);
#pragma unroll
          for (int u = 0; u < S / kRows; ++u) add_weights<false>(x[u], f, 0, bases + u * (kRows / 4), lims, part);
        } else {
#pragma unroll
          for (int u = 0; u < S / kRows; ++u) {
            product(u);
            add_weights<true>(x[u], f, jw + col, bases + u * (kRows / 4), lims + u * (kRows / 4), part);
          }
        }
        sum[0] += part[0];
        sum[1] += part[1];
      }
      if (stage + 1 < end) store(buf ^ 1);
      __syncthreads();
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) acc[y] += at_keys.there[y] ? sum[y] : 0.f;
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
  const Seq s = sequence(a, b);
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
    const long long blocks = (long long)a.B * a.key_blocks;
    auto go = [&](auto kernel, long long groups, int waves) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(blocks, groups)), dim3(64 * waves), 0, s, a);
    };
    auto by_rows = [&](auto nq) {
      constexpr int NQ = decltype(nq)::value;
      if (p.tokens == 16)
        go(short_kernel<E, D, NQ>, blocks, std::min(a.c.H_kv, 16));
      else
        a.c.H_kv <= 8 ? go(few_rows_kernel<E, D, 4, NQ>, 256 * kFewPerCu<E, D, 4, NQ>, 4)
                      : go(few_rows_kernel<E, D, 8, NQ>, 256 * kFewPerCu<E, D, 8, NQ>, 8);
    };
    if (a.T_max * a.G <= 16) by_rows(std::integral_constant<int, 1>());
    if constexpr (E::kBytes == 2) {
      if (a.T_max * a.G > 16) by_rows(std::integral_constant<int, 2>());
    }
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

WeightsPlan weights_plan(int B, int T_max, int H_kv, int G, int kv_max, int dtype) {
  WeightsPlan p = {};
  const long long n_rows = (long long)T_max * G;
  // (two tiles of fp32 rows and a block of keys pass the registers)
  p.few = n_rows <= 16 || (n_rows <= 32 && dtype == TREVS_BF16);
  // few rows: calls that leave most CUs without a workgroup of 64 tokens take 16 in each
  p.tokens = !p.few ? 4 * kKeys : (long long)B * kv_max < 64 * 128 ? 16 : 64;
  p.key_blocks = (kv_max + p.tokens - 1) / p.tokens;
  p.heads = 1;
  p.head_groups = H_kv;
  p.pieces = 1;
  if (p.few) return p;
  // Two workgroups of a CU at once, and as many again for those that see fewer rows (with twice as many prompts
  // of 4 x 2048 rows with 8/1 heads of 256 take 87 us for 75, of 2 x 2048 with 28/4 of 128 in fp32 115 for 106, of
  // 4 x 4259 in bf16 300 for 308); the parts' floats: 64 MB at most, where splitting the heads alone does not pass that.
  const long long row_tiles = (n_rows + kRows - 1) / kRows, want = 1024;
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
