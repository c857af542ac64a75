// Attention of query rows over the 8-bit paged cache: one pass over the keys
// with the running maximum and sum of the softmax, products on the matrix
// cores with fp32 sums.
//
// The heads of a group share their keys, so a group's rows (t, g), r = t G + g,
// are one product.  Logits are formed turned, S^T = K Q^T (rows tokens, columns
// query rows): the lane of a column then holds the weights of its own query
// row, in the layout in which the second product, O^T = V^T P^T, takes them as
// its operand, so they never leave its registers.  That needs the k positions
// of the second product (tokens) to be dealt to the lanes as the first one's
// output rows are; which token sits in which row of K is free, so the rows are
// dealt such that a lane holds 16 tokens in a row: 16 bytes of a value
// channel, which the cache stores token last for this.
//
// e4m3 numbers are bf16 numbers, so keys and values enter the products
// exactly.  bf16 queries do too; their calls' weights are rounded to bf16 for
// the second product (by at most 2^-8 of each, as the output is; the sum that
// divides them is of the unrounded ones, which the log-sum-exp needs).  That adds
// a tenth to a quarter to the outputs' error, 1.65e-3 relative from their own
// rounding alone: 1.82e-3 for single tokens, 1.98e-3 for questions, 2.05e-3 for
// prompts.  (Weights in two bf16 parts would take 33 % more of a prompt's time
// and up to 7 % of a token's.)  fp32
// queries and weights are split into three bf16 parts, 24 bits.  (The 8-bit
// matrix instructions would take keys unconverted, and a bf16 query as two
// e4m3 parts, but their sums came out 2^-19 off, too far for a log-sum-exp.)
#include <type_traits>

#include "cache.hpp"
#include "cut.hpp"

namespace trevs {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <class E>
constexpr int kParts = E::kBytes == 2 ? 1 : 3;

// Eight e4m3 numbers, times a power of two, as bf16.
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight fp32 values as bf16 parts that sum to them (one part: rounded).
template <int N>
__device__ __forceinline__ void split_parts(float (&x)[8], bf16x8 (&out)[N]) {
#pragma unroll
  for (int p = 0; p < N; ++p)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      out[p][j] = (__bf16)x[j];
      x[j] -= (float)out[p][j];
    }
}

__device__ __forceinline__ void load_row8(const void* q, size_t i, float (&x)[8], BF16) {
  const u32x4 w = ldg16(reinterpret_cast<const uint16_t*>(q) + i);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = bf16_lo(w[j]);
    x[2 * j + 1] = bf16_hi(w[j]);
  }
}
__device__ __forceinline__ void load_row8(const void* q, size_t i, float (&x)[8], F32) {
  const float* f = reinterpret_cast<const float*>(q) + i;
  const u32x4 a = ldg16(f), b = ldg16(f + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = __uint_as_float(a[j]);
    x[4 + j] = __uint_as_float(b[j]);
  }
}

// Bytes [0, n) of a 16-byte vector kept, the others zeroed.
__device__ __forceinline__ u32x4 keep_bytes(u32x4 v, int n) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int k = n - 4 * w;
    v[w] = k >= 4 ? v[w] : k <= 0 ? 0u : v[w] & ((1u << (8 * k)) - 1u);
  }
  return v;
}

// NaN among e4m3 values.  A row's weight for a token that it does not see is 0, which would keep the token's
// values away from it, except that 0 NaN is NaN.  So in the steps whose tokens some rows of a tile see and others
// do not, NaN values are multiplied as zeros; if there were any, a second pass over these steps finds the rows
// that see them, by products of ones for NaN with ones for the tokens seen.  (Both in the main loop took its
// registers: prompts of 4 x 4259 rows 590 -> 768 us, this way 622 -> 620.)
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {  // 1 in each byte that is NaN
  return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
}
// Not 0 if there is a NaN in v.
__device__ __forceinline__ uint32_t any_nan(u32x4 v) {
  uint32_t any = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) any |= (v[w] & 0x7f7f7f7fu) + 0x01010101u;
  return any & 0x80808080u;
}
// NaN in v set to 0; whether there was one.
__device__ __forceinline__ bool drop_nan(u32x4& v) {
  uint32_t any = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t n = nan_bytes(v[w]);
    v[w] &= ~(n * 0xffu);
    any |= n;
  }
  return any != 0;
}
// v as bf16, 1 where it is NaN and 0 where it is a number.
__device__ __forceinline__ void nan_ones(u32x4 v, bf16x8 (&ones)[2]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) v[w] = nan_bytes(v[w]) * 0x38u;  // (0x38: 1 in e4m3)
  ones[0] = widen(v[0], v[1], 1.f);
  ones[1] = widen(v[2], v[3], 1.f);
}
// A lane's 16 weights as 1 for the first n, which its row sees, and 0 for the others.
__device__ __forceinline__ void seen_ones(int n, bf16x8 (&ones)[2]) {
#pragma unroll
  for (int j = 0; j < 16; ++j) ones[j >> 3][j & 7] = (__bf16)(j < n ? 1.f : 0.f);
}

template <class E>
__device__ __forceinline__ void store4(void* out, size_t i, const float (&x)[4], E) {
  if constexpr (E::kBytes == 2) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 y;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = (__bf16)x[j];
    *reinterpret_cast<bf16x4*>(reinterpret_cast<uint16_t*>(out) + i) = y;
  } else {
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(out) + i) = make_float4(x[0], x[1], x[2], x[3]);
  }
}

// Weights may pass the running maximum by 2^kSlack before the sums are rescaled
// to a new one: fp32 sums and bf16 weights do not mind, and rescaling becomes rare.
constexpr float kSlack = 8.f;

constexpr int kStep = 64;  // tokens of a step
constexpr int kWaves = 4;
constexpr int kTileRows = 128;
// Steps that a workgroup takes side by side: the waves of a staged tile share theirs.
__host__ __device__ constexpr int side_steps(int rows) { return rows == kTileRows ? 1 : kWaves; }

// A tile is R query rows (t, g) of one group; its steps are the 64-token blocks
// that its last row sees.  Calls of few tiles, or of uneven ones, cut the
// steps of all of them, one after the other (sequences, row tiles, groups),
// into equal pieces, a workgroup to a piece: a piece that covers a
// tile finishes it, the others leave their sums to join_kernel.  (8 questions
// over 16.5 k tokens took 225 us with them in this order, 238 with groups before
// row tiles, and the same with neighbouring pieces on one XCD.)
struct Tile {
  int b, hk, rt;
};
struct Sequence {
  int rows, slot, L;  // query rows, slot, tokens
};
__device__ __forceinline__ Sequence sequence(const AttnArgs& a, int b) {
  Sequence s;
  s.rows = a.q_len ? min(max(a.q_len[b], 0), a.T_max) : a.T_max;
  s.slot = slot_of(a.slots, b, a.c.n_slots);
  s.L = slot_len(a.c.len, s.slot, a.kv_max);
  return s;
}
// Keys that the last row of a tile sees (0 for a tile without rows).
template <int R>
__device__ __forceinline__ int tile_keys(const AttnArgs& a, const Sequence& s, int rt) {
  const int n_rows = s.rows * a.G, r0 = rt * R;
  if (r0 >= n_rows) return 0;
  const int t_last = min(r0 + R - 1, n_rows - 1) / a.G;
  return max(a.causal ? min(s.L - s.rows + t_last + 1, s.L) : s.L, 0);
}
__device__ __forceinline__ int steps_of(int keys) { return (keys + kStep - 1) / kStep; }

// The steps of all sequences in one row, held by a wave: lane i of `ends` the
// end of sequence i's among the first 64 sequences (the rest is recomputed:
// its loads hit the cache).  The host sees to it that the sum fits 31 bits.
template <int R>
struct Schedule {
  int ends, total;
  static __device__ __forceinline__ int scan(const AttnArgs& a, int b0) {
    const int lane = threadIdx.x & 63, b = b0 + lane;
    int n = 0;
    if (b < a.B) {
      const Sequence s = sequence(a, b);
      for (int rt = 0; rt * R < s.rows * a.G; ++rt) n += steps_of(tile_keys<R>(a, s, rt));
    }
    return wave_incl_scan(n * a.c.H_kv, lane);
  }
  __device__ __forceinline__ void init(const AttnArgs& a) {
    ends = scan(a, 0);
    total = __builtin_amdgcn_readlane(ends, 63);
    for (int b0 = 64; b0 < a.B; b0 += 64) total += __builtin_amdgcn_readlane(scan(a, b0), 63);
  }
};

// A workgroup's way through its work: in a cut call the pieces of tiles that its steps cover, else one tile.
struct Piece {
  Tile t;
  Sequence seq;
  int u0, u1;   // steps of the tile
  int part;     // -1: the whole tile; else where its sums go
};
template <int R>
struct Walk {
  Schedule<R> s;
  Cut cut;
  int at, end;         // steps still to do
  Tile t;              // the tile that `at` lies in,
  Sequence seq;        // its sequence,
  int first, n;        // its first step and its steps
  __device__ __forceinline__ explicit Walk(const AttnArgs& a) : cut(0, 0), at(0), end(1) {
    if (!a.part) return;
    s.init(a);
    cut = Cut(s.total, gridDim.x);
    end = 0;
    if ((int)blockIdx.x >= cut.n) return;
    at = cut.start(blockIdx.x);
    end = cut.start(blockIdx.x + 1);
    locate(a);
  }
  __device__ __forceinline__ void locate(const AttnArgs& a) {
    int before = 0, e = s.ends, b0 = 0;
    while (before + __builtin_amdgcn_readlane(e, 63) <= at) {
      before += __builtin_amdgcn_readlane(e, 63);
      b0 += 64;
      e = s.scan(a, b0);
    }
    const int i = __builtin_ctzll(__ballot(before + e > at));
    t.b = b0 + i;
    first = before + (i ? __builtin_amdgcn_readlane(e, i - 1) : 0);
    seq = sequence(a, t.b);
    for (t.rt = 0;; ++t.rt) {
      n = steps_of(tile_keys<R>(a, seq, t.rt));
      if (at < first + n * a.c.H_kv) break;
      first += n * a.c.H_kv;
    }
    t.hk = (at - first) / n;
    first += t.hk * n;
  }
  // To the next tile that has steps (there is one: at < end).
  __device__ __forceinline__ void advance(const AttnArgs& a) {
    first += n;
    if (++t.hk < a.c.H_kv) return;
    t.hk = 0;
    do {
      if (++t.rt * R >= seq.rows * a.G) {
        t.rt = 0;
        seq = sequence(a, ++t.b);
      }
      n = steps_of(tile_keys<R>(a, seq, t.rt));
    } while (n == 0);
  }
  __device__ __forceinline__ bool next(const AttnArgs& a, Piece& p) {
    if (at >= end) return false;
    p.part = -1;
    p.u0 = 0;
    if (!a.part) {
      // not cut: groups (b, hk) next to each other, so that a group's tiles meet on the XCDs that share
      // its index modulo 8; the tiles with the most keys first
      const int groups = a.B * a.c.H_kv, group = blockIdx.x % groups;
      p.t.rt = a.row_tiles - 1 - blockIdx.x / groups;
      p.t.b = group / a.c.H_kv;
      p.t.hk = group - p.t.b * a.c.H_kv;
      p.seq = sequence(a, p.t.b);
      p.u1 = steps_of(tile_keys<R>(a, p.seq, p.t.rt));
      at = end;
      return true;
    }
    p.t = t;
    p.seq = seq;
    p.u0 = at - first;
    p.u1 = min(n, end - first);
    // a piece that begins its tile is the workgroup's last, one that does not its first
    if (p.u0 != 0 || p.u1 != n) p.part = 2 * blockIdx.x + (p.u0 == 0);
    if (p.u0 == 0 && threadIdx.x == 0)
      a.tile_pieces[(t.b * a.c.H_kv + t.hk) * a.row_tiles + t.rt] =
          make_int2(blockIdx.x, p.part < 0 ? (int)blockIdx.x : cut.owner(first + n - 1));
    at = first + p.u1;
    if (at < end) advance(a);
    return true;
  }
};

__device__ __forceinline__ size_t out_row(const AttnArgs& a, const Tile& t, int r) {
  const int q = r / a.G, h = t.hk * a.G + r - q * a.G;
  return ((size_t)t.b * a.T_max + q) * a.H_q + h;
}
__device__ __forceinline__ void store_lse(const AttnArgs& a, const Tile& t, int r, float m, float l) {
  const int q = r / a.G, h = t.hk * a.G + r - q * a.G;
  // (l is 0 for a row that sees no key, and NaN, as its outputs, for one that sees a NaN)
  a.lse[((size_t)t.b * a.H_q + h) * a.T_max + q] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// NaN for channel c of the staged tile's row r (counted in the group), where its output or its piece's sum is.
template <int D>
__device__ __forceinline__ void store_nan(const AttnArgs& a, const Piece& pc, int r, int c) {
  if (pc.part >= 0)
    a.part[((size_t)pc.part * kTileRows + (r - pc.t.rt * kTileRows)) * D + c] = NAN;
  else
    reinterpret_cast<__bf16*>(a.out)[out_row(a, pc.t, r) * D + c] = (__bf16)NAN;
}

// A workgroup takes 16 NQ rows of one group; its waves take every kWaves-th
// step.  Nothing is staged: a lane loads its own 16 bytes of key channels and
// of value tokens.  Bound by the cache's bytes for single tokens.
template <class E, int D, int NQ>
struct RowsShared {
  // the waves' sums side by side where they fit 34 KB, else added up by one wave after the other
  static constexpr int kSides = NQ * D <= 128 ? kWaves : 1;
  float o[kSides][16 * NQ][D + 4];
  float m[kWaves][16 * NQ], l[kWaves][16 * NQ];
};

template <bool ONCE>
__device__ __forceinline__ u32x4 load16(const void* p) {
  if constexpr (ONCE) return ldg16_stream(p);
  return ldg16(p);
}

// ONE: calls of one token a sequence, whose rows all see the same keys.
template <class E, int D, int NQ, bool ONE>
__device__ __forceinline__ void rows_piece(const AttnArgs& a, const Piece& pc, RowsShared<E, D, NQ>& sh) {
  constexpr int NP = kParts<E>;
  constexpr int R = 16 * NQ;
  // calls of at most 16 rows a group read the cache once (64 sequences of 1.2 k to 16.5 k tokens: 107 us
  // streamed, 120 not); of more, row tiles share it
  constexpr bool kOnce = NQ == 1 && !(D == 256 && E::kBytes == 4);
  auto& s_o = sh.o;
  auto& s_m = sh.m;
  auto& s_l = sh.l;
  const int lane = threadIdx.x & 63, n16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = pc.t.b, hk = pc.t.hk, r0 = pc.t.rt * R, u0 = pc.u0, u1 = pc.u1;
  const Sequence& seq = pc.seq;
  const int rows = seq.rows, slot = seq.slot, L = seq.L, n_rows = rows * a.G;
  const int n_keys = tile_keys<R>(a, seq, pc.t.rt);

  // A lane looks up the page of its 16 tokens (weights, values) a unit ahead; its key rows, of tile t
  // row 4 y + i = token 16 y + 4 t + i, lie in the page of lane group y.  Their places in a page are the
  // same in every unit (64 tokens are whole pages).
  const int shift = a.page_shift, page_mask = (1 << shift) - 1;
  const size_t page_stride = ((size_t)D << shift) * a.c.H_kv;
  const int key_row = (16 * (n16 >> 2) & page_mask) + (n16 & 3);
  const uint8_t* k_base = a.c.k + ((size_t)hk * D << shift) + key_row * D + 16 * g4;
  const uint8_t* v_base = a.c.v + ((size_t)hk * D << shift) + ((size_t)n16 << shift) + (16 * g4 & page_mask);
  const int32_t* table = a.c.table + (size_t)max(slot, 0) * a.c.max_pages;
  auto look_up = [&](int u) { return table[min((u * kStep + 16 * g4) >> shift, a.c.max_pages - 1)]; };
  int next = slot >= 0 ? look_up(u0 + wave) : -1;  // (not held up by the length)
  int lim[NQ];  // keys that this lane's query row sees
  bf16x8 q[NQ][D / 32][NP];
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int r = r0 + 16 * i + n16, t = r / a.G, g = r - t * a.G;
    // (a row past the last is not stored: it need not be masked)
    lim[i] = r < n_rows ? (a.causal ? min(L - rows + t + 1, L) : L) : n_keys;
    const size_t at = ((size_t)b * a.T_max + t) * a.q_ld + (size_t)(hk * a.G + g) * D;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      // lane group g4 holds channels 64 (c/2) + 16 g4 + 8 (c%2) .. +7, as the keys' 16-byte loads give them
      float x[8] = {};
      if (r < n_rows) load_row8(a.q, at + c / 2 * 64 + 16 * g4 + 8 * (c & 1), x, E());
      split_parts<NP>(x, q[i][c]);
    }
  }
  int lim_all = lim[0];
#pragma unroll
  for (int i = 1; i < NQ; ++i) lim_all = min(lim_all, lim[i]);

  f32x4 o[NQ][D / 16];
  float m[NQ], l[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // some rows see tokens of a step that others do not
  auto mixed = [&](int u) { return __any(lim_all < min(u * kStep + kStep, n_keys)); };
  bool nan = false;  // this lane left out NaN values
  for (int u = u0 + wave; u < u1; u += kWaves) {
    const int tok = u * kStep + 16 * g4;
    const bool there = next >= 0 && next < a.c.n_pages && tok < n_keys;
    const int page = there ? next : 0;
    const uint8_t* kp = k_base + (size_t)__shfl(page, 16 * (n16 >> 2), 64) * page_stride;
    const uint8_t* vp = v_base + (size_t)page * page_stride;
    u32x4 kw[4][D / 64], vw[D / 16];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) kw[t][c] = load16<kOnce>(kp + t * 4 * D + c * 64);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) vw[c] = load16<kOnce>(vp + ((size_t)(16 * c) << shift));
    const size_t block = (size_t)page * a.c.H_kv + hk;
    float ks = a.c.k_scale[block], vs = a.c.v_scale[block];
    next = look_up(u + kWaves);
    const bool whole = __all(there && u * kStep + kStep <= lim_all);
    f32x4 s[NQ][4];
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int t = 0; t < 4; ++t) s[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const bf16x8 k0 = widen(kw[t][c][0], kw[t][c][1], 1.f), k1 = widen(kw[t][c][2], kw[t][c][3], 1.f);
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
          for (int p = NP - 1; p >= 0; --p) {
            s[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[i][2 * c][p], s[i][t], 0, 0, 0);
            s[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[i][2 * c + 1][p], s[i][t], 0, 0, 0);
          }
      }
    if (!whole) {
      const int n_v =  // tokens of this lane whose values count
           there ? min(max(L - tok, 0), 16) : 0;
      if (!there) ks = vs = 1.f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) vw[c] = keep_bytes(vw[c], n_v);
      if (!ONE && mixed(u)) {
#pragma unroll
        for (int c = 0; c < D / 16; ++c) nan |= drop_nan(vw[c]);
      }
    }
    bf16x8 pw[NQ][2][NP];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      float x[16], top = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = s[i][e >> 2][e & 3] * (ks * a.scale_log2e);
      if (!whole) {
        const int n = there ? lim[i] - tok : 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = e < n ? x[e] : -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, x[e]);
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      if (__any(top > m[i] + kSlack)) {
        const float now = fmaxf(top, m[i]), old = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - now);
        m[i] = now;
        l[i] *= old;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) o[i][c] *= old;
      }
      const float base = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        x[e] = __builtin_amdgcn_exp2f(x[e] - base);
        l[i] += x[e];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[8 * h + j];
        split_parts<NP>(y, pw[i][h]);
      }
    }
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      const bf16x8 v0 = widen(vw[c][0], vw[c][1], vs), v1 = widen(vw[c][2], vw[c][3], vs);
#pragma unroll
      for (int i = 0; i < NQ; ++i)
#pragma unroll
        for (int p = NP - 1; p >= 0; --p) {
          o[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pw[i][0][p], o[i][c], 0, 0, 0);
          o[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pw[i][1][p], o[i][c], 0, 0, 0);
        }
    }
  }
  if (!ONE && __any(nan)) {
    for (int u = u0 + wave; u < u1; u += kWaves) {
      if (!mixed(u)) continue;
      const int tok = u * kStep + 16 * g4, p = look_up(u);
      const bool there = p >= 0 && p < a.c.n_pages && tok < n_keys;
      const uint8_t* vp = v_base + (size_t)(there ? p : 0) * page_stride;
      bf16x8 seen[NQ][2];
#pragma unroll
      for (int i = 0; i < NQ; ++i) seen_ones(there ? lim[i] - tok : 0, seen[i]);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        bf16x8 ones[2];
        nan_ones(keep_bytes(ldg16(vp + ((size_t)(16 * c) << shift)), there ? min(max(L - tok, 0), 16) : 0), ones);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          f32x4 hit = f32x4{0.f, 0.f, 0.f, 0.f};
          hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones[0], seen[i][0], hit, 0, 0, 0);
          hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones[1], seen[i][1], hit, 0, 0, 0);
#pragma unroll
          for (int j = 0; j < 4; ++j) o[i][c][j] = hit[j] > 0.f ? NAN : o[i][c][j];
        }
      }
    }
  }
  // the waves' parts, in their order
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    l[i] += __shfl_xor(l[i], 16, 64);
    l[i] += __shfl_xor(l[i], 32, 64);
    if (g4 == 0) {
      s_m[wave][16 * i + n16] = m[i];
      s_l[wave][16 * i + n16] = l[i];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_m[w][16 * i + n16]);
    const float f = m[i] == -INFINITY ? 0.f : exp2f(m[i] - top);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[i][c] *= f;
  }
  constexpr int kSides = RowsShared<E, D, NQ>::kSides;
  for (int w = 0; w < kWaves; w += kSides) {
    if (kSides > 1 || wave == w) {
#pragma unroll
      for (int i = 0; i < NQ; ++i)
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          f32x4* at = reinterpret_cast<f32x4*>(&s_o[kSides > 1 ? wave : 0][16 * i + n16][16 * c + 4 * g4]);
          *at = w == 0 ? o[i][c] : *at + o[i][c];
        }
    }
    __syncthreads();
  }
  for (int e = threadIdx.x; e < R * (D / 4); e += kWaves * 64) {
    const int r = e / (D / 4), c = e % (D / 4) * 4;
    if (r0 + r >= n_rows) break;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w)  // (a NaN logit leaves the maximum at -inf and makes the sum NaN)
      sum += s_l[w][r] * (s_m[w][r] == -INFINITY ? 0.f : exp2f(s_m[w][r] - top));
    f32x4 y = *reinterpret_cast<const f32x4*>(&s_o[0][r][c]);
#pragma unroll
    for (int w = 1; w < kSides; ++w) y += *reinterpret_cast<const f32x4*>(&s_o[w][r][c]);
    float x[4] = {y[0], y[1], y[2], y[3]};
    if (pc.part >= 0) {
      const size_t part = (size_t)pc.part * R + r;
      *reinterpret_cast<float4*>(a.part + part * D + c) = make_float4(x[0], x[1], x[2], x[3]);
      if (c == 0) a.part_ml[part] = make_float2(top, sum);
      continue;
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] *= inv;
    store4(a.out, out_row(a, pc.t, r0 + r) * D + c, x, E());
    if (a.lse && c == 0) store_lse(a, pc.t, r0 + r, top, sum);
  }
}

template <class E, int D, int NQ, bool ONE>
__global__ __launch_bounds__(kWaves * 64, NQ == 1 && D <= 128 && E::kBytes == 2 ? 3 : 1) void rows_kernel(AttnArgs a) {
  __shared__ RowsShared<E, D, NQ> sh;
  Walk<16 * NQ> walk(a);
  Piece p;
  while (walk.next(a, p)) {
    rows_piece<E, D, NQ, ONE>(a, p, sh);
    __syncthreads();  // the sums in LDS are read before the next piece's are written
  }
}

// ---------------------------------------------------------------- many rows
// A workgroup takes 128 rows of one group, its waves 32 each, and steps through
// the keys 64 tokens at a time, staged in LDS as they are stored (8 bits) one
// step ahead.  Prompts of 4 x 4259 rows with 28 heads of 128 take 588 to 635 us
// (820 to 885 TFLOP/s) by the machine, a product of 8192^3 in bf16 reaches 1212
// to 1404.  Bound by the vector instructions beside the products: a wave issues
// 368 a step (145 of them conversions, of keys and values that each of the four
// waves widens for its own rows) to 32 products; counted over a pass, vector
// units are busy 65 % of the cycles and matrix cores 38 %, half of that at the
// same time.  Logits formed half a step ahead of the exponentials, operands
// staged as bf16 (a third fewer vector instructions, twice the LDS reads) and
// 256 rows a workgroup each took the same within 3 %.

// Permutation of a staged row's 16-byte columns, by the row: 16 lanes next to
// each other read one column of 16 rows and must meet 16 different ones modulo
// 256 bytes, the width of the banks.  A 128-byte row (keys of 128 channels) leaves
// two rows to a width, a 64-byte one four; of keys the 16 rows are tokens 0-7 and
// 16-23, as their rows are dealt, of values channels 0-15.  (Counted bank
// conflicts of a prompt of 4259 rows: 3.2e7 cycles with a permutation for 8
// lanes and 128 bytes, 0 with this one.)
template <int D>
__device__ __forceinline__ int key_swizzle(int row) {
  return D == 64 ? ((row >> 2) & 1) | ((row >> 3) & 2) : ((row >> 1) & 3) | ((row >> 2) & 4);
}
__device__ __forceinline__ int value_swizzle(int row) { return (row >> 2) & 3; }

template <int D>
struct TileShared {
  static constexpr int kKeyVecs = kStep * D / 16;  // 16-byte vectors of a side
  u32x4 k[2][kKeyVecs], v[2][kKeyVecs];
  float ks[2][4], vs[2][4];  // scales of each 16 tokens; a negative key scale: absent
  int nan[kWaves];           // whether a wave left out NaN values
};

template <int D>
__device__ __forceinline__ void tile_piece(const AttnArgs& a, const Piece& pc, TileShared<D>& sh) {
  constexpr int kVecs = TileShared<D>::kKeyVecs / 256;  // of a thread
  auto& s_k = sh.k;
  auto& s_v = sh.v;
  auto& s_ks = sh.ks;
  auto& s_vs = sh.vs;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = pc.t.b, hk = pc.t.hk, r0 = pc.t.rt * kTileRows, u0 = pc.u0, u1 = pc.u1;
  const Sequence& seq = pc.seq;
  const int rows = seq.rows, slot = seq.slot, L = seq.L, n_rows = rows * a.G;
  const int n_keys = tile_keys<kTileRows>(a, seq, pc.t.rt);

  // this lane's query row: half h holds channels 32 (c/2) + 16 h + 8 (c%2) .. +7, as the keys' 16-byte reads give them
  const int r = r0 + 32 * wave + col, t = r / a.G, g = r - t * a.G;
  const bool live = r < n_rows;
  const int lim = live ? (a.causal ? min(L - rows + t + 1, L) : L) : n_keys;
  bf16x8 q[D / 16];
  {
    const size_t at = ((size_t)b * a.T_max + t) * a.q_ld + (size_t)(hk * a.G + g) * D + 16 * half;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
      q[c] = __builtin_bit_cast(
          bf16x8, live ? ldg16(reinterpret_cast<const uint16_t*>(a.q) + at + c / 2 * 32 + 8 * (c & 1)) : zero4());
  }
  // keys that every row of the wave sees (a row past the last is not stored: it need not be masked)
  const int w_first = r0 + 32 * wave;
  const int lim_all = a.causal ? min(L - rows + w_first / a.G + 1, L) : L;
  const bool busy = w_first < n_rows;  // a wave without rows only stages

  f32x16 o[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
  float m = -INFINITY, l = 0.f;

  // Vectors of a step: key vector e holds 16 channels of token e / (D/16), value vector e 16 tokens of
  // channel e / 4.  Their places in a page are the same in every step (64 tokens are whole pages); a
  // lane looks up the page of its values' 16 tokens a step ahead of the loads, and the key
  // vectors of a wave lie in one page each, whose number is one of those.  In LDS a row's 16-byte
  // columns are permuted by the row so that the lanes of a read, one row each, meet all banks.
  const int shift = a.page_shift, page_mask = (1 << shift) - 1;
  const size_t page_stride = ((size_t)D << shift) * a.c.H_kv;
  const uint8_t* k_base = a.c.k + ((size_t)hk * D << shift);
  const uint8_t* v_base = a.c.v + ((size_t)hk * D << shift) + ((size_t)(tid >> 2) << shift) + ((tid & 3) * 16 & page_mask);
  const int32_t* table = a.c.table + (size_t)max(slot, 0) * a.c.max_pages;
  const int last_page = max(n_keys - 1, 0) >> shift;
  u32x4 gk[kVecs], gv[kVecs];
  float g_ks, g_vs;
  int g_n;  // tokens of this lane's value vectors that count
  int page = -1;
  auto look_up = [&](int u) { page = table[min((u * kStep + (tid & 3) * 16) >> shift, last_page)]; };
  auto load = [&](int u) {  // (after look_up(u))
    const bool there = page >= 0 && page < a.c.n_pages;
    const int at = there ? page : 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int e = tid + 256 * i, first = (64 * wave + 256 * i) / (D / 16);  // tokens of the vector, of the wave's first
      const int p = __builtin_amdgcn_readlane(at, first >> 4);
      gk[i] = ldg16(k_base + (size_t)p * page_stride + ((e / (D / 16)) & page_mask) * D + e % (D / 16) * 16);
    }
    const uint8_t* v = v_base + (size_t)at * page_stride;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) gv[i] = ldg16(v + ((size_t)(64 * i) << shift));
    const size_t block = (size_t)at * a.c.H_kv + hk;
    g_ks = a.c.k_scale[block];
    g_vs = a.c.v_scale[block];
    g_n = there ? L - (u * kStep + (tid & 3) * 16) : 0;
    if (!there) g_ks = -1.f, g_vs = 1.f;
  };
  // from this step on some rows see tokens that others do not
  const int u_mixed = a.causal ? max(min(L - rows + r0 / a.G + 1, L), 0) / kStep : u1;
  bool nan = false;  // this wave left out NaN values
  auto store = [&](int buf, bool drop) {
    const bool mask = __any(g_n < 16);
    if (drop) {
      uint32_t found = 0;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) found |= any_nan(gv[i]);
      if (__any(found != 0)) {
        nan = true;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) drop_nan(gv[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int e = tid + 256 * i;
      const int kr = e / (D / 16), kc = e % (D / 16);
      s_k[buf][kr * (D / 16) + (kc ^ key_swizzle<D>(kr))] = gk[i];
      if (mask) gv[i] = keep_bytes(gv[i], g_n);
      const int vr = e >> 2, vc = e & 3;
      s_v[buf][vr * 4 + (vc ^ value_swizzle(vr))] = gv[i];
    }
    if (tid < 4) {
      s_ks[buf][tid] = g_ks;
      s_vs[buf][tid] = g_vs;
    }
  };
  if (u0 < u1) {
    look_up(u0);
    load(u0);
    look_up(u0 + 1);
    store(0, u0 >= u_mixed);
  }
  wait_vmem<0>();  // (the queries too: the loop then waits for its own loads only)
  __syncthreads();
  for (int u = u0; u < u1; ++u) {
    const int buf = (u - u0) & 1;
    // (past the last step: its own pages again, not used)
    load(u + 1);
    look_up(u + 2);
    if (busy) {
      f32x16 s[2];
      float ks[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        ks[y] = s_ks[buf][2 * y + half];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[y][i] = 0.f;
        // row 8j + 4h + i of the product is token 16 h + 4 j + i
        const int kr = 32 * y + 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          const u32x4 w = s_k[buf][kr * (D / 16) + ((2 * c + half) ^ key_swizzle<D>(kr))];
          s[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(w[0], w[1], 1.f), q[2 * c], s[y], 0, 0, 0);
          s[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(w[2], w[3], 1.f), q[2 * c + 1], s[y], 0, 0, 0);
        }
      }
      const bool whole = (u + 1) * kStep <= lim_all && __all(ks[0] >= 0.f && ks[1] >= 0.f);
      float f[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        f[y] = fmaxf(fabsf(ks[y]) * a.scale_log2e, 0x1p-126f);  // (never 0: the masked -inf stay what they are)
        if (!whole) {
          const int n = ks[y] >= 0.f ? lim - (u * kStep + 32 * y + 16 * half) : 0;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[y][i] = i < n ? s[y][i] : -INFINITY;
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float x = s[y][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) x = fmaxf(x, s[y][i]);
        top = fmaxf(top, x * f[y]);
      }
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      if (__any(top > m + kSlack)) {
        const float now = fmaxf(top, m), old = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
        m = now;
        l *= old;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[c][i] *= old;
      }
      const float base = m == -INFINITY ? 0.f : m;
      bf16x8 p[4];
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = __builtin_amdgcn_exp2f(fmaf(s[y][i], f[y], -base));
          l += x;
          p[2 * y + (i >> 3)][i & 7] = (__bf16)x;
        }
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const float vs = s_vs[buf][2 * y + half];
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          const int vr = 32 * c + col;
          const u32x4 w = s_v[buf][vr * 4 + ((2 * y + half) ^ value_swizzle(vr))];
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(w[0], w[1], vs), p[2 * y], o[c], 0, 0, 0);
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(w[2], w[3], vs), p[2 * y + 1], o[c], 0, 0, 0);
        }
      }
    }
    if (u + 1 == u1) sh.nan[wave] = nan;
    store(buf ^ 1, u + 1 >= u_mixed);
    __syncthreads();
  }
  l += __shfl_xor(l, 32, 64);
  if (live && pc.part >= 0) {
    const size_t part = (size_t)pc.part * kTileRows + 32 * wave + col;
    if (half == 0) a.part_ml[part] = make_float2(m, l);
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(a.part + part * D + 32 * c + 8 * j + 4 * half) =
            make_float4(o[c][4 * j], o[c][4 * j + 1], o[c][4 * j + 2], o[c][4 * j + 3]);
  } else if (live) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const size_t out = out_row(a, pc.t, r) * D;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x[4] = {o[c][4 * j] * inv, o[c][4 * j + 1] * inv, o[c][4 * j + 2] * inv, o[c][4 * j + 3] * inv};
        store4(a.out, out + 32 * c + 8 * j + 4 * half, x, BF16());
      }
    if (a.lse && half == 0) store_lse(a, pc.t, r, m, l);
  }
  if (u0 >= u1 || !(sh.nan[0] | sh.nan[1] | sh.nan[2] | sh.nan[3])) return;
  for (int tok = max(u0, u_mixed) * kStep + 16 * half; tok < u1 * kStep; tok += 32) {
    const int p = tok < n_keys ? table[tok >> shift] : -1;
    const bool there = p >= 0 && p < a.c.n_pages;
    const uint8_t* v = a.c.v + ((size_t)(there ? p : 0) * a.c.H_kv + hk) * ((size_t)D << shift) + (tok & page_mask);
    bf16x8 seen[2];
    seen_ones(there ? lim - tok : 0, seen);
    for (int c = 0; c < D / 32; ++c) {
      bf16x8 ones[2];
      nan_ones(keep_bytes(ldg16(v + ((size_t)(32 * c + col) << shift)), there ? L - tok : 0), ones);
      f32x16 hit;
#pragma unroll
      for (int i = 0; i < 16; ++i) hit[i] = 0.f;
      hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones[0], seen[0], hit, 0, 0, 0);
      hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones[1], seen[1], hit, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (hit[i] > 0.f && live) store_nan<D>(a, pc, r, 32 * c + 8 * (i >> 2) + 4 * half + (i & 3));
    }
  }
}

template <int D>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void tile_kernel(AttnArgs a) {
  __shared__ TileShared<D> sh;
  Walk<kTileRows> walk(a);
  Piece p;
  // (a piece ends with its last reads of the tile behind a barrier, those of `nan` are behind the next piece's first)
  while (walk.next(a, p)) tile_piece<D>(a, p, sh);
}

// The sums of the pieces of each cut tile joined, in the order of its steps;
// zeros for rows that see no key.  D / 4 threads hold a row, four channels
// each; tiles of many pieces (MANY: 8 or more on average) give a row to a whole
// workgroup, each D / 4 threads to every kJoinThreads / (D / 4)-th piece (one
// sequence of 16 k tokens, 64 pieces a tile: 16.7 us without, 12.9 with).
constexpr int kJoinThreads = 256;
template <class E, int D, int R, bool MANY>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(AttnArgs a) {
  constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes, kRows = MANY ? 1 : kGroups;
  __shared__ float4 s_x[MANY ? kGroups : 1][kLanes];
  __shared__ float s_l[MANY ? kGroups : 1];
  const int group = threadIdx.x / kLanes, c = threadIdx.x % kLanes * 4;
  Tile t;
  int id = blockIdx.x;
  const int row = id % (R / kRows) * kRows + (MANY ? 0 : group);
  id /= R / kRows;
  t.rt = id % a.row_tiles;
  id /= a.row_tiles;
  t.b = id / a.c.H_kv;
  t.hk = id - t.b * a.c.H_kv;
  const Sequence seq = sequence(a, t.b);
  const int r = t.rt * R + row;
  if (r >= seq.rows * a.G) return;  // (one row or whole groups of lanes: no barrier is missed)
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  float m = -INFINITY, l = 0.f;
  if (tile_keys<R>(a, seq, t.rt) > 0) {
    const int2 pieces = a.tile_pieces[(t.b * a.c.H_kv + t.hk) * a.row_tiles + t.rt];
    const int w0 = pieces.x, n = pieces.y - pieces.x + 1;
    if (n == 1) return;  // (one piece has finished it)
    // the first piece begins the tile, the others do not
    auto at = [&](int i) { return (size_t)(2 * (w0 + i) + (i == 0)) * R + row; };
    for (int i = threadIdx.x % kLanes; i < n; i += kLanes) m = fmaxf(m, a.part_ml[at(i)].x);
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
#pragma unroll 4
    for (int i = MANY ? group : 0; i < n; i += MANY ? kGroups : 1) {
      const float2 ml = a.part_ml[at(i)];
      const float4 y = *reinterpret_cast<const float4*>(a.part + at(i) * D + c);
      const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
      l = fmaf(ml.y, f, l);
      x = make_float4(fmaf(y.x, f, x.x), fmaf(y.y, f, x.y), fmaf(y.z, f, x.z), fmaf(y.w, f, x.w));
    }
    if constexpr (MANY) {
      s_x[group][c / 4] = x;
      if (c == 0) s_l[group] = l;
      __syncthreads();
      if (group) return;
      for (int g = 1; g < kGroups; ++g) {
        const float4 y = s_x[g][c / 4];
        x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
        l += s_l[g];
      }
    }
  }
  if (MANY && group) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const float out[4] = {x.x * inv, x.y * inv, x.z * inv, x.w * inv};
  store4(a.out, out_row(a, t, r) * D + c, out, E());
  if (a.lse && c == 0) store_lse(a, t, r, m, l);
}

template <class E, int D>
hipError_t launch(AttnArgs a, const AttnPlan& p, hipStream_t s) {
  a.row_tiles = p.row_tiles;
  if (p.pieces == 0) a.part = nullptr;
  const long long tiles = (long long)a.B * a.c.H_kv * p.row_tiles;
  const bool many = p.pieces >= 8 * tiles;
  auto go = [&](auto kernel, auto join, auto join_many) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(p.pieces ? p.pieces : tiles)), dim3(256), 0, s, a);
    if (!p.pieces) return;
    const long long rows = tiles * p.rows;
    if (many)
      hipLaunchKernelGGL(join_many, dim3((unsigned)rows), dim3(kJoinThreads), 0, s, a);
    else
      hipLaunchKernelGGL(join, dim3((unsigned)(rows / (kJoinThreads / (D / 4)))), dim3(kJoinThreads), 0, s, a);
  };
  static_assert(kWaves * 64 == 256, "one block size");
  auto rows = [&](auto one) {
    constexpr bool ONE = decltype(one)::value;
    if (p.rows == 16) go(rows_kernel<E, D, 1, ONE>, join_kernel<E, D, 16, false>, join_kernel<E, D, 16, true>);
    if constexpr (!(D == 256 && E::kBytes == 4)) {
      if (p.rows == 32) go(rows_kernel<E, D, 2, ONE>, join_kernel<E, D, 32, false>, join_kernel<E, D, 32, true>);
    }
  };
  a.T_max == 1 ? rows(std::true_type()) : rows(std::false_type());
  if constexpr (E::kBytes == 2) {
    if (p.rows == kTileRows) go(tile_kernel<D>, join_kernel<E, D, kTileRows, false>, join_kernel<E, D, kTileRows, true>);
  }
  return hipGetLastError();
}

}  // namespace

AttnPlan attn_plan(int B, int T_max, int H_kv, int G, int kv_max, int dtype, int d_head) {
  AttnPlan p;
  const bool bf16 = dtype == TREVS_BF16;
  const long long n_rows = (long long)T_max * G;
  p.rows = n_rows <= 16 || (d_head == 256 && !bf16) ? 16 : n_rows <= 32 || !bf16 ? 32 : kTileRows;
  p.row_tiles = (int)((n_rows + p.rows - 1) / p.rows);
  const long long tiles = (long long)B * H_kv * p.row_tiles, steps = (kv_max + kStep - 1) / kStep;
  // Workgroups of a CU at once, and the steps that one takes side by side.  By their registers three kernels
  // of 64 channels have one more than counted here, whose steps are then longer: counted as they are, calls are
  // cut that lose by it (prompts of 4 x 2048 with 16 heads, 3 for 2: 60 -> 103 us; one token of 32 sequences of
  // 4000, 4 for 3: 41 -> 47, in fp32, 3 for 2: 46 -> 52).  The kernel of 32 rows of 64 channels has 2, and gains
  // by their count (24 rows of 24 sequences of 4000, 2 for 1: 47 -> 38).
  const int per_cu = d_head == 256 ? 1
                     : p.rows == 32 ? (bf16 && d_head == 64 ? 2 : 1)
                     : p.rows == 16 && bf16 ? 3 : 2;
  const long long slots = 256LL * per_cu, side = side_steps(p.rows);
  // Uncut, the last round of workgroups leaves `idle` slots without a tile for as long as a tile takes
  // (a step of a workgroup: about 1.5 us, 3 in fp32); cut, a second launch joins the pieces and each piece
  // begins anew, about 10 us, 25 with the staged kernel's larger sums.  Measured, uncut / cut: one token of
  // 64 sequences of 1.2 k to 16.5 k tokens, 256 tiles for 768 slots, 184 / 107 us; 8 questions over 16.5 k
  // tokens, 224 for 512, 417 / 212; one token of 32 sequences of 4000 with 16 heads of 64, 512 for 768,
  // 41 / 49; a prompt of 1024 rows, 224 for 512, 36 / 51; prompts of 4 x 2048 with 16 heads of 64, 1024 for
  // 512, 64 / 142.  Calls of two rounds or more are not cut: their long tiles go first, and tiles of a group
  // that run at once share its keys in the L2, which pieces do not (prompts of 4259 rows, 3728 for 512:
  // 590 / 1093).  The steps of all must fit 31 bits.
  const long long idle = (tiles + slots - 1) / slots * slots - tiles, begin_us = p.rows == kTileRows ? 25 : 10;
  const bool cut = tiles < 2 * slots && idle * (steps / side) * (bf16 ? 3 : 6) > 2 * begin_us * slots &&
                   tiles * steps < INT32_MAX;
  p.pieces = cut ? (int)std::min(slots, (tiles * steps + side - 1) / side) : 0;
  return p;
}

hipError_t launch_kv8_attention(const AttnArgs& a, const AttnPlan& p, int dtype, int d_head, hipStream_t s) {
  auto by_head = [&](auto e) {
    using E = decltype(e);
    if (d_head == 64) return launch<E, 64>(a, p, s);
    if (d_head == 128) return launch<E, 128>(a, p, s);
    return launch<E, 256>(a, p, s);
  };
  return dtype == TREVS_BF16 ? by_head(BF16()) : by_head(F32());
}

}  // namespace trevs
