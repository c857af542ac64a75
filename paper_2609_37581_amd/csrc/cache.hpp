// The 8-bit paged K/V cache on the device: views, scales and conversions
// shared by the kernels that write, move and read it, and their launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/trevs.h"
#include "common.hpp"

namespace trevs {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// One layer of a cache (k, v and the scales point at the layer).
struct CacheView {
  uint8_t* k;         // [n_pages,H_kv,page,d]
  uint8_t* v;         // [n_pages,H_kv,d,page]
  float* k_scale;     // [n_pages,H_kv]
  float* v_scale;
  const int32_t* table;
  const int32_t* len;
  int n_pages, H_kv, n_slots, max_pages;
};

inline CacheView layer_view(const trevs_kv8_cache& c, int layer) {
  const size_t blocks = (size_t)c.n_pages * c.H_kv, bytes = blocks * c.page_tokens * c.d_head;
  CacheView v;
  v.k = c.k + layer * bytes;
  v.v = c.v + layer * bytes;
  v.k_scale = c.k_scale + layer * blocks;
  v.v_scale = c.v_scale + layer * blocks;
  v.table = c.table;
  v.len = c.len;
  v.n_pages = c.n_pages;
  v.H_kv = c.H_kv;
  v.n_slots = c.n_slots;
  v.max_pages = c.max_pages;
  return v;
}

// Slot of sequence b, -1 if it names none.
__device__ __forceinline__ int slot_of(const int32_t* slots, int b, int n_slots) {
  const int s = slots ? slots[b] : b;
  return s >= 0 && s < n_slots ? s : -1;
}
// Tokens of a slot (clamped: the lengths live in device memory).
__device__ __forceinline__ int slot_len(const int32_t* len, int slot, int max_tokens) {
  return slot < 0 ? 0 : min(max(len[slot], 0), max_tokens);
}
// Page j of a slot, -1 if the entry names none.
__device__ __forceinline__ int page_at(const CacheView& c, int slot, int j) {
  const int p = c.table[(size_t)slot * c.max_pages + j];
  return p >= 0 && p < c.n_pages ? p : -1;
}

// The smallest power of two s with amax <= 448 s, in 2^-126..2^120.  With
// amax = 1.f 2^E and 448 = 1.75 2^8, s = 2^(E-8), or 2^(E-7) when 1.f > 1.75:
// read off the bits, so no division rounds it.
__device__ __forceinline__ float block_scale(float amax) {
  const uint32_t u = __float_as_uint(amax);
  int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);  // biased by 127
  e = min(max(e, 1), 247);
  return __uint_as_float((uint32_t)e << 23);
}
// 1 / s for a power of two 2^-126..2^120 (2^126 and 2^-120 are normal too).
__device__ __forceinline__ float pow2_inverse(float s) {
  return __uint_as_float((254u << 23) - __float_as_uint(s));
}

// Four values over their block's scale as e4m3 bytes (round to nearest even;
// the callers' scales keep |x| * inv within 448, so nothing saturates).
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ void from_e4m3(uint32_t w, float (&x)[4]) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = lo[0];
  x[1] = lo[1];
  x[2] = hi[0];
  x[3] = hi[1];
}
// Four e4m3 values moved to another scale (`ratio` = old scale / new scale).
__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t w, float ratio) {
  float x[4];
  from_e4m3(w, x);
  return to_e4m3(x[0] * ratio, x[1] * ratio, x[2] * ratio, x[3] * ratio);
}

// ------------------------------------------------------------------ launchers
struct RopeTensor {
  const uint8_t* in;
  uint8_t* out;
  long long in_ld, out_ld;  // bytes from one row to the next
  int H;
};
struct RopeArgs {
  RopeTensor t[2];          // q, k (H = 0: absent)
  const double* freqs;
  const int64_t* pos;
  long long rows;           // B * S
  int d_head, rot_dim, n_pos;
  int bound[TREVS_MAX_POS_PLANES];  // pairs before bound[p] belong to planes 0..p
  int copy_tail;            // values past rot_dim are copied (0: every tensor is turned in place)
  float attn_factor;        // negated sine for the inverse is `sign`
  float sign;
};
int rope_rows(long long rows, int rot_dim);  // rows of a workgroup
hipError_t launch_rope(const RopeArgs& a, int interleaved, int dtype, hipStream_t s);

struct NormRopeArgs {
  RopeArgs rope;
  const void* q_weight;     // null: ones
  const void* k_weight;
  float eps, weight_offset;
  int weight_bf16, per_head;
};
hipError_t launch_norm_rope(const NormRopeArgs& n, int interleaved, int dtype, hipStream_t s);

struct WriteArgs {
  CacheView c;
  const void* k;
  const void* v;
  long long k_ld, v_ld;     // elements
  const int32_t* n_new;
  const int32_t* slots;
  int B, T_max, frames;     // frames: pages a sequence's rows may touch
};
hipError_t launch_kv8_write(const WriteArgs& a, int dtype, int d_head, int page, hipStream_t s);

struct CompactArgs {
  CacheView c;              // layer 0
  const int32_t* kept;
  const int32_t* src;
  const int32_t* dst;
  int B, P, K_in, n_kept, n_layers;
  int frames;               // blocks of a sequence and head that the launch has workgroups for;
  int turns;                // others are taken in turns (0: there are none)
};
hipError_t launch_kv8_compact(const CompactArgs& a, int d_head, int page, hipStream_t s);

// What eviction does with one request: its slot (-1: nothing), tokens before and
// after, the first kept token that is not where it was (n: none), and the first
// page that is given up.
struct EvictInfo {
  int slot, len, n, moved, first_page;
};
struct EvictArgs {
  CacheView c;              // layer 0
  int32_t* ref;
  float* score;             // [n_slots, max_pages * page]
  const int32_t* keep;
  const int32_t* slots;
  int32_t* n_evicted;
  int32_t* kept_idx;        // [B,n_keep]
  EvictInfo* info;          // [B]
  int32_t* old;             // [B,max_pages] the slots' pages before
  int B, n_keep, n_first, n_last, n_layers, page_shift;
  int frames, turns;        // as in CompactArgs
};
hipError_t launch_evict_select(const EvictArgs& a, hipStream_t s);
hipError_t launch_evict_pages(const EvictArgs& a, hipStream_t s);
hipError_t launch_kv8_evict(const EvictArgs& a, int d_head, int page, hipStream_t s);

struct CopyArgs {
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
  const int32_t* src;
  const int32_t* dst;
  int n, n_layers, n_pages, H_kv;
  int page_bytes;           // bytes of one page's keys: H_kv * page_tokens * d_head
};
hipError_t launch_kv8_copy(const CopyArgs& a, hipStream_t s);

struct AttnArgs {
  CacheView c;
  const void* q;
  long long q_ld;           // elements
  const int32_t* q_len;
  const int32_t* slots;
  void* out;
  float* lse;
  int B, T_max, H_q, G, causal, kv_max, page_shift;
  float scale_log2e;
  int row_tiles;
  float* part;              // cut calls (else null): [2 pieces,rows,D] sums of a workgroup's pieces
  float2* part_ml;          // [2 pieces,rows] their (maximum, sum), base 2
  int2* tile_pieces;        // [B,H_kv,row_tiles] first and last workgroup of each tile with steps
};
// Launch shape of one problem size.
struct AttnPlan {
  int rows;                 // query rows of a tile
  int row_tiles;
  int pieces;               // the most workgroups that the steps of all tiles are cut for, 0: a tile to a workgroup
};
AttnPlan attn_plan(int B, int T_max, int H_kv, int G, int kv_max, int dtype, int d_head);
hipError_t launch_kv8_attention(const AttnArgs& a, const AttnPlan& p, int dtype, int d_head, hipStream_t s);

// How the weights of a call are split: few query rows a group in one launch, many
// into parts of (KV heads, pieces of the rows), summed by a second one.
struct WeightsPlan {
  bool few;
  int tokens;               // of a workgroup's block
  int key_blocks, heads, head_groups, pieces;
};
struct WeightsArgs {
  CacheView c;
  const void* q;
  long long q_ld;           // elements
  const int32_t* q_len;
  const int32_t* slots;
  const float* lse;
  float* score;             // [n_slots,width]
  float* part;              // [B,head_groups,pieces,kv_max]
  int B, T_max, H_q, G, causal, kv_max, width, page_shift;
  float scale_log2e, decay;
  int key_blocks, heads, head_groups, pieces;
};
WeightsPlan weights_plan(int B, int T_max, int H_kv, int G, int kv_max, int dtype);
hipError_t launch_kv8_weights(const WeightsArgs& a, const WeightsPlan& p, int dtype, int d_head, hipStream_t s);

struct PagesArgs {
  int32_t* table;
  int32_t* len;
  int32_t* ref;
  int n_pages, n_slots, max_pages, page_shift;
  int n;
};
hipError_t launch_pages_reserve(const PagesArgs& a, const int32_t* slots, const int32_t* n_new, int32_t* granted,
                                int32_t* copy_src, int32_t* copy_dst, hipStream_t s);
hipError_t launch_pages_fork(const PagesArgs& a, const int32_t* src, const int32_t* dst, const int32_t* n_tokens,
                             int32_t* done, hipStream_t s);
hipError_t launch_pages_reorder(const PagesArgs& a, int groups, int width, const int32_t* slots, const int32_t* parent,
                                float* score, hipStream_t s);
hipError_t launch_pages_free(const PagesArgs& a, const int32_t* slots, const int32_t* keep, hipStream_t s);

}  // namespace trevs
