// Host side of the serving-cache entry points: rotary positions and head norms,
// the 8-bit paged K/V cache, its attention and its page operations, eviction and
// beam search.  Arguments are validated before anything is launched; nothing
// allocates device memory or waits for the device.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "beam.hpp"
#include "cache.hpp"
#include "host.hpp"

using namespace trevs;

namespace {

// A [rows, width] view whose rows lie ld bytes apart.
struct Rows {
  const void* p;
  int64_t rows, width, ld;  // bytes
  Span span() const { return Span{p, p && rows ? (size_t)((rows - 1) * ld + width) : 0}; }
};

// Views into one buffer (q, k and v beside each other in a row) may interleave:
// with one row distance they meet only where their columns do.
bool overlap(const Rows& a, const Rows& b) {
  if (!trevs::overlap(a.span(), b.span())) return false;
  if (a.ld != b.ld) return true;
  const int64_t diff = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
  const int64_t col = ((diff % a.ld) + a.ld) % a.ld;
  return col < a.width || col + b.width > a.ld;
}
bool overlap(const Rows& a, Span b) { return trevs::overlap(a.span(), b); }

// Row distance in elements: 0 stands for dense rows; 0 is returned for an invalid one.
int64_t row_ld(int64_t ld, int64_t width, int elem) {
  if (ld == 0) return width;
  return ld < width || ld > INT32_MAX || (ld * elem) % 16 ? 0 : ld;
}

bool head_size_ok(int d) { return d == 64 || d == 128 || d == 256; }

// ------------------------------------------------------------------- rotary
trevs_status validate_rope(const trevs_rope_args* a) {
  if (!a || a->struct_size != sizeof(trevs_rope_args)) return TREVS_ERR_INVALID_ARG;
  if (a->dtype != TREVS_F32 && a->dtype != TREVS_BF16) return TREVS_ERR_INVALID_ARG;
  if (a->B < 1 || a->S < 1 || a->H_q < 0 || a->H_k < 0 || a->H_q + (int64_t)a->H_k < 1) return TREVS_ERR_INVALID_ARG;
  if (a->d_head < 1 || a->rot_dim < 16 || a->rot_dim % 16 || a->rot_dim > a->d_head) return TREVS_ERR_INVALID_ARG;
  if (a->n_pos < 1 || a->n_pos > TREVS_MAX_POS_PLANES) return TREVS_ERR_INVALID_ARG;
  if ((a->interleaved | a->inverse) & ~1) return TREVS_ERR_INVALID_ARG;
  if (!finite(a->attn_factor)) return TREVS_ERR_INVALID_ARG;
  int64_t pairs = 0;
  for (int p = 0; p < a->n_pos; ++p) {
    if (a->section[p] < 0) return TREVS_ERR_INVALID_ARG;
    pairs += a->section[p];
  }
  if (pairs != a->rot_dim / 2) return TREVS_ERR_INVALID_ARG;
  if (!a->freqs || !a->pos || !aligned(a->freqs, 8) || !aligned(a->pos, 8)) return TREVS_ERR_INVALID_ARG;
  const int e = elem_bytes(a->dtype);
  const void* in[2] = {a->q, a->k};
  void* out[2] = {a->q_out, a->k_out};
  const int H[2] = {a->H_q, a->H_k};
  const int64_t in_ld[2] = {a->q_ld, a->k_ld}, out_ld[2] = {a->q_out_ld, a->k_out_ld};
  if (!head_size_ok(a->d_head)) return TREVS_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)a->B * a->S;
  if (rows * a->n_pos > INT32_MAX || a->H_q > 1024 || a->H_k > 1024) return TREVS_ERR_UNSUPPORTED;
  const int per_group = rope_rows(rows, a->rot_dim);
  if ((rows + per_group - 1) / per_group > kMaxGroups) return TREVS_ERR_UNSUPPORTED;
  Rows src[2] = {}, dst[2] = {};
  for (int i = 0; i < 2; ++i) {
    if (H[i] == 0) continue;
    const int64_t width = (int64_t)H[i] * a->d_head, li = row_ld(in_ld[i], width, e), lo = row_ld(out_ld[i], width, e);
    if (!in[i] || !out[i] || !aligned(in[i], 16) || !aligned(out[i], 16) || !li || !lo) return TREVS_ERR_INVALID_ARG;
    if (in[i] == out[i] && li != lo) return TREVS_ERR_INVALID_ARG;
    src[i] = Rows{in[i], rows, width * e, li * e};
    dst[i] = Rows{out[i], rows, width * e, lo * e};
  }
  const Span pos{a->pos, (size_t)rows * a->n_pos * 8}, freqs{a->freqs, (size_t)a->rot_dim / 2 * 8};
  for (int i = 0; i < 2; ++i) {
    if (H[i] == 0) continue;
    if (overlap(dst[i], pos) || overlap(dst[i], freqs)) return TREVS_ERR_INVALID_ARG;
    for (int j = 0; j < 2; ++j) {
      if (H[j] == 0) continue;
      if (!(i == j && in[i] == out[i]) && overlap(dst[i], src[j])) return TREVS_ERR_INVALID_ARG;
      if (j > i && overlap(dst[i], dst[j])) return TREVS_ERR_INVALID_ARG;
    }
  }
  return TREVS_OK;
}

RopeArgs rope_args(const trevs_rope_args* a) {
  const int e = elem_bytes(a->dtype);
  RopeArgs r = {};
  const void* in[2] = {a->q, a->k};
  void* out[2] = {a->q_out, a->k_out};
  const int H[2] = {a->H_q, a->H_k};
  const int64_t in_ld[2] = {a->q_ld, a->k_ld}, out_ld[2] = {a->q_out_ld, a->k_out_ld};
  for (int i = 0; i < 2; ++i) {
    const int64_t width = (int64_t)H[i] * a->d_head;
    r.t[i].in = reinterpret_cast<const uint8_t*>(in[i]);
    r.t[i].out = reinterpret_cast<uint8_t*>(out[i]);
    r.t[i].in_ld = row_ld(in_ld[i], width, e) * e;
    r.t[i].out_ld = row_ld(out_ld[i], width, e) * e;
    r.t[i].H = H[i];
    r.copy_tail |= H[i] > 0 && in[i] != out[i];
  }
  r.freqs = a->freqs;
  r.pos = a->pos;
  r.rows = (long long)a->B * a->S;
  r.d_head = a->d_head;
  r.rot_dim = a->rot_dim;
  r.n_pos = a->n_pos;
  for (int p = 0, at = 0; p < a->n_pos; ++p) r.bound[p] = at += a->section[p];
  r.attn_factor = a->attn_factor;
  r.sign = a->inverse ? -1.f : 1.f;
  return r;
}

trevs_status validate_norm_rope(const trevs_norm_rope_args* a) {
  if (!a || a->struct_size != sizeof(trevs_norm_rope_args)) return TREVS_ERR_INVALID_ARG;
  if (a->weight_dtype != TREVS_F32 && a->weight_dtype != TREVS_BF16) return TREVS_ERR_INVALID_ARG;
  if (!(a->eps >= FLT_MIN) || !finite(a->eps) || !finite(a->weight_offset) || (a->per_head & ~1))
    return TREVS_ERR_INVALID_ARG;
  if (!aligned(a->q_weight, 16) || !aligned(a->k_weight, 16)) return TREVS_ERR_INVALID_ARG;
  const trevs_rope_args* r = &a->rope;
  TREVS_TRY(validate_rope(r));
  if (r->inverse) return TREVS_ERR_INVALID_ARG;
  // the weights lie outside what is written
  const int e = elem_bytes(r->dtype), we = elem_bytes(a->weight_dtype);
  const void* weight[2] = {a->q_weight, a->k_weight};
  void* out[2] = {r->q_out, r->k_out};
  const int H[2] = {r->H_q, r->H_k};
  const int64_t out_ld[2] = {r->q_out_ld, r->k_out_ld};
  for (int i = 0; i < 2; ++i) {
    if (H[i] == 0) continue;
    const int64_t width = (int64_t)H[i] * r->d_head;
    const Rows to{out[i], (int64_t)r->B * r->S, width * e, row_ld(out_ld[i], width, e) * e};
    for (int j = 0; j < 2; ++j) {
      if (H[j] == 0 || !weight[j]) continue;
      const int64_t n = (int64_t)(a->per_head ? H[j] : 1) * r->d_head;
      if (overlap(to, Span{weight[j], (size_t)n * we})) return TREVS_ERR_INVALID_ARG;
    }
  }
  return TREVS_OK;
}

// -------------------------------------------------------------------- cache
trevs_status validate_cache(const trevs_kv8_cache* c) {
  if (!c || c->struct_size != sizeof(trevs_kv8_cache)) return TREVS_ERR_INVALID_ARG;
  if (c->n_layers < 1 || c->n_pages < 1 || c->H_kv < 1 || c->n_slots < 1 || c->max_pages < 1)
    return TREVS_ERR_INVALID_ARG;
  if (c->d_head < 1 || c->page_tokens < 1) return TREVS_ERR_INVALID_ARG;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->table || !c->len || !c->ref) return TREVS_ERR_INVALID_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4) ||
      !aligned(c->table, 4) || !aligned(c->len, 4) || !aligned(c->ref, 4))
    return TREVS_ERR_INVALID_ARG;
  if (!head_size_ok(c->d_head)) return TREVS_ERR_UNSUPPORTED;
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64) return TREVS_ERR_UNSUPPORTED;
  if (c->n_layers > 1024 || c->H_kv > 1024) return TREVS_ERR_UNSUPPORTED;
  if ((int64_t)c->max_pages * c->page_tokens > (1 << 30)) return TREVS_ERR_UNSUPPORTED;
  return TREVS_OK;
}

constexpr int kCacheSpans = 7;
void cache_spans(const trevs_kv8_cache* c, Span (&s)[kCacheSpans]) {
  const size_t blocks = (size_t)c->n_layers * c->n_pages * c->H_kv, bytes = blocks * c->page_tokens * c->d_head;
  s[0] = Span{c->k, bytes};
  s[1] = Span{c->v, bytes};
  s[2] = Span{c->k_scale, blocks * 4};
  s[3] = Span{c->v_scale, blocks * 4};
  s[4] = Span{c->table, (size_t)c->n_slots * c->max_pages * 4};
  s[5] = Span{c->len, (size_t)c->n_slots * 4};
  s[6] = Span{c->ref, (size_t)c->n_pages * 4};
}
bool meets_cache(const trevs_kv8_cache* c, Span x) {
  Span s[kCacheSpans];
  cache_spans(c, s);
  for (const Span& y : s)
    if (overlap(x, y)) return true;
  return false;
}

trevs_status validate_list(const trevs_kv8_cache* c, int32_t n, const int32_t* slots, bool slots_needed) {
  TREVS_TRY(validate_cache(c));
  if (n < 1 || (slots_needed && !slots) || !aligned(slots, 4)) return TREVS_ERR_INVALID_ARG;
  if (!slots && n > c->n_slots) return TREVS_ERR_INVALID_ARG;
  if (n > TREVS_MAX_PAGE_REQUESTS) return TREVS_ERR_UNSUPPORTED;
  return TREVS_OK;
}

int page_shift(const trevs_kv8_cache* c) { return c->page_tokens == 16 ? 4 : c->page_tokens == 32 ? 5 : 6; }

PagesArgs pages_args(const trevs_kv8_cache* c, int n) {
  PagesArgs p;
  p.table = c->table;
  p.len = c->len;
  p.ref = c->ref;
  p.n_pages = c->n_pages;
  p.n_slots = c->n_slots;
  p.max_pages = c->max_pages;
  p.page_shift = page_shift(c);
  p.n = n;
  return p;
}

trevs_status validate_write(const trevs_kv8_cache* c, const trevs_kv8_write_args* a) {
  TREVS_TRY(validate_cache(c));
  if (!a || a->struct_size != sizeof(trevs_kv8_write_args)) return TREVS_ERR_INVALID_ARG;
  if (a->dtype != TREVS_F32 && a->dtype != TREVS_BF16) return TREVS_ERR_INVALID_ARG;
  if (a->B < 1 || a->T_max < 1 || a->layer < 0 || a->layer >= c->n_layers) return TREVS_ERR_INVALID_ARG;
  if (!a->slots && a->B > c->n_slots) return TREVS_ERR_INVALID_ARG;
  const int e = elem_bytes(a->dtype);
  const int64_t width = (int64_t)c->H_kv * c->d_head, rows = (int64_t)a->B * a->T_max;
  const int64_t kl = row_ld(a->k_ld, width, e), vl = row_ld(a->v_ld, width, e);
  if (!a->k || !a->v || !aligned(a->k, 16) || !aligned(a->v, 16) || !kl || !vl) return TREVS_ERR_INVALID_ARG;
  if (!aligned(a->n_new, 4) || !aligned(a->slots, 4)) return TREVS_ERR_INVALID_ARG;
  if (rows > INT32_MAX) return TREVS_ERR_UNSUPPORTED;
  const int64_t frames = ((int64_t)a->T_max + c->page_tokens - 2) / c->page_tokens + 1;
  if (a->B * frames * c->H_kv > kMaxGroups) return TREVS_ERR_UNSUPPORTED;
  const Rows k{a->k, rows, width * e, kl * e}, v{a->v, rows, width * e, vl * e};
  if (meets_cache(c, k.span()) || meets_cache(c, v.span()) || meets_cache(c, Span{a->n_new, (size_t)a->B * 4}) ||
      meets_cache(c, Span{a->slots, (size_t)a->B * 4}))
    return TREVS_ERR_INVALID_ARG;
  return TREVS_OK;
}

int max_keys(const trevs_kv8_cache* c, const trevs_kv8_attention_args* a) {
  return a->kv_max ? a->kv_max : c->max_pages * c->page_tokens;
}
AttnPlan plan_of(const trevs_kv8_cache* c, const trevs_kv8_attention_args* a) {
  return attn_plan(a->B, a->T_max, c->H_kv, a->H_q / c->H_kv, max_keys(c, a), a->dtype, c->d_head);
}

trevs_status validate_attention(const trevs_kv8_cache* c, const trevs_kv8_attention_args* a) {
  TREVS_TRY(validate_cache(c));
  if (!a || a->struct_size != sizeof(trevs_kv8_attention_args)) return TREVS_ERR_INVALID_ARG;
  if (a->dtype != TREVS_F32 && a->dtype != TREVS_BF16) return TREVS_ERR_INVALID_ARG;
  if (a->B < 1 || a->T_max < 1 || a->layer < 0 || a->layer >= c->n_layers) return TREVS_ERR_INVALID_ARG;
  if (a->H_q < 1 || a->H_q % c->H_kv || (a->causal & ~1)) return TREVS_ERR_INVALID_ARG;
  if (a->kv_max < 0 || a->kv_max > c->max_pages * c->page_tokens) return TREVS_ERR_INVALID_ARG;
  if (!finite(a->scale) || a->scale <= 0.f) return TREVS_ERR_INVALID_ARG;
  if (!a->slots && a->B > c->n_slots) return TREVS_ERR_INVALID_ARG;
  const int e = elem_bytes(a->dtype);
  const int64_t width = (int64_t)a->H_q * c->d_head, rows = (int64_t)a->B * a->T_max;
  const int64_t ql = row_ld(a->q_ld, width, e);
  if (!a->q || !a->out || !aligned(a->q, 16) || !aligned(a->out, 16) || !ql) return TREVS_ERR_INVALID_ARG;
  if (!aligned(a->q_len, 4) || !aligned(a->slots, 4) || !aligned(a->lse, 4)) return TREVS_ERR_INVALID_ARG;
  if (a->H_q > 1024 || rows * a->H_q > INT32_MAX - 1024) return TREVS_ERR_UNSUPPORTED;  // (row tiles stay in 32 bits)
  const Rows q{a->q, rows, width * e, ql * e};
  const Span out[] = {{a->out, (size_t)(rows * width * e)}, {a->lse, a->lse ? (size_t)(rows * a->H_q * 4) : 0}};
  const Span in[] = {q.span(), {a->q_len, a->q_len ? (size_t)a->B * 4 : 0}, {a->slots, a->slots ? (size_t)a->B * 4 : 0}};
  if (any_overlap(out, 2, in, 3)) return TREVS_ERR_INVALID_ARG;
  for (const Span& o : out)
    if (meets_cache(c, o)) return TREVS_ERR_INVALID_ARG;
  if ((int64_t)a->B * c->H_kv * plan_of(c, a).row_tiles > kMaxGroups) return TREVS_ERR_UNSUPPORTED;
  return TREVS_OK;
}

// Cut calls: the tiles' pieces, then their sums: (maximum, sum) pairs and values.
struct AttnLayout {
  AttnPlan plan;
  size_t part_ml, part, total;
};
AttnLayout attention_layout(const trevs_kv8_cache* c, const trevs_kv8_attention_args* a) {
  AttnLayout L;
  L.plan = plan_of(c, a);
  const size_t parts = (size_t)2 * L.plan.pieces * L.plan.rows;
  L.part_ml = parts ? align_up((size_t)a->B * c->H_kv * L.plan.row_tiles * sizeof(int2)) : 0;
  L.part = L.part_ml + align_up(parts * sizeof(float2));
  L.total = std::max(L.part + align_up(parts * c->d_head * sizeof(float)), kWsAlign);
  return L;
}

trevs_status validate_compact(const trevs_kv8_cache* c, const trevs_kv8_compact_args* a) {
  TREVS_TRY(validate_cache(c));
  if (!a || a->struct_size != sizeof(trevs_kv8_compact_args)) return TREVS_ERR_INVALID_ARG;
  if (a->B < 1 || a->P < 0 || a->K_in < 1 || a->n_kept < 1 || a->n_kept > a->K_in) return TREVS_ERR_INVALID_ARG;
  if (!a->kept_idx || !a->src_slots || !a->dst_slots) return TREVS_ERR_INVALID_ARG;
  if (!aligned(a->kept_idx, 4) || !aligned(a->src_slots, 4) || !aligned(a->dst_slots, 4)) return TREVS_ERR_INVALID_ARG;
  if ((int64_t)a->P + a->K_in > (int64_t)c->max_pages * c->page_tokens) return TREVS_ERR_INVALID_ARG;
  if ((int64_t)a->B * a->n_kept > INT32_MAX) return TREVS_ERR_UNSUPPORTED;
  if ((int64_t)c->n_layers * a->B * c->H_kv > kMaxGroups) return TREVS_ERR_UNSUPPORTED;
  const size_t B = a->B;
  if (meets_cache(c, Span{a->kept_idx, B * a->n_kept * 4}) || meets_cache(c, Span{a->src_slots, B * 4}) ||
      meets_cache(c, Span{a->dst_slots, B * 4}))
    return TREVS_ERR_INVALID_ARG;
  return TREVS_OK;
}

// The compaction's launch: the sequences' lengths are on the device, so it has a workgroup for every block that
// the table can hold (a shorter source is skipped), unless that is more than twice what the prefix and the kept
// rows fill twice, or 8192 workgroups of keys and values: longer sequences' blocks are then taken in turns.
void plan_compact(const trevs_kv8_cache* c, const trevs_kv8_compact_args* a, CompactArgs* t) {
  const int64_t each = (int64_t)c->n_layers * a->B * c->H_kv, page = c->page_tokens;
  const int64_t table = ((int64_t)c->max_pages * page - a->K_in + a->n_kept + page - 1) / page;
  const int64_t wanted = std::max(2 * (((int64_t)a->P + a->n_kept + page - 1) / page), 4096 / each);
  t->frames = (int)std::min(table > 2 * wanted ? wanted : table, kMaxGroups / each);
  t->turns = t->frames < table;
}

size_t score_bytes(const trevs_kv8_cache* c) { return (size_t)c->n_slots * c->max_pages * c->page_tokens * 4; }

int weights_keys(const trevs_kv8_cache* c, const trevs_kv8_weights_args* a) {
  return a->kv_max ? a->kv_max : c->max_pages * c->page_tokens;
}
WeightsPlan plan_of(const trevs_kv8_cache* c, const trevs_kv8_weights_args* a) {
  return weights_plan(a->B, a->T_max, c->H_kv, a->H_q / c->H_kv, weights_keys(c, a), a->dtype);
}

trevs_status validate_weights(const trevs_kv8_cache* c, const trevs_kv8_weights_args* a) {
  TREVS_TRY(validate_cache(c));
  if (!a || a->struct_size != sizeof(trevs_kv8_weights_args)) return TREVS_ERR_INVALID_ARG;
  if (a->dtype != TREVS_F32 && a->dtype != TREVS_BF16) return TREVS_ERR_INVALID_ARG;
  if (a->B < 1 || a->T_max < 1 || a->layer < 0 || a->layer >= c->n_layers) return TREVS_ERR_INVALID_ARG;
  if (a->H_q < 1 || a->H_q % c->H_kv || (a->causal & ~1)) return TREVS_ERR_INVALID_ARG;
  if (a->kv_max < 0 || a->kv_max > c->max_pages * c->page_tokens) return TREVS_ERR_INVALID_ARG;
  if (!finite(a->scale) || a->scale <= 0.f || !finite(a->decay) || a->decay < 0.f) return TREVS_ERR_INVALID_ARG;
  if (a->B > c->n_slots) return TREVS_ERR_INVALID_ARG;  // (no slot twice)
  const int e = elem_bytes(a->dtype);
  const int64_t width = (int64_t)a->H_q * c->d_head, rows = (int64_t)a->B * a->T_max;
  const int64_t ql = row_ld(a->q_ld, width, e);
  if (!a->q || !a->lse || !a->score || !aligned(a->q, 16) || !aligned(a->lse, 4) || !aligned(a->score, 4) || !ql)
    return TREVS_ERR_INVALID_ARG;
  if (!aligned(a->q_len, 4) || !aligned(a->slots, 4)) return TREVS_ERR_INVALID_ARG;
  if (a->H_q > 1024 || rows * a->H_q > INT32_MAX - 1024 || a->B > 65535) return TREVS_ERR_UNSUPPORTED;
  const Rows q{a->q, rows, width * e, ql * e};
  const Span score{a->score, score_bytes(c)};
  const Span in[] = {q.span(), {a->q_len, a->q_len ? (size_t)a->B * 4 : 0}, {a->slots, a->slots ? (size_t)a->B * 4 : 0},
                     {a->lse, (size_t)(rows * a->H_q * 4)}};
  if (any_overlap(&score, 1, in, 4) || meets_cache(c, score)) return TREVS_ERR_INVALID_ARG;
  const WeightsPlan p = plan_of(c, a);
  const int64_t groups = (int64_t)a->B * p.head_groups * p.key_blocks;
  if (p.few ? (int64_t)a->B * p.key_blocks > INT32_MAX : groups > kMaxGroups / p.pieces) return TREVS_ERR_UNSUPPORTED;
  return TREVS_OK;
}
size_t weights_bytes(const trevs_kv8_cache* c, const trevs_kv8_weights_args* a) {
  const WeightsPlan p = plan_of(c, a);
  if (p.few) return kWsAlign;
  return align_up((size_t)a->B * p.head_groups * p.pieces * weights_keys(c, a) * sizeof(float));
}

trevs_status validate_evict(const trevs_kv8_cache* c, const trevs_kv8_evict_args* a) {
  TREVS_TRY(validate_cache(c));
  if (!a || a->struct_size != sizeof(trevs_kv8_evict_args)) return TREVS_ERR_INVALID_ARG;
  if (a->B < 1 || a->n_keep < 1 || a->n_first < 0 || a->n_last < 0 || (int64_t)a->n_first + a->n_last > a->n_keep)
    return TREVS_ERR_INVALID_ARG;
  if (!a->score || !a->n_evicted || !a->kept_idx) return TREVS_ERR_INVALID_ARG;
  if (!aligned(a->score, 4) || !aligned(a->n_evicted, 4) || !aligned(a->kept_idx, 4) || !aligned(a->keep, 4) ||
      !aligned(a->slots, 4))
    return TREVS_ERR_INVALID_ARG;
  if (!a->slots && a->B > c->n_slots) return TREVS_ERR_INVALID_ARG;
  if (a->B > TREVS_MAX_PAGE_REQUESTS) return TREVS_ERR_UNSUPPORTED;
  // (places up to a workgroup past the list stay in 32 bits)
  if ((int64_t)a->B * a->n_keep > INT32_MAX - 1024) return TREVS_ERR_UNSUPPORTED;
  if ((int64_t)c->n_layers * a->B * c->H_kv + a->B > kMaxGroups) return TREVS_ERR_UNSUPPORTED;
  const size_t list = (size_t)a->B * 4;
  const Span out[] = {{a->score, score_bytes(c)}, {a->n_evicted, list}, {a->kept_idx, list * a->n_keep}};
  const Span in[] = {{a->keep, a->keep ? list : 0}, {a->slots, a->slots ? list : 0}};
  if (any_overlap(out, 3, in, 2)) return TREVS_ERR_INVALID_ARG;
  for (const Span& x : out)
    if (meets_cache(c, x)) return TREVS_ERR_INVALID_ARG;
  for (const Span& x : in)
    if (meets_cache(c, x)) return TREVS_ERR_INVALID_ARG;
  return TREVS_OK;
}
size_t evict_info_bytes(const trevs_kv8_evict_args* a) { return align_up((size_t)a->B * sizeof(EvictInfo)); }

// ---------------------------------------------------------------- beam search
int beam_chunks(const trevs_beam_select_args* a) {
  const int chunk = beam_chunk(a->dtype);
  return (int)(((int64_t)a->V + chunk - 1) / chunk);
}

trevs_status validate_beam(const trevs_beam_select_args* a) {
  if (!a || a->struct_size != sizeof(trevs_beam_select_args)) return TREVS_ERR_INVALID_ARG;
  if (a->dtype != TREVS_F32 && a->dtype != TREVS_BF16) return TREVS_ERR_INVALID_ARG;
  if (a->B < 1 || a->W < 1 || a->V < 1 || a->n_out < 1 || a->eos < 0 || a->eos >= a->V) return TREVS_ERR_INVALID_ARG;
  if (a->logits_ld != 0 && a->logits_ld < a->V) return TREVS_ERR_INVALID_ARG;
  const int e = elem_bytes(a->dtype);
  if (!a->logits || !a->score || !a->score_out || !a->parent || !a->token) return TREVS_ERR_INVALID_ARG;
  if (!aligned(a->logits, e) || !aligned(a->score, 4) || !aligned(a->done, 4) || !aligned(a->score_out, 4) ||
      !aligned(a->parent, 4) || !aligned(a->token, 4))
    return TREVS_ERR_INVALID_ARG;
  if (a->W > TREVS_MAX_BEAMS || a->n_out > TREVS_MAX_BEAM_OUT || a->logits_ld > INT32_MAX) return TREVS_ERR_UNSUPPORTED;
  // (places up to a chunk past the vocabulary stay in 32 bits)
  if ((int64_t)a->W * a->V > INT32_MAX - beam_chunk(a->dtype) || (int64_t)a->B * a->W > INT32_MAX)
    return TREVS_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)a->B * a->W, ld = a->logits_ld ? a->logits_ld : a->V;
  if (rows > kMaxGroups / beam_chunks(a) || a->B > kMaxGroups / 4) return TREVS_ERR_UNSUPPORTED;
  const size_t list = (size_t)a->B * a->n_out * 4;
  const Span out[] = {{a->score_out, list}, {a->parent, list}, {a->token, list}};
  const Span in[] = {{a->logits, (size_t)((rows - 1) * ld + a->V) * e}, {a->score, (size_t)rows * 4},
                     {a->done, a->done ? (size_t)rows * 4 : 0}};
  if (any_overlap(out, 3, in, 3)) return TREVS_ERR_INVALID_ARG;
  return TREVS_OK;
}
size_t beam_part_bytes(const trevs_beam_select_args* a) {
  return align_up((size_t)a->B * a->W * beam_chunks(a) * sizeof(float2));
}

}  // namespace

extern "C" {

size_t trevs_rope_args_size(void) { return sizeof(trevs_rope_args); }
size_t trevs_kv8_cache_size(void) { return sizeof(trevs_kv8_cache); }
size_t trevs_kv8_write_args_size(void) { return sizeof(trevs_kv8_write_args); }
size_t trevs_kv8_attention_args_size(void) { return sizeof(trevs_kv8_attention_args); }
size_t trevs_kv8_compact_args_size(void) { return sizeof(trevs_kv8_compact_args); }
size_t trevs_norm_rope_args_size(void) { return sizeof(trevs_norm_rope_args); }
size_t trevs_kv8_weights_args_size(void) { return sizeof(trevs_kv8_weights_args); }
size_t trevs_kv8_evict_args_size(void) { return sizeof(trevs_kv8_evict_args); }
size_t trevs_beam_select_args_size(void) { return sizeof(trevs_beam_select_args); }

trevs_status trevs_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double original_len,
                                    double beta_fast, double beta_slow, double* freqs) {
  if (!freqs || rot_dim < 2 || rot_dim % 2 || !isfinite(base) || base <= 0.0) return TREVS_ERR_INVALID_ARG;
  if (scaling < TREVS_ROPE_NONE || scaling > TREVS_ROPE_PARTS) return TREVS_ERR_INVALID_ARG;
  if (scaling != TREVS_ROPE_NONE && (!isfinite(factor) || factor <= 0.0)) return TREVS_ERR_INVALID_ARG;
  if (scaling == TREVS_ROPE_PARTS && (!isfinite(original_len) || original_len <= 0.0 || !isfinite(beta_fast) ||
                                      !isfinite(beta_slow) || beta_fast <= beta_slow))
    return TREVS_ERR_INVALID_ARG;
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / rot_dim) / 6.283185307179586476925;
    if (scaling == TREVS_ROPE_LINEAR) f /= factor;
    if (scaling == TREVS_ROPE_PARTS) {
      const double own = std::min(std::max((original_len * f - beta_slow) / (beta_fast - beta_slow), 0.0), 1.0);
      f = f * own + f / factor * (1.0 - own);
    }
    freqs[i] = f;
  }
  return TREVS_OK;
}

trevs_status trevs_rope(const trevs_rope_args* a, void* stream) {
  TREVS_TRY(validate_rope(a));
  TREVS_HIP(launch_rope(rope_args(a), a->interleaved, a->dtype, reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

trevs_status trevs_norm_rope(const trevs_norm_rope_args* a, void* stream) {
  TREVS_TRY(validate_norm_rope(a));
  NormRopeArgs n;
  n.rope = rope_args(&a->rope);
  n.q_weight = a->q_weight;
  n.k_weight = a->k_weight;
  n.eps = a->eps;
  n.weight_offset = a->weight_offset;
  n.weight_bf16 = a->weight_dtype == TREVS_BF16;
  n.per_head = a->per_head;
  TREVS_HIP(launch_norm_rope(n, a->rope.interleaved, a->rope.dtype, reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

trevs_status trevs_pages_reserve(const trevs_kv8_cache* c, int32_t n, const int32_t* slots, const int32_t* n_new,
                                 int32_t* granted, int32_t* copy_src, int32_t* copy_dst, void* stream) {
  TREVS_TRY(validate_list(c, n, slots, false));
  if (!n_new || !granted || !copy_src || !copy_dst) return TREVS_ERR_INVALID_ARG;
  if (!aligned(n_new, 4) || !aligned(granted, 4) || !aligned(copy_src, 4) || !aligned(copy_dst, 4))
    return TREVS_ERR_INVALID_ARG;
  const size_t bytes = (size_t)n * 4;
  const Span out[] = {{granted, bytes}, {copy_src, bytes}, {copy_dst, bytes}};
  const Span in[] = {{slots, slots ? bytes : 0}, {n_new, bytes}};
  if (any_overlap(out, 3, in, 2)) return TREVS_ERR_INVALID_ARG;
  for (const Span& x : out)
    if (meets_cache(c, x)) return TREVS_ERR_INVALID_ARG;
  for (const Span& x : in)
    if (meets_cache(c, x)) return TREVS_ERR_INVALID_ARG;
  TREVS_HIP(launch_pages_reserve(pages_args(c, n), slots, n_new, granted, copy_src, copy_dst,
                                 reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

trevs_status trevs_pages_fork(const trevs_kv8_cache* c, int32_t n, const int32_t* src, const int32_t* dst,
                              const int32_t* n_tokens, int32_t* done, void* stream) {
  TREVS_TRY(validate_list(c, n, src, true));
  if (!dst || !done || !aligned(dst, 4) || !aligned(n_tokens, 4) || !aligned(done, 4)) return TREVS_ERR_INVALID_ARG;
  const size_t bytes = (size_t)n * 4;
  const Span out[] = {{done, bytes}};
  const Span in[] = {{src, bytes}, {dst, bytes}, {n_tokens, n_tokens ? bytes : 0}};
  if (any_overlap(out, 1, in, 3) || meets_cache(c, out[0])) return TREVS_ERR_INVALID_ARG;
  for (const Span& x : in)
    if (meets_cache(c, x)) return TREVS_ERR_INVALID_ARG;
  TREVS_HIP(launch_pages_fork(pages_args(c, n), src, dst, n_tokens, done, reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

trevs_status trevs_pages_free(const trevs_kv8_cache* c, int32_t n, const int32_t* slots, const int32_t* keep,
                              void* stream) {
  TREVS_TRY(validate_list(c, n, slots, false));
  if (!aligned(keep, 4)) return TREVS_ERR_INVALID_ARG;
  if (meets_cache(c, Span{slots, slots ? (size_t)n * 4 : 0}) || meets_cache(c, Span{keep, keep ? (size_t)n * 4 : 0}))
    return TREVS_ERR_INVALID_ARG;
  TREVS_HIP(launch_pages_free(pages_args(c, n), slots, keep, reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

trevs_status trevs_kv8_copy_pages(const trevs_kv8_cache* c, int32_t n, const int32_t* src, const int32_t* dst,
                                  void* stream) {
  TREVS_TRY(validate_cache(c));
  if (n < 1 || !src || !dst || !aligned(src, 4) || !aligned(dst, 4)) return TREVS_ERR_INVALID_ARG;
  if (n > kMaxGroups) return TREVS_ERR_UNSUPPORTED;
  if (meets_cache(c, Span{src, (size_t)n * 4}) || meets_cache(c, Span{dst, (size_t)n * 4}))
    return TREVS_ERR_INVALID_ARG;
  CopyArgs a;
  a.k = c->k;
  a.v = c->v;
  a.k_scale = c->k_scale;
  a.v_scale = c->v_scale;
  a.src = src;
  a.dst = dst;
  a.n = n;
  a.n_layers = c->n_layers;
  a.n_pages = c->n_pages;
  a.H_kv = c->H_kv;
  a.page_bytes = c->H_kv * c->page_tokens * c->d_head;
  TREVS_HIP(launch_kv8_copy(a, reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

trevs_status trevs_kv8_write(const trevs_kv8_cache* c, const trevs_kv8_write_args* a, void* stream) {
  TREVS_TRY(validate_write(c, a));
  const int64_t width = (int64_t)c->H_kv * c->d_head;
  WriteArgs w;
  w.c = layer_view(*c, a->layer);
  w.k = a->k;
  w.v = a->v;
  w.k_ld = a->k_ld ? a->k_ld : width;
  w.v_ld = a->v_ld ? a->v_ld : width;
  w.n_new = a->n_new;
  w.slots = a->slots;
  w.B = a->B;
  w.T_max = a->T_max;
  w.frames = (int)(((int64_t)a->T_max + c->page_tokens - 2) / c->page_tokens + 1);
  TREVS_HIP(launch_kv8_write(w, a->dtype, c->d_head, c->page_tokens, reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

size_t trevs_kv8_attention_workspace_size(const trevs_kv8_cache* c, const trevs_kv8_attention_args* a) {
  if (validate_attention(c, a) != TREVS_OK) return 0;
  return attention_layout(c, a).total;
}

trevs_status trevs_kv8_attention(const trevs_kv8_cache* c, const trevs_kv8_attention_args* a, void* ws,
                                 size_t ws_bytes, void* stream) {
  TREVS_TRY(validate_attention(c, a));
  const AttnLayout L = attention_layout(c, a);
  TREVS_TRY(check_ws(ws, ws_bytes, L.total));
  AttnArgs t = {};
  t.c = layer_view(*c, a->layer);
  t.q = a->q;
  t.q_ld = a->q_ld ? a->q_ld : (int64_t)a->H_q * c->d_head;
  t.q_len = a->q_len;
  t.slots = a->slots;
  t.out = a->out;
  t.lse = a->lse;
  t.B = a->B;
  t.T_max = a->T_max;
  t.H_q = a->H_q;
  t.G = a->H_q / c->H_kv;
  t.causal = a->causal;
  t.kv_max = max_keys(c, a);
  t.page_shift = page_shift(c);
  t.scale_log2e = a->scale * kLog2e;
  t.tile_pieces = reinterpret_cast<int2*>(ws);
  t.part_ml = reinterpret_cast<float2*>(reinterpret_cast<uint8_t*>(ws) + L.part_ml);
  t.part = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(ws) + L.part);
  TREVS_HIP(launch_kv8_attention(t, L.plan, a->dtype, c->d_head, reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

trevs_status trevs_kv8_compact(const trevs_kv8_cache* c, const trevs_kv8_compact_args* a, void* stream) {
  TREVS_TRY(validate_compact(c, a));
  CompactArgs t;
  t.c = layer_view(*c, 0);
  t.kept = a->kept_idx;
  t.src = a->src_slots;
  t.dst = a->dst_slots;
  t.B = a->B;
  t.P = a->P;
  t.K_in = a->K_in;
  t.n_kept = a->n_kept;
  t.n_layers = c->n_layers;
  plan_compact(c, a, &t);
  TREVS_HIP(launch_kv8_compact(t, c->d_head, c->page_tokens, reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

size_t trevs_kv8_weights_workspace_size(const trevs_kv8_cache* c, const trevs_kv8_weights_args* a) {
  if (validate_weights(c, a) != TREVS_OK) return 0;
  return weights_bytes(c, a);
}

trevs_status trevs_kv8_weights(const trevs_kv8_cache* c, const trevs_kv8_weights_args* a, void* ws, size_t ws_bytes,
                               void* stream) {
  TREVS_TRY(validate_weights(c, a));
  TREVS_TRY(check_ws(ws, ws_bytes, weights_bytes(c, a)));
  const WeightsPlan p = plan_of(c, a);
  WeightsArgs t;
  t.c = layer_view(*c, a->layer);
  t.q = a->q;
  t.q_ld = a->q_ld ? a->q_ld : (int64_t)a->H_q * c->d_head;
  t.q_len = a->q_len;
  t.slots = a->slots;
  t.lse = a->lse;
  t.score = a->score;
  t.part = reinterpret_cast<float*>(ws);
  t.B = a->B;
  t.T_max = a->T_max;
  t.H_q = a->H_q;
  t.G = a->H_q / c->H_kv;
  t.causal = a->causal;
  t.kv_max = weights_keys(c, a);
  t.width = c->max_pages * c->page_tokens;
  t.page_shift = page_shift(c);
  t.scale_log2e = a->scale * kLog2e;
  t.decay = a->decay;
  t.key_blocks = p.key_blocks;
  t.heads = p.heads;
  t.head_groups = p.head_groups;
  t.pieces = p.pieces;
  TREVS_HIP(launch_kv8_weights(t, p, a->dtype, c->d_head, reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

size_t trevs_kv8_evict_workspace_size(const trevs_kv8_cache* c, const trevs_kv8_evict_args* a) {
  if (validate_evict(c, a) != TREVS_OK) return 0;
  return evict_info_bytes(a) + align_up((size_t)a->B * c->max_pages * sizeof(int32_t));
}

trevs_status trevs_kv8_evict(const trevs_kv8_cache* c, const trevs_kv8_evict_args* a, void* ws, size_t ws_bytes,
                             void* stream) {
  TREVS_TRY(validate_evict(c, a));
  TREVS_TRY(check_ws(ws, ws_bytes, trevs_kv8_evict_workspace_size(c, a)));
  EvictArgs t;
  t.c = layer_view(*c, 0);
  t.ref = c->ref;
  t.score = a->score;
  t.keep = a->keep;
  t.slots = a->slots;
  t.n_evicted = a->n_evicted;
  t.kept_idx = a->kept_idx;
  t.info = reinterpret_cast<EvictInfo*>(ws);
  t.old = reinterpret_cast<int32_t*>(reinterpret_cast<uint8_t*>(ws) + evict_info_bytes(a));
  t.B = a->B;
  t.n_keep = a->n_keep;
  t.n_first = a->n_first;
  t.n_last = a->n_last;
  t.n_layers = c->n_layers;
  t.page_shift = page_shift(c);
  // a workgroup for every block that the kept tokens can fill, or as many as a launch holds, taken in turns
  const int64_t each = (int64_t)c->n_layers * a->B * c->H_kv, page = c->page_tokens;
  const int64_t blocks = std::min(((int64_t)a->n_keep + page - 1) / page, (int64_t)c->max_pages);
  t.frames = (int)std::min(blocks, (kMaxGroups - a->B) / each);
  t.turns = t.frames < blocks;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  TREVS_HIP(launch_evict_select(t, s));
  TREVS_HIP(launch_evict_pages(t, s));
  TREVS_HIP(launch_kv8_evict(t, c->d_head, c->page_tokens, s));
  return TREVS_OK;
}

trevs_status trevs_pages_reorder(const trevs_kv8_cache* c, int32_t n_groups, int32_t W, const int32_t* slots,
                                 const int32_t* parent, float* score, void* stream) {
  TREVS_TRY(validate_cache(c));
  if (n_groups < 1 || W < 1 || !parent) return TREVS_ERR_INVALID_ARG;
  if (!aligned(slots, 4) || !aligned(parent, 4) || !aligned(score, 4)) return TREVS_ERR_INVALID_ARG;
  const int64_t n = (int64_t)n_groups * W;
  if (!slots && n > c->n_slots) return TREVS_ERR_INVALID_ARG;
  if (W > TREVS_MAX_BEAMS || n > TREVS_MAX_PAGE_REQUESTS) return TREVS_ERR_UNSUPPORTED;
  const Span in[] = {{slots, slots ? (size_t)n * 4 : 0}, {parent, (size_t)n * 4}};
  const Span out{score, score ? score_bytes(c) : 0};
  if (any_overlap(&out, 1, in, 2) || meets_cache(c, out) || meets_cache(c, in[0]) || meets_cache(c, in[1]))
    return TREVS_ERR_INVALID_ARG;
  TREVS_HIP(launch_pages_reorder(pages_args(c, (int)n), n_groups, W, slots, parent, score,
                                 reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

size_t trevs_beam_select_workspace_size(const trevs_beam_select_args* a) {
  if (validate_beam(a) != TREVS_OK) return 0;
  return beam_part_bytes(a) + align_up((size_t)a->B * a->W * beam_chunks(a) * beam_stride(a->n_out) * sizeof(uint64_t));
}

trevs_status trevs_beam_select(const trevs_beam_select_args* a, void* ws, size_t ws_bytes, void* stream) {
  TREVS_TRY(validate_beam(a));
  TREVS_TRY(check_ws(ws, ws_bytes, trevs_beam_select_workspace_size(a)));
  BeamArgs t;
  t.logits = a->logits;
  t.ld = a->logits_ld ? a->logits_ld : a->V;
  t.score = a->score;
  t.done = a->done;
  t.score_out = a->score_out;
  t.parent = a->parent;
  t.token = a->token;
  t.part = reinterpret_cast<float2*>(ws);
  t.cand = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(ws) + beam_part_bytes(a));
  t.B = a->B;
  t.W = a->W;
  t.V = a->V;
  t.n = a->n_out;
  t.eos = a->eos;
  t.chunks = beam_chunks(a);
  t.stride = beam_stride(a->n_out);
  TREVS_HIP(launch_beam_select(t, a->dtype, reinterpret_cast<hipStream_t>(stream)));
  return TREVS_OK;
}

}  // extern "C"
