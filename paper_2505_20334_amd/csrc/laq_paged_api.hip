// C ABI of rotary positions and the paged cache in 32, 16 or 8 bits (declared in include/laq_cache.h): argument checks and dispatch.
#include <math.h>

#include "laq_paged.h"

namespace laq {

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
constexpr int64_t MOST_ROWS = 0x7fffffff;
constexpr int32_t MOST_HEADS = 32768;
// A launch has less than 2^32 threads in a dimension: 64 a token at most, 32 a row.
constexpr int64_t MOST_TOKENS = 1 << 25, MOST_LISTED = 1 << 26;

int paged_view(const laq_cache* cache, bool need_k, bool need_v, PagedView* view) {
  if (!cache) return LAQ_ERR_INVALID;
  const laq_cache& c = *cache;
  if (c.n_blocks < 1 || c.Hkv < 1 || c.Hkv > MOST_HEADS || c.block_rows < 16 || c.block_rows % 16) return LAQ_ERR_INVALID;
  if (c.d < 8 || c.d > 256 || c.d % 8 || c.type < LAQ_F32 || c.type > LAQ_E4M3) return LAQ_ERR_INVALID;
  if ((int64_t)c.n_blocks * c.block_rows > MOST_ROWS) return LAQ_ERR_INVALID;
  if ((need_k && (!c.k || !aligned16(c.k))) || (need_v && (!c.v || !aligned16(c.v)))) return LAQ_ERR_INVALID;
  const bool scaled = c.type == LAQ_E4M3;
  if (scaled && ((need_k && (!c.k_scale || !aligned16(c.k_scale))) || (need_v && (!c.v_scale || !aligned16(c.v_scale))))) return LAQ_ERR_INVALID;
  *view = PagedView{{c.k, scaled ? c.k_scale : nullptr}, {c.v, scaled ? c.v_scale : nullptr}, c.n_blocks, c.block_rows, c.Hkv, c.d, c.type,
                    c.stride_block, c.stride_head, c.stride_row};
  if (c.stride_block == 0 && c.stride_head == 0 && c.stride_row == 0) {
    view->row = c.d;
    view->head = view->row * c.block_rows;
    view->block = view->head * c.Hkv;
  }
  if (view->block < 1 || view->head < 1 || view->row < c.d || view->row > (1 << 24)) return LAQ_ERR_INVALID;
  // (the last row's place is a number of 64 bits)
  if (view->block > (1LL << 60) / c.n_blocks || view->head > (1LL << 60) / c.Hkv) return LAQ_ERR_INVALID;
  return (view->block | view->head | view->row) % 8 ? LAQ_ERR_INVALID : LAQ_OK;
}

// Rows of tokens: LAQ_OK with the strides filled in (no rows: x null), or LAQ_ERR_INVALID.
static int token_heads(const laq_heads* h, int d, int dtype, int64_t n_tokens, TokenHeads* out) {
  *out = TokenHeads{nullptr, 0, 0, 0};
  if (dtype != LAQ_F32 && dtype != LAQ_BF16) return LAQ_ERR_INVALID;
  if (!h || !h->x) return LAQ_OK;
  if (h->heads < 1 || h->heads > 65535 || !aligned16(h->x)) return LAQ_ERR_INVALID;
  *out = TokenHeads{h->x, h->heads, h->stride_token, h->stride_head};
  if (h->stride_token == 0 && h->stride_head == 0) {
    out->head = d;
    out->token = (int64_t)h->heads * d;
    return LAQ_OK;
  }
  const int per16 = dtype == LAQ_F32 ? 4 : 8;
  // (one token or one head: its stride is never used, and a view of one may have any)
  if (h->stride_token < 0 || h->stride_head < 0 || (h->stride_token < 1 && n_tokens > 1) || (h->stride_head < 1 && h->heads > 1)) return LAQ_ERR_INVALID;
  if (h->stride_token > (1LL << 60) / (n_tokens + 1) || h->stride_head > (1LL << 60) / h->heads) return LAQ_ERR_INVALID;
  return h->stride_token % per16 || h->stride_head % per16 ? LAQ_ERR_INVALID : LAQ_OK;
}

static int rope_args(const laq_rope_plan* rope, int d, const int32_t* positions, RopeArgs* out) {
  if (rope->rot < 2 || rope->rot > d || rope->rot % 2 || (rope->layout != LAQ_ROPE_HALF && rope->layout != LAQ_ROPE_INTERLEAVED)) return LAQ_ERR_INVALID;
  if (!rope->inv_freq || !(rope->mscale == rope->mscale) || isinf(rope->mscale)) return LAQ_ERR_INVALID;
  *out = RopeArgs{rope->inv_freq, positions, rope->rot, rope->layout == LAQ_ROPE_INTERLEAVED, rope->mscale};
  return LAQ_OK;
}

// An output of rotated heads beside its input.
static bool out_fits(const TokenHeads& x, const TokenHeads& out) { return (x.x != nullptr) == (out.x != nullptr) && x.heads == out.heads; }

static int done(hipError_t e) { return e == hipSuccess ? LAQ_OK : LAQ_ERR_DEVICE; }

static int rope_impl(const laq_rope_plan* rope, int32_t dtype, int64_t n_tokens, int32_t d, const laq_heads* q, const laq_heads* k,
                     const int32_t* positions, const laq_heads* q_out, const laq_heads* k_out, hipStream_t st) {
  TokenCall t{};
  t.n_tokens = n_tokens;
  t.d = d;
  if (n_tokens < 0 || d < 8 || d > 256 || d % 8 || !rope || rope_args(rope, d, positions, &t.rope) != LAQ_OK) return LAQ_ERR_INVALID;
  if (token_heads(q, d, dtype, n_tokens, &t.q) || token_heads(k, d, dtype, n_tokens, &t.k) || token_heads(q_out, d, dtype, n_tokens, &t.q_out) ||
      token_heads(k_out, d, dtype, n_tokens, &t.k_out))
    return LAQ_ERR_INVALID;
  if (n_tokens == 0) return LAQ_OK;      // (the addresses of tensors without elements are NULL)
  if (!positions || (!t.q.x && !t.k.x) || !out_fits(t.q, t.q_out) || !out_fits(t.k, t.k_out)) return LAQ_ERR_INVALID;
  if (n_tokens > MOST_TOKENS) return LAQ_ERR_UNSUPPORTED;
  return done(launch_token_rows(t, dtype, nullptr, st));
}

static int append_impl(const laq_cache* cache, int32_t dtype, int64_t n_tokens, const laq_heads* k, const laq_heads* v, const int32_t* slots,
                       const laq_rope_plan* rope, const int32_t* positions, const laq_heads* q, const laq_heads* q_out, hipStream_t st) {
  TokenCall t{};
  PagedView c;
  const bool has_k = k && k->x, has_v = v && v->x, has_q = q && q->x;
  if (paged_view(cache, has_k, has_v, &c) != LAQ_OK || n_tokens < 0) return LAQ_ERR_INVALID;
  t.n_tokens = n_tokens;
  t.d = c.d;
  t.slots = slots;
  if (rope && rope_args(rope, c.d, positions, &t.rope) != LAQ_OK) return LAQ_ERR_INVALID;
  if (token_heads(q, c.d, dtype, n_tokens, &t.q) || token_heads(k, c.d, dtype, n_tokens, &t.k) || token_heads(v, c.d, dtype, n_tokens, &t.v) ||
      token_heads(q_out, c.d, dtype, n_tokens, &t.q_out))
    return LAQ_ERR_INVALID;
  if (n_tokens == 0) return LAQ_OK;
  if ((!has_k && !has_v) || !slots || (has_k && t.k.heads != c.Hkv) || (has_v && t.v.heads != c.Hkv)) return LAQ_ERR_INVALID;
  if (rope ? !positions || !out_fits(t.q, t.q_out) : has_q) return LAQ_ERR_INVALID;
  if (n_tokens > MOST_TOKENS) return LAQ_ERR_UNSUPPORTED;
  return done(launch_token_rows(t, dtype, &c, st));
}

static int paged_compact_impl(const laq_shape* shape, const void* k, const void* v, const int32_t* idx, const int32_t* budget,
                              const laq_cache* cache, const int32_t* slots, hipStream_t st) {
  ScoreGeom g;
  KvLayout lay;
  const int rc = check_source(shape, budget, &g, &lay);
  if (rc != LAQ_OK) return rc;
  PagedView c;
  if (paged_view(cache, true, v != nullptr, &c) != LAQ_OK || c.Hkv != g.Hkv || c.d != g.d) return LAQ_ERR_INVALID;
  if (!k || !idx || !slots || !aligned16(k) || !aligned16(v)) return LAQ_ERR_INVALID;
  int64_t row = 0;
  for (int i = 0; i < g.n_inst; ++i)
    if ((budget[i] < g.L ? budget[i] : g.L) > MOST_LISTED) return LAQ_ERR_UNSUPPORTED;
  for (int i0 = 0; i0 < g.n_inst; i0 += MAX_INST_PER_LAUNCH) {
    const int n = g.n_inst - i0 < MAX_INST_PER_LAUNCH ? g.n_inst - i0 : MAX_INST_PER_LAUNCH;
    InstTable tab;
    int most = 0;
    for (int i = 0; i < n; ++i) {
      tab.bk[i] = budget[i0 + i] < g.L ? budget[i0 + i] : g.L;
      tab.row0[i] = row;
      row += (int64_t)g.Hkv * tab.bk[i];
      if (tab.bk[i] > most) most = tab.bk[i];
    }
    if (launch_paged_compact(c, shape->dtype, n, i0, most, g.L, lay, tab, k, v, idx, slots, st) != hipSuccess) return LAQ_ERR_DEVICE;
  }
  return LAQ_OK;
}

static int load_impl(const laq_cache* cache, int32_t dtype, int64_t n_tokens, const int32_t* slots, void* k, void* v, hipStream_t st) {
  PagedView c;
  if (paged_view(cache, k != nullptr, v != nullptr, &c) != LAQ_OK) return LAQ_ERR_INVALID;
  if (n_tokens < 0 || (dtype != LAQ_F32 && dtype != LAQ_BF16)) return LAQ_ERR_INVALID;
  if (n_tokens == 0) return LAQ_OK;
  if ((!k && !v) || !aligned16(k) || !aligned16(v) || !slots) return LAQ_ERR_INVALID;
  if (n_tokens > MOST_LISTED / c.Hkv) return LAQ_ERR_UNSUPPORTED;
  return done(launch_paged_load(c, dtype, n_tokens, slots, k, v, st));
}

static bool attention_sizes_ok(const PagedView& c, int32_t Hq, int32_t dtype, int32_t n, int64_t n_tokens, int32_t max_rows) {
  return Hq >= 1 && Hq % c.Hkv == 0 && Hq <= 65535 && (dtype == LAQ_F32 || dtype == LAQ_BF16) && n >= 1 && n_tokens >= 0 &&
         n_tokens <= MOST_ROWS / Hq && max_rows >= 1;
}

static int attention_impl(const laq_cache* cache, int32_t dtype, float scale, int32_t n, int64_t n_tokens, const int32_t* start, const laq_heads* q,
                          const int32_t* table, int32_t width, const int32_t* rows, int32_t max_rows, void* out, float* lse, void* ws,
                          size_t ws_bytes, hipStream_t st) {
  PagedView c;
  if (!q || paged_view(cache, true, true, &c) != LAQ_OK || !attention_sizes_ok(c, q->heads, dtype, n, n_tokens, max_rows)) return LAQ_ERR_INVALID;
  if (width < 1 || (int64_t)width * c.block_rows > MOST_ROWS || max_rows > width * c.block_rows) return LAQ_ERR_INVALID;
  if (!(scale == scale) || isinf(scale) || (!start && n_tokens != n)) return LAQ_ERR_INVALID;
  TokenHeads t;
  if (token_heads(q, c.d, dtype, n_tokens, &t) != LAQ_OK) return LAQ_ERR_INVALID;
  if (n_tokens == 0) return LAQ_OK;
  if (!t.x || !table || !rows || !out || !aligned16(out)) return LAQ_ERR_INVALID;
  if (dtype == LAQ_BF16 && c.type == LAQ_F32) return LAQ_ERR_UNSUPPORTED;
  if (ws && (ws_bytes < paged_attention_bytes(c, q->heads, dtype, n, n_tokens, max_rows) || !aligned16(ws))) return LAQ_ERR_WORKSPACE;
  const float s = scale > 0.f ? scale : 1.0f / sqrtf((float)c.d);
  const PagedAttention a{q->heads, n, width, max_rows, s * 1.44269504088896340736f, n_tokens, t, start, table, rows, out, lse};
  if (!paged_attention_fits(c, dtype, a, ws)) return LAQ_ERR_UNSUPPORTED;
  return done(launch_paged_attention(c, dtype, a, ws, st));
}

}  // namespace laq

extern "C" {

int laq_rope(const laq_rope_plan* rope, int32_t dtype, int64_t n_tokens, int32_t d, const laq_heads* q, const laq_heads* k, const int32_t* positions,
             const laq_heads* q_out, const laq_heads* k_out, void* stream) {
  return laq::rope_impl(rope, dtype, n_tokens, d, q, k, positions, q_out, k_out, static_cast<hipStream_t>(stream));
}

int laq_cache_append(const laq_cache* cache, int32_t dtype, int64_t n_tokens, const laq_heads* k, const laq_heads* v, const int32_t* slots,
                     const laq_rope_plan* rope, const int32_t* positions, const laq_heads* q, const laq_heads* q_out, void* stream) {
  return laq::append_impl(cache, dtype, n_tokens, k, v, slots, rope, positions, q, q_out, static_cast<hipStream_t>(stream));
}

int laq_cache_compact(const laq_shape* shape, const void* k, const void* v, const int32_t* idx, const int32_t* budget, const laq_cache* cache,
                      const int32_t* slots, void* stream) {
  return laq::paged_compact_impl(shape, k, v, idx, budget, cache, slots, static_cast<hipStream_t>(stream));
}

int laq_cache_load(const laq_cache* cache, int32_t dtype, int64_t n_tokens, const int32_t* slots, void* k, void* v, void* stream) {
  return laq::load_impl(cache, dtype, n_tokens, slots, k, v, static_cast<hipStream_t>(stream));
}

size_t laq_cache_attention_workspace_bytes(const laq_cache* cache, int32_t Hq, int32_t dtype, int32_t n, int64_t n_tokens, int32_t max_rows) {
  laq::PagedView c;
  if (laq::paged_view(cache, false, false, &c) != LAQ_OK || !laq::attention_sizes_ok(c, Hq, dtype, n, n_tokens, max_rows)) return 0;
  return laq::paged_attention_bytes(c, Hq, dtype, n, n_tokens, max_rows);
}

int laq_cache_attention(const laq_cache* cache, int32_t dtype, float scale, int32_t n, int64_t n_tokens, const int32_t* start, const laq_heads* q,
                        const int32_t* block_table, int32_t blocks_per_inst, const int32_t* rows, int32_t max_rows, void* out, float* lse,
                        void* ws, size_t ws_bytes, void* stream) {
  return laq::attention_impl(cache, dtype, scale, n, n_tokens, start, q, block_table, blocks_per_inst, rows, max_rows, out, lse, ws, ws_bytes,
                             static_cast<hipStream_t>(stream));
}

}  // extern "C"
