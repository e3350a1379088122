// C ABI of the paged 4-bit cache (declared in include/laq_fp4.h): argument checks and dispatch.
#include <math.h>

#include "laq_fp4_codes.h"

namespace laq {

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
constexpr int64_t MOST_ROWS = 0x7fffffff;
constexpr int32_t MOST_HEADS = 32768;

int fp4_view(const laq_fp4_cache* cache, bool need_k, bool need_v, Fp4View* view) {
  if (!cache) return LAQ_ERR_INVALID;
  const laq_fp4_cache& c = *cache;
  if (c.n_blocks < 1 || c.Hkv < 1 || c.Hkv > MOST_HEADS || c.block_rows < 16 || c.block_rows % 16) return LAQ_ERR_INVALID;
  if (c.d < 32 || c.d > 256 || c.d % 32) return LAQ_ERR_INVALID;
  if ((int64_t)c.n_blocks * c.block_rows > MOST_ROWS) return LAQ_ERR_INVALID;
  if ((need_k && (!c.k || !c.k_scale)) || (need_v && (!c.v || !c.v_scale))) return LAQ_ERR_INVALID;
  if ((need_k && !aligned16(c.k)) || (need_v && !aligned16(c.v))) return LAQ_ERR_INVALID;
  const int64_t given[6] = {c.stride_block, c.stride_head, c.stride_row, c.scale_stride_block, c.scale_stride_head, c.scale_stride_row};
  int zeros = 0;
  for (int64_t s : given) {
    if (s < 0) return LAQ_ERR_INVALID;
    zeros += s == 0;
  }
  *view = Fp4View{{c.k, c.k_scale}, {c.v, c.v_scale}, c.n_blocks, c.block_rows, c.Hkv, c.d,
                  given[0], given[1], given[2], given[3], given[4], given[5]};
  if (zeros == 6) {
    view->row = c.d / 2;
    view->head = view->row * c.block_rows;
    view->block = view->head * c.Hkv;
    view->scale_row = c.d / 32;
    view->scale_head = view->scale_row * c.block_rows;
    view->scale_block = view->scale_head * c.Hkv;
  } else if (zeros) {
    return LAQ_ERR_INVALID;
  }
  if (view->block > 0xffffffffLL || view->scale_block > 0xffffffffLL) return LAQ_ERR_INVALID;
  if (view->row > (1 << 27) || view->scale_row > (1 << 27)) return LAQ_ERR_INVALID;      // (16 rows are addressed with 32 bits)
  if (view->row < c.d / 2 || view->scale_row < c.d / 32 || (view->block | view->head | view->row) % 16) return LAQ_ERR_INVALID;
  return LAQ_OK;
}

// Strides of [n_tokens, heads, d] tensors: dense where both are zero.
static int token_strides(int heads, int d, int dtype, int64_t* token, int64_t* head) {
  if (dtype != LAQ_F32 && dtype != LAQ_BF16) return LAQ_ERR_INVALID;
  if (*token == 0 && *head == 0) {
    *head = d;
    *token = (int64_t)heads * d;
    return LAQ_OK;
  }
  const int per16 = dtype == LAQ_F32 ? 4 : 8;
  return *token < 1 || *head < 1 || *token % per16 || *head % per16 ? LAQ_ERR_INVALID : LAQ_OK;
}

static int done(hipError_t e) { return e == hipSuccess ? LAQ_OK : LAQ_ERR_DEVICE; }
// Threads that one launch may have in a dimension: the row kernels have one for eight numbers.
constexpr int64_t MOST_PIECES = 0xffffff00;

static int block_map_impl(int32_t n, int32_t block_rows, int32_t n_blocks, int32_t width, const int32_t* add, int32_t* rows, int32_t* table,
                          int32_t* list, int32_t* state, int32_t* start, int32_t* slots, int64_t n_slots, hipStream_t st) {
  if (n < 1 || block_rows < 16 || block_rows % 16 || n_blocks < 1 || width < 1 || n_slots < 0) return LAQ_ERR_INVALID;
  if ((int64_t)n_blocks * block_rows > MOST_ROWS || (int64_t)width * block_rows > MOST_ROWS || n_slots > MOST_ROWS) return LAQ_ERR_INVALID;
  if ((int64_t)n * width > MOST_ROWS) return LAQ_ERR_UNSUPPORTED;
  if (!add || !rows || !table || !list || !state || (!slots && n_slots)) return LAQ_ERR_INVALID;
  return done(launch_block_map(n, block_rows, n_blocks, width, add, rows, table, list, state, start, slots, n_slots, st));
}

static int store_impl(const laq_fp4_cache* cache, int32_t dtype, int64_t n_tokens, const void* k, const void* v, int64_t stride_token,
                      int64_t stride_head, const int32_t* slots, hipStream_t st) {
  Fp4View c;
  if (fp4_view(cache, k != nullptr, v != nullptr, &c) != LAQ_OK) return LAQ_ERR_INVALID;
  if (n_tokens < 0 || token_strides(c.Hkv, c.d, dtype, &stride_token, &stride_head) != LAQ_OK) return LAQ_ERR_INVALID;
  if (n_tokens == 0) return LAQ_OK;      // (the addresses of tensors without elements are NULL)
  if ((!k && !v) || !aligned16(k) || !aligned16(v) || !slots) return LAQ_ERR_INVALID;
  if (n_tokens > MOST_PIECES / c.Hkv / (c.d / 8)) return LAQ_ERR_UNSUPPORTED;
  return done(launch_fp4_store(c, dtype, n_tokens, k, v, stride_token, stride_head, slots, st));
}

static int load_impl(const laq_fp4_cache* cache, int32_t dtype, int64_t n_tokens, const int32_t* slots, void* k, void* v, hipStream_t st) {
  Fp4View c;
  if (fp4_view(cache, k != nullptr, v != nullptr, &c) != LAQ_OK) return LAQ_ERR_INVALID;
  if (n_tokens < 0 || (dtype != LAQ_F32 && dtype != LAQ_BF16)) return LAQ_ERR_INVALID;
  if (n_tokens == 0) return LAQ_OK;
  if ((!k && !v) || !aligned16(k) || !aligned16(v) || !slots) return LAQ_ERR_INVALID;
  if (n_tokens > MOST_PIECES / c.Hkv / (c.d / 8)) return LAQ_ERR_UNSUPPORTED;
  return done(launch_fp4_load(c, dtype, n_tokens, slots, k, v, st));
}

static int fp4_compact_impl(const laq_shape* shape, const void* k, const void* v, const int32_t* idx, const int32_t* budget,
                            const laq_fp4_cache* cache, const int32_t* slots, hipStream_t st) {
  ScoreGeom g;
  KvLayout lay;
  const int rc = check_source(shape, budget, &g, &lay);
  if (rc != LAQ_OK) return rc;
  Fp4View c;
  if (fp4_view(cache, true, v != nullptr, &c) != LAQ_OK || c.Hkv != g.Hkv || c.d != g.d) return LAQ_ERR_INVALID;
  if (!k || !idx || !slots || !aligned16(k) || !aligned16(v)) return LAQ_ERR_INVALID;
  int64_t row = 0;
  for (int i = 0; i < g.n_inst; ++i)
    if ((int64_t)(budget[i] < g.L ? budget[i] : g.L) > MOST_PIECES / 32 / g.Hkv) return LAQ_ERR_UNSUPPORTED;
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
    if (launch_fp4_compact(c, shape->dtype, n, i0, most, g.L, lay, tab, k, v, idx, slots, st) != hipSuccess) return LAQ_ERR_DEVICE;
  }
  return LAQ_OK;
}

static bool attention_sizes_ok(const Fp4View& c, int32_t Hq, int32_t dtype, int32_t n, int64_t n_tokens, int32_t max_rows) {
  return Hq >= 1 && Hq % c.Hkv == 0 && Hq <= 65535 && (dtype == LAQ_F32 || dtype == LAQ_BF16) && n >= 1 && n_tokens >= 0 &&
         n_tokens <= MOST_ROWS / Hq && max_rows >= 1;
}

static int attention_impl(const laq_fp4_cache* cache, int32_t Hq, int32_t dtype, float scale, int32_t n, int64_t n_tokens, const int32_t* start,
                          const void* q, int64_t stride_token, int64_t stride_head, const int32_t* table, int32_t width, const int32_t* rows,
                          int32_t max_rows, void* out, float* lse, void* ws, size_t ws_bytes, hipStream_t st) {
  Fp4View c;
  if (fp4_view(cache, true, true, &c) != LAQ_OK || !attention_sizes_ok(c, Hq, dtype, n, n_tokens, max_rows)) return LAQ_ERR_INVALID;
  if (width < 1 || (int64_t)width * c.block_rows > MOST_ROWS || max_rows > width * c.block_rows) return LAQ_ERR_INVALID;
  if (!(scale == scale) || isinf(scale) || (!start && n_tokens != n)) return LAQ_ERR_INVALID;
  if (token_strides(Hq, c.d, dtype, &stride_token, &stride_head) != LAQ_OK) return LAQ_ERR_INVALID;
  if (n_tokens == 0) return LAQ_OK;
  if (!q || !table || !rows || !out || !aligned16(q) || !aligned16(out)) return LAQ_ERR_INVALID;
  if (ws && (ws_bytes < fp4_attention_bytes(c, Hq, dtype, n, n_tokens, max_rows) || !aligned16(ws))) return LAQ_ERR_WORKSPACE;
  const float s = scale > 0.f ? scale : 1.0f / sqrtf((float)c.d);
  const Fp4Attention a{Hq, n, width, max_rows, s * 1.44269504088896340736f, n_tokens, stride_token, stride_head, start, table, rows, q, out, lse};
  if (!fp4_attention_fits(c, dtype, a, ws)) return LAQ_ERR_UNSUPPORTED;
  return done(launch_fp4_attention(c, dtype, a, ws, st));
}

}  // namespace laq

extern "C" {

int laq_block_map(int32_t n, int32_t block_rows, int32_t n_blocks, int32_t blocks_per_inst, const int32_t* add, int32_t* rows,
                  int32_t* block_table, int32_t* free_blocks, int32_t* state, int32_t* start, int32_t* slots, int64_t n_slots, void* stream) {
  return laq::block_map_impl(n, block_rows, n_blocks, blocks_per_inst, add, rows, block_table, free_blocks, state, start, slots, n_slots,
                             static_cast<hipStream_t>(stream));
}

int laq_fp4_store(const laq_fp4_cache* cache, int32_t dtype, int64_t n_tokens, const void* k, const void* v, int64_t stride_token,
                  int64_t stride_head, const int32_t* slots, void* stream) {
  return laq::store_impl(cache, dtype, n_tokens, k, v, stride_token, stride_head, slots, static_cast<hipStream_t>(stream));
}

int laq_fp4_compact(const laq_shape* shape, const void* k, const void* v, const int32_t* idx, const int32_t* budget,
                    const laq_fp4_cache* cache, const int32_t* slots, void* stream) {
  return laq::fp4_compact_impl(shape, k, v, idx, budget, cache, slots, static_cast<hipStream_t>(stream));
}

int laq_fp4_load(const laq_fp4_cache* cache, int32_t dtype, int64_t n_tokens, const int32_t* slots, void* k, void* v, void* stream) {
  return laq::load_impl(cache, dtype, n_tokens, slots, k, v, static_cast<hipStream_t>(stream));
}

size_t laq_fp4_attention_workspace_bytes(const laq_fp4_cache* cache, int32_t Hq, int32_t dtype, int32_t n, int64_t n_tokens,
                                         int32_t max_rows) {
  laq::Fp4View c;
  if (laq::fp4_view(cache, false, false, &c) != LAQ_OK || !laq::attention_sizes_ok(c, Hq, dtype, n, n_tokens, max_rows)) return 0;
  return laq::fp4_attention_bytes(c, Hq, dtype, n, n_tokens, max_rows);
}

int laq_fp4_attention(const laq_fp4_cache* cache, int32_t Hq, int32_t dtype, float scale, int32_t n, int64_t n_tokens,
                      const int32_t* start, const void* q, int64_t stride_token, int64_t stride_head, const int32_t* block_table,
                      int32_t blocks_per_inst, const int32_t* rows, int32_t max_rows, void* out, float* lse, void* ws, size_t ws_bytes,
                      void* stream) {
  return laq::attention_impl(cache, Hq, dtype, scale, n, n_tokens, start, q, stride_token, stride_head, block_table, blocks_per_inst, rows,
                             max_rows, out, lse, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

}  // extern "C"
