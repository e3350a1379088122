// The paged cache of fp32, bf16 or e4m3 numbers as its kernels see it, and the conversions (include/laq_cache.h has the format).
#pragma once

#include "laq_cache.h"
#include "laq_internal.h"

namespace laq {

struct E4m3 { uint8_t x; };              // a number of a cache in 8 bits

struct PagedPlane {                      // K or V
  void* x;
  uint8_t* scales;
};
struct PagedView {
  PagedPlane k, v;
  int32_t n_blocks, block_rows, Hkv, d, type;
  int64_t block, head, row;              // elements
};

// Rows of tokens.
struct TokenHeads {
  void* x;
  int32_t heads;
  int64_t token, head;                   // elements
};

struct RopeArgs {
  const float* inv_freq;
  const int32_t* positions;
  int32_t rot, interleaved;
  float mscale;
};

// Scale byte of a row in 8 bits from the bits of its largest magnitude (fp32; an infinity or a NaN: the largest bits).  What is added carries into
// the exponent above 1.75.
__device__ __forceinline__ uint32_t e4m3_scale_of(uint32_t most) {
  const int e = (int)((most + 0x1fffffu) >> 23) - 8;
  return most >= 0x7f800000u ? 255u : (uint32_t)max(e, 27);
}
// 255 is an infinity here, which makes a NaN of the zeros that stand with it.
__device__ __forceinline__ float e4m3_scale_value(uint32_t s) { return __uint_as_float(s ? s << 23 : 0x400000u); }

// Where a slot lies: false if it is none of the cache.
__device__ __forceinline__ bool paged_slot(const PagedView& c, int slot, int* block, int* row) {
  *block = (int)((uint32_t)slot / (uint32_t)c.block_rows);
  *row = slot - *block * c.block_rows;
  return slot >= 0 && *block < c.n_blocks;
}

// Checks a cache and fills in the strides of a dense one.  LAQ_OK or LAQ_ERR_INVALID.  need_k / need_v: the call touches that plane.
int paged_view(const laq_cache* cache, bool need_k, bool need_v, PagedView* view);

// q, k (and v) of tokens: q to q_out, k and v to the cache, or k to k_out where there is none.
struct TokenCall {
  int64_t n_tokens;
  int32_t d;
  TokenHeads q, k, v, q_out, k_out;      // x null: none
  const int32_t* slots;
  RopeArgs rope;                         // inv_freq null: none
};
hipError_t launch_token_rows(const TokenCall& t, int dtype, const PagedView* cache, hipStream_t st);
// instances inst0 .. inst0 + n - 1, `most` rows of a KV head at most
hipError_t launch_paged_compact(const PagedView& c, int dtype, int n, int inst0, int most, int L, const KvLayout& lay, const InstTable& tab,
                                const void* k, const void* v, const int32_t* idx, const int32_t* slots, hipStream_t st);
hipError_t launch_paged_load(const PagedView& c, int dtype, int64_t n_tokens, const int32_t* slots, void* k, void* v, hipStream_t st);

// A call of laq_cache_attention.
struct PagedAttention {
  int32_t Hq, n, blocks_per_inst, max_rows;
  float scale2;                          // scale * log2(e)
  int64_t n_tokens;
  TokenHeads q;
  const int32_t *start, *table, *rows;
  void* out;
  float* lse;
};
size_t paged_attention_bytes(const PagedView& c, int Hq, int dtype, int n, int64_t n_tokens, int max_rows);
bool paged_attention_fits(const PagedView& c, int dtype, const PagedAttention& a, bool cut);      // in a launch
hipError_t launch_paged_attention(const PagedView& c, int dtype, const PagedAttention& a, void* ws, hipStream_t st);

}  // namespace laq
