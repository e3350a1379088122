// The paged cache of fp32, bf16 or e4m3 numbers as its kernels see it, and the conversions (include/laq_cache.h has the format).
#pragma once

#include "laq_cache.h"
#include "laq_internal.h"

namespace laq {

struct E4m3 { uint8_t x; };              // a number of a cache in 8 bits

constexpr int COMPUTE_UNITS = 256;

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
// How the launch is cut, from what the host knows.
struct AttPlan {
  int32_t tile;                          // score rows of a column
  int32_t columns;                       // columns of a KV head over all requests, at most
  int32_t shares;                        // workgroups that share all keys of all columns out evenly; 0: one workgroup a column
};

// The ranges of columns that several workgroups share.  A workgroup has two places: 2w for a column that began in another workgroup's share, 2w + 1 for one
// that begins in its own and goes on; a place has mz[tile] (m and z), sums[tile][d] and a mark.  A workgroup that is done with a range writes the launch's nonce
// there, after its sums have arrived, and then looks at the marks of all ranges of the column: who finds all of them joins the ranges, in their order, and
// clears the marks, so that a replayed launch, whose nonce is the same, finds none of its own.  The workspace comes as the allocator left it: one of its words passes for a
// launch's mark once in 2^64 (laq_marks.h).  Two may find all of them (both write the same); one that comes to look when another has begun to clear finds that it is not
// needed.  (Counting in by compare and swap: 64 workgroups of a column take turns, one request of 32768 rows x 8 heads 61 us.)
struct Partials {
  unsigned long long* marks;
  float2* mz;
  float* sums;
  unsigned long long nonce;
};

// chunks of a prompt: whether that kernel takes a call, and the call
bool paged_prompt_call(const PagedView& c, int Hq, int dtype, int n, int64_t n_tokens);
hipError_t launch_paged_prompt(const PagedView& c, const PagedAttention& a, hipStream_t st);
size_t paged_attention_bytes(const PagedView& c, int Hq, int dtype, int n, int64_t n_tokens, int max_rows);
bool paged_attention_fits(const PagedView& c, int dtype, const PagedAttention& a, bool cut);      // in a launch
hipError_t launch_paged_attention(const PagedView& c, int dtype, const PagedAttention& a, void* ws, hipStream_t st);

}  // namespace laq
