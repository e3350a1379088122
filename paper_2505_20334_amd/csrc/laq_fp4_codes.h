// The 4-bit cache as its kernels see it, and the two conversions (include/laq_fp4.h has the format).
//
// The matrix cores' number formats include this one, and gfx950 converts two numbers per instruction with the scale applied: codes to
// bf16 (exact: two bits of fraction and a power of two) and bf16 or fp32 to codes (to the nearest, ties to even, the largest code at most).
// A conversion has the rate of an fp32 multiplication.
#pragma once

#include "laq_fp4.h"
#include "laq_internal.h"

namespace laq {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct Fp4Plane {                        // K or V
  uint8_t *codes, *scales;
};
struct Fp4View {
  Fp4Plane k, v;
  int32_t n_blocks, block_rows, Hkv, d;
  int64_t block, head, row;              // bytes
  int64_t scale_block, scale_head, scale_row;
};

// Scale byte of a block from the bits of its largest magnitude (fp32; an infinity or a NaN: the largest bits).  Adding a quarter of the
// mantissa's range carries into the exponent from 1.75 on.
__device__ __forceinline__ uint32_t fp4_scale_of(uint32_t most) {
  const int e = (int)((most + 0x200000u) >> 23) - 2;
  return most >= 0x7f800000u ? 255u : (uint32_t)min(max(e, 27), 252);
}
__device__ __forceinline__ float fp4_scale_value(uint32_t s) { return __uint_as_float(s << 23); }

// Eight codes as bf16, in pairs.
__device__ __forceinline__ uint4 fp4_to_bf16(uint32_t codes, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return r;
}

// Where a slot lies: false if it is none of the cache.
__device__ __forceinline__ bool fp4_slot(const Fp4View& c, int slot, int* block, int* row) {
  *block = (int)((uint32_t)slot / (uint32_t)c.block_rows);
  *row = slot - *block * c.block_rows;
  return slot >= 0 && *block < c.n_blocks;
}

// Checks a cache and fills in the strides of a dense one.  LAQ_OK or LAQ_ERR_INVALID.  need_k / need_v: the call touches that plane.
int fp4_view(const laq_fp4_cache* cache, bool need_k, bool need_v, Fp4View* view);

// A call of laq_fp4_attention.
struct Fp4Attention {
  int32_t Hq, n, blocks_per_inst, max_rows;
  float scale2;                          // scale * log2(e)
  int64_t n_tokens, stride_token, stride_head;
  const int32_t *start, *table, *rows;
  const void* q;
  void* out;
  float* lse;
};

hipError_t launch_block_map(int n, int block_rows, int n_blocks, int width, const int32_t* add, int32_t* rows, int32_t* table, int32_t* list,
                            int32_t* state, int32_t* start, int32_t* slots, int64_t n_slots, hipStream_t st);
hipError_t launch_fp4_store(const Fp4View& c, int dtype, int64_t n_tokens, const void* k, const void* v, int64_t stride_token,
                            int64_t stride_head, const int32_t* slots, hipStream_t st);
// instances inst0 .. inst0 + n - 1, `most` rows of a KV head at most
hipError_t launch_fp4_compact(const Fp4View& c, int dtype, int n, int inst0, int most, int L, const KvLayout& lay, const InstTable& tab,
                              const void* k, const void* v, const int32_t* idx, const int32_t* slots, hipStream_t st);
hipError_t launch_fp4_load(const Fp4View& c, int dtype, int64_t n_tokens, const int32_t* slots, void* k, void* v, hipStream_t st);
size_t fp4_attention_bytes(const Fp4View& c, int Hq, int dtype, int n, int64_t n_tokens, int max_rows);
bool fp4_attention_fits(const Fp4View& c, int dtype, const Fp4Attention& a, bool cut);      // in a launch
hipError_t launch_fp4_attention(const Fp4View& c, int dtype, const Fp4Attention& a, void* ws, hipStream_t st);

}  // namespace laq
