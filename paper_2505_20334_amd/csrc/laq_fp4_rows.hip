// Rows into the 4-bit cache and back (include/laq_fp4.h: laq_fp4_store, laq_fp4_compact, laq_fp4_load).
//
// A lane has eight numbers of a row, four adjacent lanes a block of 32: they agree on its largest magnitude with two lane exchanges, and
// each turns its numbers into one word of codes with four conversions.  Reads are 16 bytes a lane (fp32: 32), codes are written 16 bytes a
// block.  Bound: memory; a number costs about two instructions.
#include <type_traits>

#include "laq_fp4_codes.h"

namespace laq {

namespace {

constexpr int ROWS_THREADS = 256;

// The largest magnitude's bits over the lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true));       // lane ^ 1
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));    // lane ^ 2
}

// Reads of rows that one workgroup reads once, past the caches (32 x 8 heads, 2048 to 128 rows of 8192 compacted and loaded: 81 -> 73 us).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4 read_once(const void* p) { return __builtin_nontemporal_load(static_cast<const u32x4*>(p)); }

struct Piece16 {
  uint4 x;
  __device__ __forceinline__ void read(const uint16_t* p) { x = __builtin_bit_cast(uint4, read_once(p)); }
  __device__ __forceinline__ uint32_t most() const {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
    return m << 16;
  }
  __device__ __forceinline__ uint32_t codes(float scale) const {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.x), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.y), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.z), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, x.w), scale, 3);
  }
};
struct Piece32 {
  float4 a, b;
  __device__ __forceinline__ void read(const float* p) {
    a = __builtin_bit_cast(float4, read_once(p));
    b = __builtin_bit_cast(float4, read_once(p + 4));
  }
  __device__ __forceinline__ uint32_t most() const {
    const float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ uint32_t codes(float scale) const {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a.x, a.y, scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, a.z, a.w, scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, b.x, b.y, scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, b.z, b.w, scale, 3);
  }
};
template <typename T> struct PieceOfRow { using type = Piece16; };
template <> struct PieceOfRow<float> { using type = Piece32; };

// A workgroup's lanes over rows of d / 8 pieces: as many rows as fit, a number of times.
template <int D32>
struct RowLanes {
  static constexpr int PIECES = 4 * D32, ROWS = ROWS_THREADS / PIECES;
  int row, col;
  bool on;
  __device__ __forceinline__ RowLanes() : row(threadIdx.x / PIECES), col(threadIdx.x % PIECES), on((int)threadIdx.x < ROWS * PIECES) {}
};
// Rows that a lane has in flight, K and V of each.  Rows that lie in order: two (16381 tokens x 8 heads of d = 128 stored in 33.2 us, with one
// 33.8).  Rows that are looked up in a list first: one, since more workgroups hide the wait better than longer ones (32 x 8 heads, 2048 to
// 128 rows of 8192 compacted and loaded, one 72.5 us, two 76.5, four 76.9).
constexpr int PASSES_ORDERED = 2, PASSES_LISTED = 1;

__device__ __forceinline__ int64_t code_at(const Fp4View& c, int block, int head, int row) { return block * c.block + head * c.head + row * c.row; }
__device__ __forceinline__ int64_t scale_at(const Fp4View& c, int block, int head, int row) { return block * c.scale_block + head * c.scale_head + row * c.scale_row; }

// A piece to its place.  All lanes of a quad come here together.
template <typename P>
__device__ __forceinline__ void put(const Fp4Plane& plane, const P& p, int64_t codes_to, int64_t scale_to, int col) {
  const uint32_t scale = fp4_scale_of(quad_max(p.most()));
  const uint32_t codes = scale == 255u ? 0u : p.codes(fp4_scale_value(scale));
  *reinterpret_cast<uint32_t*>(plane.codes + codes_to + col * 4) = codes;
  if ((col & 3) == 0) plane.scales[scale_to + (col >> 2)] = (uint8_t)scale;
}

struct TokenRows {
  int64_t n_rows;                        // tokens x heads
  int64_t token, head;                   // elements between tokens and heads
  uint64_t per_head;                     // ceil(2^32 / Hkv): x / Hkv = x * per_head >> 32 for x below 2^17 (and Hkv up to 2^15)
};
// Token and head of a lane's row: `first` (the same for the workgroup) and `more` rows.
__device__ __forceinline__ int64_t token_of(const Fp4View& c, const TokenRows& t, int64_t first, int more, int* head) {
  const int64_t token = first / c.Hkv;
  const uint32_t x = (uint32_t)(first - token * c.Hkv) + more, q = (uint32_t)(x * t.per_head >> 32);
  *head = (int)(x - q * c.Hkv);
  return token + q;
}

template <typename T, int D32>
__global__ __launch_bounds__(ROWS_THREADS) void fp4_store_kernel(Fp4View c, TokenRows t, const T* __restrict__ k, const T* __restrict__ v,
                                                                 const int32_t* __restrict__ slots) {
  const RowLanes<D32> l;
  constexpr int PASSES = PASSES_ORDERED;
  const int64_t first = (int64_t)blockIdx.x * (l.ROWS * PASSES);
  typename PieceOfRow<T>::type kp[PASSES], vp[PASSES];
  int slot[PASSES], head[PASSES];
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const int more = u * l.ROWS + l.row;
    slot[u] = -1;
    if (!l.on || first + more >= t.n_rows) continue;
    const int64_t token = token_of(c, t, first, more, &head[u]), from = token * t.token + head[u] * t.head + l.col * 8;
    slot[u] = slots[token];
    if (k) kp[u].read(k + from);
    if (v) vp[u].read(v + from);
  }
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    int block, row;
    if (!fp4_slot(c, slot[u], &block, &row)) continue;
    const int64_t codes_to = code_at(c, block, head[u], row), scale_to = scale_at(c, block, head[u], row);
    if (k) put(c.k, kp[u], codes_to, scale_to, l.col);
    if (v) put(c.v, vp[u], codes_to, scale_to, l.col);
  }
}

// A workgroup has rows of one head of an instance; the list has an entry for each, the slots one for all heads.
template <typename T, int D32>
__global__ __launch_bounds__(ROWS_THREADS) void fp4_compact_kernel(Fp4View c, int L, KvLayout lay, InstTable tab, int inst0, const T* __restrict__ k,
                                                                   const T* __restrict__ v, const int32_t* __restrict__ idx,
                                                                   const int32_t* __restrict__ slots) {
  const RowLanes<D32> l;
  constexpr int PASSES = PASSES_LISTED;
  const int li = blockIdx.z, head = blockIdx.y, bk = tab.rows(li), r0 = blockIdx.x * (l.ROWS * PASSES);
  if (r0 >= bk) return;
  const int64_t first = tab.first(li), from_head = (int64_t)(inst0 + li) * lay.inst + head * lay.head + l.col * 8;
  typename PieceOfRow<T>::type kp[PASSES], vp[PASSES];
  int j[PASSES], slot[PASSES];
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const int r = r0 + u * l.ROWS + l.row;
    j[u] = -1;
    slot[u] = -1;
    if (l.on && r < bk) {
      j[u] = idx[first + (int64_t)head * bk + r];
      slot[u] = slots[first / c.Hkv + r];
    }
  }
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    if (j[u] < 0 || j[u] >= L) {
      slot[u] = -1;
      continue;
    }
    int64_t from = from_head;
    int row = j[u];
    if (lay.table) from += paged_block_offset(lay, inst0 + li, j[u], &row);
    from += (int64_t)row * lay.row;
    kp[u].read(k + from);
    if (v) vp[u].read(v + from);
  }
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    int block, row;
    if (!fp4_slot(c, slot[u], &block, &row)) continue;
    const int64_t codes_to = code_at(c, block, head, row), scale_to = scale_at(c, block, head, row);
    put(c.k, kp[u], codes_to, scale_to, l.col);
    if (v) put(c.v, vp[u], codes_to, scale_to, l.col);
  }
}

__device__ __forceinline__ void put_numbers(uint16_t* out, uint4 x) { *reinterpret_cast<uint4*>(out) = x; }
__device__ __forceinline__ void put_numbers(float* out, uint4 x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = w[i] << 16;
    f[2 * i + 1] = w[i] & 0xffff0000u;
  }
  *reinterpret_cast<uint4*>(out) = uint4{f[0], f[1], f[2], f[3]};
  *reinterpret_cast<uint4*>(out + 4) = uint4{f[4], f[5], f[6], f[7]};
}

template <typename T, int D32>
__global__ __launch_bounds__(ROWS_THREADS) void fp4_load_kernel(Fp4View c, TokenRows t, const int32_t* __restrict__ slots, T* __restrict__ k,
                                                                T* __restrict__ v) {
  const RowLanes<D32> l;
  constexpr int PASSES = PASSES_ORDERED;
  const int64_t first = (int64_t)blockIdx.x * (l.ROWS * PASSES);
  int slot[PASSES], head[PASSES];
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const int more = u * l.ROWS + l.row;
    if (l.on && first + more < t.n_rows) slot[u] = slots[token_of(c, t, first, more, &head[u])];
  }
  uint32_t codes[PASSES][2], scale[PASSES][2];
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
#pragma unroll
    for (int i = 0; i < 2; ++i) codes[u][i] = scale[u][i] = 0;
    int block, row;
    if (!l.on || first + u * l.ROWS + l.row >= t.n_rows || !fp4_slot(c, slot[u], &block, &row)) continue;
    const int64_t codes_at = code_at(c, block, head[u], row) + l.col * 4, scales_at = scale_at(c, block, head[u], row) + (l.col >> 2);
    if (k) {
      codes[u][0] = *reinterpret_cast<const uint32_t*>(c.k.codes + codes_at);
      scale[u][0] = c.k.scales[scales_at];
    }
    if (v) {
      codes[u][1] = *reinterpret_cast<const uint32_t*>(c.v.codes + codes_at);
      scale[u][1] = c.v.scales[scales_at];
    }
  }
#pragma unroll
  for (int u = 0; u < PASSES; ++u) {
    const int64_t row = first + u * l.ROWS + l.row;
    if (!l.on || row >= t.n_rows) continue;
    const int64_t to = row * (8 * l.PIECES) + l.col * 8;
    if (k) put_numbers(k + to, fp4_to_bf16(codes[u][0], fp4_scale_value(scale[u][0])));
    if (v) put_numbers(v + to, fp4_to_bf16(codes[u][1], fp4_scale_value(scale[u][1])));
  }
}

// f(head size / 32) with the type of the rows
template <typename F>
hipError_t by_size(int d, const F& f) {
  switch (d / 32) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 5: return f(std::integral_constant<int, 5>{});
    case 6: return f(std::integral_constant<int, 6>{});
    case 7: return f(std::integral_constant<int, 7>{});
    default: return f(std::integral_constant<int, 8>{});
  }
}
template <int D32, int PASSES>
unsigned workgroups(int64_t rows) {
  return (unsigned)((rows + RowLanes<D32>::ROWS * PASSES - 1) / (RowLanes<D32>::ROWS * PASSES));
}

template <typename T>
hipError_t store(const Fp4View& c, const TokenRows& t, const void* k, const void* v, const int32_t* slots, hipStream_t st) {
  return by_size(c.d, [&](auto d32) {
    hipLaunchKernelGGL((fp4_store_kernel<T, d32()>), dim3(workgroups<d32(), PASSES_ORDERED>(t.n_rows)), dim3(ROWS_THREADS), 0, st, c, t, static_cast<const T*>(k),
                       static_cast<const T*>(v), slots);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t compact(const Fp4View& c, int n, int inst0, int most, int L, const KvLayout& lay, const InstTable& tab, const void* k, const void* v,
                   const int32_t* idx, const int32_t* slots, hipStream_t st) {
  return by_size(c.d, [&](auto d32) {
    hipLaunchKernelGGL((fp4_compact_kernel<T, d32()>), dim3(workgroups<d32(), PASSES_LISTED>(most), c.Hkv, n), dim3(ROWS_THREADS), 0, st, c, L, lay, tab, inst0,
                       static_cast<const T*>(k), static_cast<const T*>(v), idx, slots);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t load(const Fp4View& c, const TokenRows& t, const int32_t* slots, void* k, void* v, hipStream_t st) {
  return by_size(c.d, [&](auto d32) {
    hipLaunchKernelGGL((fp4_load_kernel<T, d32()>), dim3(workgroups<d32(), PASSES_ORDERED>(t.n_rows)), dim3(ROWS_THREADS), 0, st, c, t, slots, static_cast<T*>(k),
                       static_cast<T*>(v));
    return hipGetLastError();
  });
}

TokenRows token_rows(const Fp4View& c, int64_t n_tokens, int64_t stride_token, int64_t stride_head) {
  return TokenRows{n_tokens * c.Hkv, stride_token, stride_head, ((1ull << 32) + c.Hkv - 1) / c.Hkv};
}

}  // namespace

hipError_t launch_fp4_store(const Fp4View& c, int dtype, int64_t n_tokens, const void* k, const void* v, int64_t stride_token,
                            int64_t stride_head, const int32_t* slots, hipStream_t st) {
  const TokenRows t = token_rows(c, n_tokens, stride_token, stride_head);
  return dtype == LAQ_BF16 ? store<uint16_t>(c, t, k, v, slots, st) : store<float>(c, t, k, v, slots, st);
}

hipError_t launch_fp4_compact(const Fp4View& c, int dtype, int n, int inst0, int most, int L, const KvLayout& lay, const InstTable& tab,
                              const void* k, const void* v, const int32_t* idx, const int32_t* slots, hipStream_t st) {
  return dtype == LAQ_BF16 ? compact<uint16_t>(c, n, inst0, most, L, lay, tab, k, v, idx, slots, st)
                           : compact<float>(c, n, inst0, most, L, lay, tab, k, v, idx, slots, st);
}

hipError_t launch_fp4_load(const Fp4View& c, int dtype, int64_t n_tokens, const int32_t* slots, void* k, void* v, hipStream_t st) {
  const TokenRows t = token_rows(c, n_tokens, 0, 0);
  return dtype == LAQ_BF16 ? load<uint16_t>(c, t, slots, k, v, st) : load<float>(c, t, slots, k, v, st);
}

}  // namespace laq
