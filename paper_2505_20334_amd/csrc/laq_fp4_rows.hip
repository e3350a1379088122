// Rows into the 4-bit cache and back (include/laq_fp4.h: laq_fp4_store, laq_fp4_compact, laq_fp4_load).
//
// A lane has eight numbers of a row, four adjacent lanes a block of 32: they agree on its largest magnitude with two lane exchanges, and
// each turns its numbers into one word of codes with four conversions.  Reads are 16 bytes a lane (fp32: 32), codes are written 16 bytes a
// block.  Bound: memory; a number costs about two instructions.
#include "laq_fp4_codes.h"
#include "laq_lanegroup.h"

namespace laq {

namespace {

constexpr int ROWS_THREADS = 256;

// The largest magnitude's bits over the lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true));       // lane ^ 1
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));    // lane ^ 2
}

struct Piece16 {
  uint4 x;
  __device__ __forceinline__ void read(const uint16_t* p) { x = *reinterpret_cast<const uint4*>(p); }
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
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
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

// Piece `col` of a row at src to (block, head, row) of a plane.  All lanes of a quad come here together.
template <typename T>
__device__ __forceinline__ void put(const Fp4View& c, const Fp4Plane& plane, const T* src, int col, int block, int head, int row) {
  typename PieceOfRow<T>::type p;
  p.read(src + col * 8);
  const uint32_t scale = fp4_scale_of(quad_max(p.most()));
  const uint32_t codes = scale == 255u ? 0u : p.codes(fp4_scale_value(scale));
  *reinterpret_cast<uint32_t*>(plane.codes + block * c.block + head * c.head + row * c.row + col * 4) = codes;
  if ((col & 3) == 0) plane.scales[block * c.scale_block + head * c.scale_head + row * c.scale_row + (col >> 2)] = (uint8_t)scale;
}

// Which token and which of its pieces a thread has, `per` pieces a token.
__device__ __forceinline__ int64_t token_of(int per, int* piece) {
  const int64_t first = (int64_t)blockIdx.x * ROWS_THREADS, token = first / per;      // (of the workgroup)
  const uint32_t at = (uint32_t)(first - token * per) + threadIdx.x, more = at / (uint32_t)per;
  *piece = (int)(at - more * per);
  return token + more;
}

struct TokenRows {
  int64_t n_tokens, token, head;         // elements between tokens and heads
};

template <typename T>
__global__ __launch_bounds__(ROWS_THREADS) void fp4_store_kernel(Fp4View c, TokenRows t, const T* __restrict__ k, const T* __restrict__ v,
                                                                 const int32_t* __restrict__ slots) {
  const int pieces = c.d / 8;
  int piece, block, row;
  const int64_t token = token_of(c.Hkv * pieces, &piece);
  if (token >= t.n_tokens || !fp4_slot(c, slots[token], &block, &row)) return;
  const int head = piece / pieces, col = piece - head * pieces;
  const T* src = (blockIdx.y == 0 && k ? k : v) + token * t.token + head * t.head;
  put(c, blockIdx.y == 0 && k ? c.k : c.v, src, col, block, head, row);
}

// The list's own order: a row of one head is d / 8 adjacent lanes, a head's rows follow one another (laq_compact.hip).
template <typename T, typename TAB>
__global__ __launch_bounds__(ROWS_THREADS) void fp4_compact_kernel(Fp4View c, int L, KvLayout lay, TAB tab, int inst0, const T* __restrict__ k,
                                                                   const T* __restrict__ v, const int32_t* __restrict__ idx,
                                                                   const int32_t* __restrict__ slots) {
  const int pieces = c.d / 8, li = blockIdx.z, bk = tab.rows(li);
  int col;
  const int64_t at = token_of(pieces, &col);
  if (at >= (int64_t)c.Hkv * bk) return;
  const int head = (int)((uint32_t)at / (uint32_t)bk), r = (int)at - head * bk;
  const int64_t first = tab.first(li);   // (of the list; the slots have one entry for all heads)
  const int j = idx[first + at];
  int block, row;
  if (j < 0 || j >= L || !fp4_slot(c, slots[first / c.Hkv + r], &block, &row)) return;
  int64_t from = (int64_t)(inst0 + li) * lay.inst + (int64_t)j * lay.row;
  if (lay.table) {
    int in_block;
    from = paged_block_offset(lay, inst0 + li, j, &in_block);
    from += (int64_t)in_block * lay.row;
  }
  const T* src = (blockIdx.y == 0 ? k : v) + from + head * lay.head;
  put(c, blockIdx.y == 0 ? c.k : c.v, src, col, block, head, row);
}

template <typename T>
__global__ __launch_bounds__(ROWS_THREADS) void fp4_load_kernel(Fp4View c, int64_t n_tokens, const int32_t* __restrict__ slots,
                                                                T* __restrict__ k, T* __restrict__ v) {
  const int pieces = c.d / 8, per = c.Hkv * pieces;
  int piece, block, row;
  const int64_t token = token_of(per, &piece);
  if (token >= n_tokens) return;
  const bool first = blockIdx.y == 0 && k;
  const Fp4Plane plane = first ? c.k : c.v;
  uint4 x = {0, 0, 0, 0};
  if (fp4_slot(c, slots[token], &block, &row)) {
    const int head = piece / pieces, col = piece - head * pieces;
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(plane.codes + block * c.block + head * c.head + row * c.row + col * 4);
    const uint32_t scale = plane.scales[block * c.scale_block + head * c.scale_head + row * c.scale_row + (col >> 2)];
    x = fp4_to_bf16(codes, fp4_scale_value(scale));
  }
  T* out = (first ? k : v) + (token * per + piece) * 8;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(out) = x;
  } else {
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
}

unsigned workgroups(int64_t pieces) { return (unsigned)((pieces + ROWS_THREADS - 1) / ROWS_THREADS); }

template <typename T>
hipError_t store(const Fp4View& c, const TokenRows& t, const void* k, const void* v, const int32_t* slots, hipStream_t st) {
  hipLaunchKernelGGL(fp4_store_kernel<T>, dim3(workgroups(t.n_tokens * c.Hkv * (c.d / 8)), k && v ? 2 : 1), dim3(ROWS_THREADS), 0, st, c, t,
                     static_cast<const T*>(k), static_cast<const T*>(v), slots);
  return hipGetLastError();
}

template <typename T, typename TAB>
hipError_t compact(const Fp4View& c, int n, int inst0, int most, int L, const KvLayout& lay, const TAB& tab, const void* k, const void* v,
                   const int32_t* idx, const int32_t* slots, hipStream_t st) {
  hipLaunchKernelGGL((fp4_compact_kernel<T, TAB>), dim3(workgroups((int64_t)c.Hkv * most * (c.d / 8)), v ? 2 : 1, n), dim3(ROWS_THREADS), 0, st, c,
                     L, lay, tab, inst0, static_cast<const T*>(k), static_cast<const T*>(v), idx, slots);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_fp4_store(const Fp4View& c, int dtype, int64_t n_tokens, const void* k, const void* v, int64_t stride_token,
                            int64_t stride_head, const int32_t* slots, hipStream_t st) {
  const TokenRows t{n_tokens, stride_token, stride_head};
  return dtype == LAQ_BF16 ? store<uint16_t>(c, t, k, v, slots, st) : store<float>(c, t, k, v, slots, st);
}

hipError_t launch_fp4_compact(const Fp4View& c, int dtype, int n, int inst0, int most, int L, const KvLayout& lay, const InstTable& tab,
                              const void* k, const void* v, const int32_t* idx, const int32_t* slots, hipStream_t st) {
  return dtype == LAQ_BF16 ? compact<uint16_t>(c, n, inst0, most, L, lay, tab, k, v, idx, slots, st)
                           : compact<float>(c, n, inst0, most, L, lay, tab, k, v, idx, slots, st);
}

hipError_t launch_fp4_load(const Fp4View& c, int dtype, int64_t n_tokens, const int32_t* slots, void* k, void* v, hipStream_t st) {
  const dim3 grid(workgroups(n_tokens * c.Hkv * (c.d / 8)), k && v ? 2 : 1);
  if (dtype == LAQ_BF16)
    hipLaunchKernelGGL(fp4_load_kernel<uint16_t>, grid, dim3(ROWS_THREADS), 0, st, c, n_tokens, slots, static_cast<uint16_t*>(k), static_cast<uint16_t*>(v));
  else
    hipLaunchKernelGGL(fp4_load_kernel<float>, grid, dim3(ROWS_THREADS), 0, st, c, n_tokens, slots, static_cast<float*>(k), static_cast<float*>(v));
  return hipGetLastError();
}

}  // namespace laq
