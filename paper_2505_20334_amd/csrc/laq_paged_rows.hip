// Rotary positions, and rows into the paged cache of 32, 16 or 8 bits and back (include/laq_cache.h: laq_rope, laq_cache_append,
// laq_cache_compact, laq_cache_load).
//
// A lane has eight numbers of a row, the 8, 16 or 32 adjacent lanes of a group one row, so that a row is read before any of it is written (a
// rotation in place) and its largest magnitude takes three to five lane exchanges.  Bound: memory.
//
// A workgroup has the heads of a few tokens: the sines and cosines of their pairs are made once, a pair a thread, and lie in LDS for all heads.
// An angle is position * frequency in 64 bits, where a position of 31 bits times 24 bits of frequency leaves 2^-53 of up to 2^31, reduced by two
// parts of pi / 2 (106 bits), and sine and cosine are Taylor's series on [-pi/4, pi/4] up to x^15 and x^16, less than 2^-53 away: about 30 instructions in 64 bits.
#include <type_traits>

#include "laq_paged.h"

namespace laq {

namespace {

constexpr int ROWS_THREADS = 256;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct Eight { float f[8]; };

__device__ __forceinline__ Eight read8(const uint16_t* p) {
  const u32x4 x = *reinterpret_cast<const u32x4*>(p);
  Eight r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.f[2 * i] = __uint_as_float(x[i] << 16);
    r.f[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
  }
  return r;
}
__device__ __forceinline__ Eight read8(const float* p) {
  const u32x4 a = *reinterpret_cast<const u32x4*>(p), b = *reinterpret_cast<const u32x4*>(p + 4);
  Eight r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.f[i] = __uint_as_float(a[i]);
    r.f[4 + i] = __uint_as_float(b[i]);
  }
  return r;
}
__device__ __forceinline__ float read1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float read1(const float* p) { return *p; }

__device__ __forceinline__ void write8(uint16_t* p, const Eight& v) {
  u32x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v.f[2 * i], v.f[2 * i + 1]}), bf16x2));
  *reinterpret_cast<u32x4*>(p) = x;
}
__device__ __forceinline__ void write8(float* p, const Eight& v) {
  u32x4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = __float_as_uint(v.f[i]);
    b[i] = __float_as_uint(v.f[4 + i]);
  }
  *reinterpret_cast<u32x4*>(p) = a;
  *reinterpret_cast<u32x4*>(p + 4) = b;
}

// Eight numbers of the cache.
__device__ __forceinline__ Eight read8(const E4m3* p, float scale) {
  const uint2 x = *reinterpret_cast<const uint2*>(p);
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(x.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(x.x, true);
  const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8(x.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8(x.y, true);
  return Eight{{a[0] * scale, a[1] * scale, b[0] * scale, b[1] * scale, c[0] * scale, c[1] * scale, d[0] * scale, d[1] * scale}};
}

template <typename C> constexpr bool scaled() { return std::is_same<C, E4m3>::value; }

// The largest of x over the LANES lanes of a group.
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
#pragma unroll
  for (int m = 1; m < LANES; m *= 2) x = max(x, (uint32_t)__shfl_xor((int)x, m));
  return x;
}

// Where a row of the cache begins, and its scale.
__device__ __forceinline__ int64_t row_at(const PagedView& c, int block, int head, int row) { return block * c.block + head * c.head + row * c.row; }
__device__ __forceinline__ int64_t scale_at(const PagedView& c, int block, int head, int row) {
  return ((int64_t)block * c.Hkv + head) * c.block_rows + row;
}

// A lane's numbers of a row to its place.  All lanes of a group come here together; those behind the row's end with zeros and on = false.
template <typename C, int LANES>
__device__ __forceinline__ void put(const PagedPlane& plane, const Eight& v, int64_t to, int64_t scale_to, int col, bool on) {
  if constexpr (scaled<C>()) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v.f[i]) & 0x7fffffffu);
    const uint32_t s = e4m3_scale_of(group_max<LANES>(most));
    const float by = __uint_as_float((254u - s) << 23);              // (s = 255: not used)
    uint32_t lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v.f[0] * by, v.f[1] * by, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v.f[2] * by, v.f[3] * by, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v.f[4] * by, v.f[5] * by, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v.f[6] * by, v.f[7] * by, hi, true);
    if (on) *reinterpret_cast<uint2*>(static_cast<E4m3*>(plane.x) + to + col * 8) = s == 255u ? uint2{0, 0} : uint2{lo, hi};
    if (col == 0) plane.scales[scale_to] = (uint8_t)s;
  } else {
    if (on) write8(static_cast<C*>(plane.x) + to + col * 8, v);
  }
}

// Sine and cosine of an angle given in 64 bits.
__device__ __forceinline__ void sine_cosine(double angle, double* s, double* c) {
  const double n = __builtin_rint(angle * 0.63661977236758134308);              // 2 / pi
  double x = __builtin_fma(-n, 1.57079632679489655800e+00, angle);              // pi / 2 in two parts
  x = __builtin_fma(-n, 6.12323399573676603587e-17, x);
  const double y = x * x;
  double p = -1.0 / 1307674368000.0, q = 1.0 / 20922789888000.0;                // 1 / 15!, 1 / 16!
  p = __builtin_fma(p, y, 1.0 / 6227020800.0);
  p = __builtin_fma(p, y, -1.0 / 39916800.0);
  p = __builtin_fma(p, y, 1.0 / 362880.0);
  p = __builtin_fma(p, y, -1.0 / 5040.0);
  p = __builtin_fma(p, y, 1.0 / 120.0);
  p = __builtin_fma(p, y, -1.0 / 6.0);
  q = __builtin_fma(q, y, -1.0 / 87178291200.0);
  q = __builtin_fma(q, y, 1.0 / 479001600.0);
  q = __builtin_fma(q, y, -1.0 / 3628800.0);
  q = __builtin_fma(q, y, 1.0 / 40320.0);
  q = __builtin_fma(q, y, -1.0 / 720.0);
  q = __builtin_fma(q, y, 1.0 / 24.0);
  q = __builtin_fma(q, y, -0.5);
  const double sx = __builtin_fma(p * y, x, x), cx = __builtin_fma(q, y, 1.0);
  const int quarter = (int)((long long)n & 3);
  *s = quarter & 1 ? cx : sx;
  *c = quarter & 1 ? sx : cx;
  if (quarter & 2) *s = -*s;
  if (quarter == 1 || quarter == 2) *c = -*c;
}

// x * cos + other * sin, each product and the sum rounded: the result does not depend on which of them a fused operation would take.
__device__ __forceinline__ float turned(float x, float c, float other, float s) {
#pragma clang fp contract(off)
  const float a = x * c, b = other * s;
  return a + b;
}

// T: the tokens' rows; C: the cache's numbers (T itself, where k goes to k_out).  LANES: of a row.  ROPE: 0 none; 1 the two numbers of a pair lie in
// the same lane, or in the same place of another lane's; 2 anywhere.
template <typename T, typename C, int LANES, int ROPE, bool CACHE>
__global__ __launch_bounds__(ROWS_THREADS) void token_rows_kernel(TokenCall t, PagedView c, int tokens_each, int rows_each) {
  constexpr int ROWS = ROWS_THREADS / LANES;                         // rows that a workgroup has at once
  __shared__ float2 turn[ROPE ? 4 * 128 : 1];                        // [tokens_each][rot / 2]: cos, sin
  const int col = threadIdx.x % LANES, lane_row = threadIdx.x / LANES;
  const int64_t t0 = (int64_t)blockIdx.x * tokens_each;
  const int tokens = (int)min((int64_t)tokens_each, t.n_tokens - t0);
  const int pairs = t.rope.rot / 2;
  if constexpr (ROPE != 0) {
    for (int i = threadIdx.x; i < tokens * pairs; i += ROWS_THREADS) {
      const int tok = i / pairs, j = i - tok * pairs;
      double s, co;
      sine_cosine((double)t.rope.positions[t0 + tok] * (double)t.rope.inv_freq[j], &s, &co);
      turn[i] = float2{(float)(co * (double)t.rope.mscale), (float)(s * (double)t.rope.mscale)};
    }
    __syncthreads();
  }
  const bool on = col * 8 < t.d;
  const int first = blockIdx.y * rows_each, q_rows = t.q.heads, qk_rows = q_rows + t.k.heads, all = qk_rows + t.v.heads;
  const int end = min(first + rows_each, all);
  for (int tok = 0; tok < tokens; ++tok) {
    // what turns this lane's numbers: x * co + other * si
    float co[8], si[8];
    int other_col = 0;
    if constexpr (ROPE != 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = col * 8 + e;
        const bool in = at < t.rope.rot, upper = t.rope.interleaved ? at & 1 : at >= pairs;
        const int j = t.rope.interleaved ? at >> 1 : upper ? at - pairs : at;
        const float2 w = in ? turn[tok * pairs + j] : float2{1.f, 0.f};
        co[e] = w.x;
        si[e] = upper ? w.y : -w.y;
      }
      other_col = t.rope.interleaved ? col : col * 8 < pairs ? col + pairs / 8 : col - pairs / 8;
    }
    int block = 0, row = 0;
    const bool kept = CACHE && paged_slot(c, t.slots[t0 + tok], &block, &row);
    for (int r0 = first; r0 < end; r0 += ROWS) {
      const int r = r0 + lane_row;
      if (r >= end) continue;                                        // (a group's lanes together)
      const bool is_q = r < q_rows, is_k = !is_q && r < qk_rows;
      const int head = is_q ? r : is_k ? r - q_rows : r - qk_rows;
      const TokenHeads& from = is_q ? t.q : is_k ? t.k : t.v;
      const T* src = static_cast<const T*>(from.x) + (t0 + tok) * from.token + head * from.head;
      Eight v{};
      if (on) v = read8(src + col * 8);
      if (ROPE != 0 && (is_q || is_k)) {
        Eight o = v;
        if (t.rope.interleaved) {
#pragma unroll
          for (int e = 0; e < 8; ++e) o.f[e] = v.f[e ^ 1];
        } else if (ROPE == 1) {
#pragma unroll
          for (int e = 0; e < 8; ++e) o.f[e] = __shfl(v.f[e], other_col, LANES);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int at = col * 8 + e;
            if (at < t.rope.rot) o.f[e] = read1(src + (at < pairs ? at + pairs : at - pairs));
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col * 8 + e < t.rope.rot) v.f[e] = turned(v.f[e], co[e], o.f[e], si[e]);
      }
      if (is_q || !CACHE) {
        const TokenHeads& to = is_q ? t.q_out : t.k_out;
        if (on) write8(static_cast<T*>(to.x) + (t0 + tok) * to.token + head * to.head + col * 8, v);
      } else if (kept) {
        put<C, LANES>(is_k ? c.k : c.v, v, row_at(c, block, head, row), scale_at(c, block, head, row), col, on);
      }
    }
  }
}

// A workgroup has rows of one head of an instance; the list has an entry for each, the slots one for all heads.
template <typename T, typename C, int LANES>
__global__ __launch_bounds__(ROWS_THREADS) void paged_compact_kernel(PagedView c, int L, KvLayout lay, InstTable tab, int inst0, const T* __restrict__ k,
                                                                     const T* __restrict__ v, const int32_t* __restrict__ idx,
                                                                     const int32_t* __restrict__ slots) {
  constexpr int ROWS = ROWS_THREADS / LANES;
  const int col = threadIdx.x % LANES, li = blockIdx.z, head = blockIdx.y, bk = tab.rows(li), r = blockIdx.x * ROWS + threadIdx.x / LANES;
  if (r >= bk) return;
  const int64_t first = tab.first(li);
  const int j = idx[first + (int64_t)head * bk + r], slot = slots[first / c.Hkv + r];
  int block, row;
  if (j < 0 || j >= L || !paged_slot(c, slot, &block, &row)) return;
  const bool on = col * 8 < c.d;
  int64_t from = (int64_t)(inst0 + li) * lay.inst + head * lay.head + col * 8;
  int at = j;
  if (lay.table) from += paged_block_offset(lay, inst0 + li, j, &at);
  from += (int64_t)at * lay.row;
  Eight kv{}, vv{};
  if (on) kv = read8(k + from);
  if (on && v) vv = read8(v + from);
  const int64_t to = row_at(c, block, head, row), scale_to = scale_at(c, block, head, row);
  put<C, LANES>(c.k, kv, to, scale_to, col, on);
  if (v) put<C, LANES>(c.v, vv, to, scale_to, col, on);
}

template <typename T, typename C, int LANES>
__global__ __launch_bounds__(ROWS_THREADS) void paged_load_kernel(PagedView c, int64_t n_rows, const int32_t* __restrict__ slots, T* __restrict__ k,
                                                                  T* __restrict__ v) {
  constexpr int ROWS = ROWS_THREADS / LANES;
  const int col = threadIdx.x % LANES;
  const int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  if (r >= n_rows || col * 8 >= c.d) return;
  const uint32_t token = (uint32_t)r / (uint32_t)c.Hkv;              // (n_rows < 2^28)
  const int head = (int)((uint32_t)r - token * (uint32_t)c.Hkv);
  int block, row;
  const bool there = paged_slot(c, slots[token], &block, &row);
  const int64_t at = there ? row_at(c, block, head, row) + col * 8 : 0, scale = there ? scale_at(c, block, head, row) : 0;
  const auto one = [&](const PagedPlane& plane, T* out) {
    Eight x{};
    if (there) {
      if constexpr (scaled<C>()) x = read8(static_cast<const E4m3*>(plane.x) + at, e4m3_scale_value(plane.scales[scale]));
      else x = read8(static_cast<const C*>(plane.x) + at);
    }
    write8(out + r * c.d + col * 8, x);
  };
  if (k) one(c.k, k);
  if (v) one(c.v, v);
}

// f(lanes of a row) with the least that a row of d numbers has room in
template <typename F>
hipError_t by_size(int d, const F& f) {
  if (d <= 64) return f(std::integral_constant<int, 8>{});
  if (d <= 128) return f(std::integral_constant<int, 16>{});
  return f(std::integral_constant<int, 32>{});
}
// f(a null pointer of the type) for the types of rows and of the cache's numbers
template <typename F>
hipError_t by_types(int dtype, int type, const F& f) {
  const auto second = [&](auto rows) {
    switch (type) {
      case LAQ_F32: return f(rows, (float*)nullptr);
      case LAQ_BF16: return f(rows, (uint16_t*)nullptr);
      default: return f(rows, (E4m3*)nullptr);
    }
  };
  return dtype == LAQ_BF16 ? second((uint16_t*)nullptr) : second((float*)nullptr);
}
template <typename P> using Of = std::remove_pointer_t<P>;

// How a call's rotation finds the other number of a pair.
int rope_kind(const RopeArgs& r) { return !r.inv_freq ? 0 : r.interleaved || r.rot % 16 == 0 ? 1 : 2; }

template <typename T, typename C, int LANES, bool CACHE>
hipError_t token_rows(const TokenCall& t, const PagedView& c, hipStream_t st) {
  constexpr int ROWS = ROWS_THREADS / LANES;
  const int all = t.q.heads + t.k.heads + t.v.heads;
  // few tokens: a row a group, so that the call is as short as it can be; many: four tokens to a workgroup, all their heads
  const bool few = t.n_tokens <= 256;
  const int tokens_each = few ? 1 : 4, rows_each = few ? ROWS : (all + ROWS - 1) / ROWS * ROWS;
  const dim3 grid((unsigned)((t.n_tokens + tokens_each - 1) / tokens_each), (unsigned)((all + rows_each - 1) / rows_each));
  switch (rope_kind(t.rope)) {
    case 0: hipLaunchKernelGGL((token_rows_kernel<T, C, LANES, 0, CACHE>), grid, dim3(ROWS_THREADS), 0, st, t, c, tokens_each, rows_each); break;
    case 1: hipLaunchKernelGGL((token_rows_kernel<T, C, LANES, 1, CACHE>), grid, dim3(ROWS_THREADS), 0, st, t, c, tokens_each, rows_each); break;
    default: hipLaunchKernelGGL((token_rows_kernel<T, C, LANES, 2, CACHE>), grid, dim3(ROWS_THREADS), 0, st, t, c, tokens_each, rows_each); break;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_token_rows(const TokenCall& t, int dtype, const PagedView* cache, hipStream_t st) {
  return by_size(t.d, [&](auto lanes) {
    if (!cache) {
      return dtype == LAQ_BF16 ? token_rows<uint16_t, uint16_t, lanes(), false>(t, PagedView{}, st) : token_rows<float, float, lanes(), false>(t, PagedView{}, st);
    }
    return by_types(dtype, cache->type, [&](auto rows, auto numbers) { return token_rows<Of<decltype(rows)>, Of<decltype(numbers)>, lanes(), true>(t, *cache, st); });
  });
}

hipError_t launch_paged_compact(const PagedView& c, int dtype, int n, int inst0, int most, int L, const KvLayout& lay, const InstTable& tab,
                                const void* k, const void* v, const int32_t* idx, const int32_t* slots, hipStream_t st) {
  return by_size(c.d, [&](auto lanes) {
    return by_types(dtype, c.type, [&](auto rows, auto numbers) {
      using T = Of<decltype(rows)>;
      constexpr int ROWS = ROWS_THREADS / lanes();
      hipLaunchKernelGGL((paged_compact_kernel<T, Of<decltype(numbers)>, lanes()>), dim3((most + ROWS - 1) / ROWS, c.Hkv, n), dim3(ROWS_THREADS), 0, st, c, L,
                         lay, tab, inst0, static_cast<const T*>(k), static_cast<const T*>(v), idx, slots);
      return hipGetLastError();
    });
  });
}

hipError_t launch_paged_load(const PagedView& c, int dtype, int64_t n_tokens, const int32_t* slots, void* k, void* v, hipStream_t st) {
  const int64_t n_rows = n_tokens * c.Hkv;
  return by_size(c.d, [&](auto lanes) {
    return by_types(dtype, c.type, [&](auto rows, auto numbers) {
      using T = Of<decltype(rows)>;
      constexpr int ROWS = ROWS_THREADS / lanes();
      hipLaunchKernelGGL((paged_load_kernel<T, Of<decltype(numbers)>, lanes()>), dim3((unsigned)((n_rows + ROWS - 1) / ROWS)), dim3(ROWS_THREADS), 0, st, c,
                         n_rows, slots, static_cast<T*>(k), static_cast<T*>(v));
      return hipGetLastError();
    });
  });
}

}  // namespace laq
