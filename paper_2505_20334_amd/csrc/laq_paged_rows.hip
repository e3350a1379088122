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

// Rows that are read once, past the caches where a call has more of them than the caches hold (MANY_BYTES): 16381 tokens x 40 heads of d = 128 rotated 81 -> 73 us,
// appended and loaded 108 -> 90; in smaller calls, whose rows the caches still have from whoever made them, it costs (2048 tokens 17 -> 24 us).  So are the rows that
// laq_cache_load writes (32 layers compacted and loaded 99 -> 87 us), but not what is written to a cache, which is read soon.
constexpr int64_t MANY_BYTES = 128ll << 20;
template <bool PAST> __device__ __forceinline__ u32x4 get16(const void* p) {
  return PAST ? __builtin_nontemporal_load(static_cast<const u32x4*>(p)) : *static_cast<const u32x4*>(p);
}
template <bool PAST> __device__ __forceinline__ void put16(void* p, u32x4 x) {
  if constexpr (PAST) __builtin_nontemporal_store(x, static_cast<u32x4*>(p));
  else *static_cast<u32x4*>(p) = x;
}

template <bool PAST> __device__ __forceinline__ Eight read8(const uint16_t* p) {
  const u32x4 x = get16<PAST>(p);
  Eight r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.f[2 * i] = __uint_as_float(x[i] << 16);
    r.f[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
  }
  return r;
}
template <bool PAST> __device__ __forceinline__ Eight read8(const float* p) {
  const u32x4 a = get16<PAST>(p), b = get16<PAST>(p + 4);
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

template <bool PAST = false> __device__ __forceinline__ void write8(uint16_t* p, const Eight& v) {
  u32x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v.f[2 * i], v.f[2 * i + 1]}), bf16x2));
  put16<PAST>(p, x);
}
template <bool PAST = false> __device__ __forceinline__ void write8(float* p, const Eight& v) {
  u32x4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = __float_as_uint(v.f[i]);
    b[i] = __float_as_uint(v.f[4 + i]);
  }
  put16<PAST>(p, a);
  put16<PAST>(p + 4, b);
}

// Eight numbers of the cache.
__device__ __forceinline__ Eight read8(const E4m3* p, float scale) {
  const uint2 x = *reinterpret_cast<const uint2*>(p);
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(x.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(x.x, true);
  const f32x2 c = __builtin_amdgcn_cvt_pk_f32_fp8(x.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8(x.y, true);
  return Eight{{a[0] * scale, a[1] * scale, b[0] * scale, b[1] * scale, c[0] * scale, c[1] * scale, d[0] * scale, d[1] * scale}};
}

template <typename C> constexpr bool scaled() { return std::is_same<C, E4m3>::value; }

// The largest of x over the LANES lanes of a group: neighbours, pairs, and the mirrored other half of 8 and of 16 lanes, without LDS.
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true));
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xf, 0xf, true));
  if constexpr (LANES >= 16) x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xf, 0xf, true));
  if constexpr (LANES >= 32) x = max(x, (uint32_t)__shfl_xor((int)x, 16));
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

// How a rotation finds the other number of a pair.
enum { ROPE_NONE, ROPE_PIECES, ROPE_ANY, ROPE_NEIGHBOURS };      // in the same place of another lane's piece; anywhere; in the same piece

// T: the tokens' rows; C: the cache's numbers (T itself, where k goes to k_out).  LANES: of a row.  A workgroup has rows_each rows of each of tokens_each tokens,
// ROWS at a time, the reads of U times as many under way together.
template <typename T, typename C, int LANES, int ROPE, bool CACHE, bool PAST>
__global__ __launch_bounds__(ROWS_THREADS) void token_rows_kernel(TokenCall t, PagedView c, int tokens_each, int rows_each) {
  constexpr int ROWS = ROWS_THREADS / LANES;                         // rows that a workgroup has at once
  constexpr int U = 2;
  __shared__ alignas(16) float2 turn[ROPE ? 4 * 128 : 1];            // [tokens_each][rot / 2]: cos, sin
  const int col = threadIdx.x % LANES, lane_row = threadIdx.x / LANES;
  const int64_t t0 = (int64_t)blockIdx.x * tokens_each;
  const int tokens = (int)min((int64_t)tokens_each, t.n_tokens - t0);
  const int pairs = t.rope.rot / 2;
  const bool on = col * 8 < t.d;
  const int first = blockIdx.y * rows_each, q_rows = t.q.heads, qk_rows = q_rows + t.k.heads, all = qk_rows + t.v.heads;
  const int here = min(rows_each, all - first), times = (here + ROWS - 1) / ROWS;      // of a token
  // this lane's row number i of the workgroup (false: none)
  struct Row { int tok, head, kind; const T* src; };                 // kind 0 q, 1 k, 2 v
  const auto row_of = [&](int i, Row& r) {
    r.tok = i / times;
    const int at = first + (i - r.tok * times) * ROWS + lane_row;
    if (at >= first + here) return false;
    r.kind = at < q_rows ? 0 : at < qk_rows ? 1 : 2;
    r.head = at - (r.kind == 0 ? 0 : r.kind == 1 ? q_rows : qk_rows);
    const TokenHeads& from = r.kind == 0 ? t.q : r.kind == 1 ? t.k : t.v;
    r.src = static_cast<const T*>(from.x) + (t0 + r.tok) * from.token + r.head * from.head;
    return true;
  };
  if constexpr (ROPE != ROPE_NONE) {
    for (int i = threadIdx.x; i < tokens * pairs; i += ROWS_THREADS) {
      const int tok = i / pairs, j = i - tok * pairs;
      double s, co;
      sine_cosine((double)t.rope.positions[t0 + tok] * (double)t.rope.inv_freq[j], &s, &co);
      turn[i] = float2{(float)(co * (double)t.rope.mscale), (float)(s * (double)t.rope.mscale)};
    }
    __syncthreads();
  }
  // (a group's lanes are together in all that follows: a row is read before any of it is written)
  for (int i0 = 0; i0 < tokens * times; i0 += U) {
    Row row[U];
    Eight v[U];
    bool is[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      is[u] = i0 + u < tokens * times && row_of(i0 + u, row[u]);
      v[u] = Eight{};
      if (is[u] && on) v[u] = read8<PAST>(row[u].src + col * 8);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!is[u]) continue;
      const Row& r = row[u];
      if (ROPE != ROPE_NONE && r.kind < 2) {
        const float2* const by = turn + r.tok * pairs;
        if constexpr (ROPE == ROPE_PIECES) {
          const bool upper = col * 8 >= pairs, in = col * 8 < t.rope.rot;
          const int other = upper ? col - pairs / 8 : col + pairs / 8, j0 = upper ? col * 8 - pairs : col * 8;
          Eight o;
#pragma unroll
          for (int e = 0; e < 8; ++e) o.f[e] = __shfl(v[u].f[e], other, LANES);
          if (in) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const float4 w = *reinterpret_cast<const float4*>(by + j0 + e);      // (pairs is a multiple of 8)
              v[u].f[e] = turned(v[u].f[e], w.x, o.f[e], upper ? w.y : -w.y);
              v[u].f[e + 1] = turned(v[u].f[e + 1], w.z, o.f[e + 1], upper ? w.w : -w.w);
            }
          }
        } else if constexpr (ROPE == ROPE_NEIGHBOURS) {
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const int j = col * 4 + e / 2;
            if (j < pairs) {
              const float2 w = by[j];
              const float a = v[u].f[e], b = v[u].f[e + 1];
              v[u].f[e] = turned(a, w.x, b, -w.y);
              v[u].f[e + 1] = turned(b, w.x, a, w.y);
            }
          }
        } else {
          Eight o{};
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int at = col * 8 + e;
            if (at < t.rope.rot) o.f[e] = read1(r.src + (at < pairs ? at + pairs : at - pairs));
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int at = col * 8 + e;
            if (at < t.rope.rot) {
              const float2 w = by[at < pairs ? at : at - pairs];
              v[u].f[e] = turned(v[u].f[e], w.x, o.f[e], at < pairs ? -w.y : w.y);
            }
          }
        }
      }
      if (r.kind == 0 || !CACHE) {
        const TokenHeads& to = r.kind == 0 ? t.q_out : t.k_out;
        if (on) write8(static_cast<T*>(to.x) + (t0 + r.tok) * to.token + r.head * to.head + col * 8, v[u]);
      } else {
        int block, at;
        if (paged_slot(c, t.slots[t0 + r.tok], &block, &at))
          put<C, LANES>(r.kind == 1 ? c.k : c.v, v[u], row_at(c, block, r.head, at), scale_at(c, block, r.head, at), col, on);
      }
    }
  }
}

// A workgroup has rows of one head of an instance; the list has an entry for each, the slots one for all heads.
template <typename T, typename C, int LANES, bool PAST>
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
  if (on) kv = read8<PAST>(k + from);
  if (on && v) vv = read8<PAST>(v + from);
  const int64_t to = row_at(c, block, head, row), scale_to = scale_at(c, block, head, row);
  put<C, LANES>(c.k, kv, to, scale_to, col, on);
  if (v) put<C, LANES>(c.v, vv, to, scale_to, col, on);
}

template <typename T, typename C, int LANES, bool PAST>
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
      else x = read8<PAST>(static_cast<const C*>(plane.x) + at);
    }
    write8<PAST>(out + r * c.d + col * 8, x);
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

int rope_kind(const RopeArgs& r) { return !r.inv_freq ? ROPE_NONE : r.interleaved ? ROPE_NEIGHBOURS : r.rot % 16 == 0 ? ROPE_PIECES : ROPE_ANY; }

template <typename T, typename C, int LANES, bool CACHE>
hipError_t token_rows(const TokenCall& t, const PagedView& c, hipStream_t st) {
  constexpr int ROWS = ROWS_THREADS / LANES;
  const int all = t.q.heads + t.k.heads + t.v.heads;
  // Few tokens: a row a group, so that the call is as short as it can be; more: all heads of a token to a workgroup, of two, of four, whose sines and cosines
  // and first reads are then made together.  us, 40 heads of d = 128: 512 tokens 5.1, as later ones 5.9; 2048 12.4 : 10.9 : 12.5; 4096 20.2 : 17.9 : 16.8 : 20.3;
  // 16381 73.2 : 74.3 : 73.6 : 72.8
  const bool few = t.n_tokens <= 512;
  const int tokens_each = t.n_tokens <= 2048 ? 1 : t.n_tokens <= 8192 ? 2 : 4, rows_each = few ? ROWS : (all + ROWS - 1) / ROWS * ROWS;
  const dim3 grid((unsigned)((t.n_tokens + tokens_each - 1) / tokens_each), (unsigned)((all + rows_each - 1) / rows_each));
  const bool past = t.n_tokens * all * t.d * (int64_t)sizeof(T) >= MANY_BYTES;
  const auto start = [&](auto rope) {
    if (past) hipLaunchKernelGGL((token_rows_kernel<T, C, LANES, rope(), CACHE, true>), grid, dim3(ROWS_THREADS), 0, st, t, c, tokens_each, rows_each);
    else hipLaunchKernelGGL((token_rows_kernel<T, C, LANES, rope(), CACHE, false>), grid, dim3(ROWS_THREADS), 0, st, t, c, tokens_each, rows_each);
  };
  switch (rope_kind(t.rope)) {
    case ROPE_NONE: start(std::integral_constant<int, ROPE_NONE>{}); break;
    case ROPE_PIECES: start(std::integral_constant<int, ROPE_PIECES>{}); break;
    case ROPE_NEIGHBOURS: start(std::integral_constant<int, ROPE_NEIGHBOURS>{}); break;
    default: start(std::integral_constant<int, ROPE_ANY>{});
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
      const auto start = [&](auto past) {
        hipLaunchKernelGGL((paged_compact_kernel<T, Of<decltype(numbers)>, lanes(), past()>), dim3((most + ROWS - 1) / ROWS, c.Hkv, n), dim3(ROWS_THREADS), 0, st, c,
                           L, lay, tab, inst0, static_cast<const T*>(k), static_cast<const T*>(v), idx, slots);
      };
      int64_t rows_kept = 0;
      for (int i = 0; i < n; ++i) rows_kept += tab.bk[i];
      if (2 * rows_kept * c.Hkv * c.d * (int64_t)sizeof(T) >= MANY_BYTES) start(std::true_type{});
      else start(std::false_type{});
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
      const auto start = [&](auto past) {
        hipLaunchKernelGGL((paged_load_kernel<T, Of<decltype(numbers)>, lanes(), past()>), dim3((unsigned)((n_rows + ROWS - 1) / ROWS)), dim3(ROWS_THREADS), 0, st, c,
                           n_rows, slots, static_cast<T*>(k), static_cast<T*>(v));
      };
      if (2 * n_rows * c.d * (int64_t)sizeof(T) >= MANY_BYTES / 4) start(std::true_type{});
      else start(std::false_type{});
      return hipGetLastError();
    });
  });
}

}  // namespace laq
