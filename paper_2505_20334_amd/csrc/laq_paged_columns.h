// What the attention kernels over the paged cache share: requests and their columns of score rows, numbers of the cache as they are read, and outputs.
#pragma once

#include <type_traits>

#include "laq_find.h"
#include "laq_paged.h"

namespace laq {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float MINUS_INF = -__builtin_inff();

__device__ __forceinline__ uint32_t pack2(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2)); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A request of the call.
struct Request {
  int token0, tokens, held;              // tokens 0: none, or numbers that make no sense; held: rows of the cache
};
__device__ __forceinline__ Request request_of(const PagedAttention& a, int block_rows, int i) {
  Request r{i, 1, 0};
  if (a.start) {
    const int64_t t0 = a.start[i], t1 = a.start[i + 1];
    r.token0 = (int)t0;
    r.tokens = t0 < 0 || t1 <= t0 || t1 > a.n_tokens ? 0 : (int)(t1 - t0);
  }
  r.held = max(0, min(a.rows[i], a.blocks_per_inst * block_rows));
  return r;
}
__device__ __forceinline__ int tiles_of(const Request& r, int G, int tile) { return (int)(((int64_t)r.tokens * G + tile - 1) / tile); }

// Where the columns of a request begin if every column has a workgroup: a request of R score rows has ceil(R / tile) columns, and floor(R' / tile) + i, with R'
// score rows and i requests before it, leaves at least that many between one request and the next.
__device__ __forceinline__ int64_t first_column(const PagedAttention& a, int G, int tile, int i) {
  return a.start ? (int64_t)a.start[i] * G / tile + i : (int64_t)i * ((G + tile - 1) / tile);
}
// The last request that begins at column `slot` or before it: 64 looked at at a time.
__device__ __forceinline__ int find_request(const PagedAttention& a, int G, int tile, int slot) {
  if (!a.start) return min(slot / ((G + tile - 1) / tile), a.n - 1);
  Find f{0, a.n};
  const int lane = threadIdx.x & 63;
  while (f.n > 1) {
    const bool before = f.looks(lane) && first_column(a, G, tile, f.lo + lane * f.step()) <= slot;
    f.narrow((int)__popcll(__ballot(before)));
  }
  return uniform(f.lo);
}

// What a column is: a tile of score rows of a request.
struct Column {
  int row0, rows;                        // its first score row in the request, and their number (0: no such column)
  int token0, tokens, held;              // of the request
  __device__ int last(int row, int G) const { return held - tokens + (row0 + row) / G; }      // the last key that a score row sees
  __device__ int keys(int G) const { return max(0, last(rows - 1, G) + 1); }
};
__device__ __forceinline__ Column column_of(const Request& r, int G, int tile, int64_t t) {
  const int64_t row0 = t * tile, all = (int64_t)r.tokens * G;
  if (t < 0 || row0 >= all) return Column{0, 0, 0, 1, 0};
  return Column{(int)row0, (int)min((int64_t)tile, all - row0), r.token0, r.tokens, r.held};
}

// N numbers of the cache in a row, as they lie.
template <typename E, int N> struct Raw;
template <> struct Raw<float, 4> { u32x4 x; };
template <> struct Raw<uint16_t, 8> { u32x4 x; };
template <> struct Raw<uint16_t, 4> { u32x2 x; };
template <> struct Raw<E4m3, 8> { u32x2 x; };
template <> struct Raw<E4m3, 4> { uint32_t x; };

template <typename R> __device__ __forceinline__ void clear(R& r) { r.x = {}; }

// As pairs of bf16 (scale: of 8 bits).
__device__ __forceinline__ uint32_t pair_of(uint32_t codes, float scale, bool high) {
  return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))
              : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false));
}
__device__ __forceinline__ u32x4 pairs(const Raw<uint16_t, 8>& r, float) { return r.x; }
__device__ __forceinline__ u32x2 pairs(const Raw<uint16_t, 4>& r, float) { return r.x; }
__device__ __forceinline__ u32x4 pairs(const Raw<E4m3, 8>& r, float s) {
  return u32x4{pair_of(r.x[0], s, false), pair_of(r.x[0], s, true), pair_of(r.x[1], s, false), pair_of(r.x[1], s, true)};
}
__device__ __forceinline__ u32x2 pairs(const Raw<E4m3, 4>& r, float s) { return u32x2{pair_of(r.x, s, false), pair_of(r.x, s, true)}; }
// As fp32.
__device__ __forceinline__ f32x4 floats(const Raw<float, 4>& r) { return __builtin_bit_cast(f32x4, r.x); }

// Infinities and NaN among numbers of V.
template <typename E, int N>
__device__ __forceinline__ bool has_odd(const Raw<E, N>& r, uint32_t scale) {
  bool odd = false;
  if constexpr (std::is_same<E, float>::value) {
#pragma unroll
    for (int i = 0; i < 4; ++i) odd |= (r.x[i] & 0x7f800000u) == 0x7f800000u;
  } else if constexpr (std::is_same<E, uint16_t>::value) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) odd |= (r.x[i] & 0x7f800000u) == 0x7f800000u || (r.x[i] & 0x7f80u) == 0x7f80u;
  } else {
    odd = scale == 255u;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint32_t w;
      if constexpr (N == 4) w = r.x;
      else w = r.x[i / 4];
      odd |= (w >> (8 * (i % 4)) & 0x7fu) == 0x7fu;
    }
  }
  return odd;
}
// 0 in their place.
__device__ __forceinline__ uint32_t without_odd(uint32_t w, float) { return (w & 0x7f800000u) == 0x7f800000u ? 0u : w; }
__device__ __forceinline__ uint32_t without_odd(uint32_t w, uint16_t) {
  return ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u) | ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu);
}
__device__ __forceinline__ uint32_t without_odd(uint32_t w, E4m3) {
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) r |= (w >> (8 * i) & 0x7fu) == 0x7fu ? 0u : w & 255u << (8 * i);
  return r;
}
template <typename E, int N>
__device__ __forceinline__ void drop_odd(Raw<E, N>& r) {
  if constexpr (sizeof(r.x) == 4) {
    r.x = without_odd(r.x, E{});
  } else {
#pragma unroll
    for (int i = 0; i < (int)sizeof(r.x) / 4; ++i) r.x[i] = without_odd(r.x[i], E{});
  }
}
// A number of a row of V.
__device__ __forceinline__ float number(const float* row, int i, uint32_t) { return row[i]; }
__device__ __forceinline__ float number(const uint16_t* row, int i, uint32_t) { return __uint_as_float((uint32_t)row[i] << 16); }
__device__ __forceinline__ float number(const E4m3* row, int i, uint32_t scale) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(row[i].x, false);
  return a[0] * e4m3_scale_value(scale);
}

// A tile's rows, read through a buffer descriptor: reads behind its end give zeros without memory traffic, and nothing at all is read of a tile that is not
// there.  So the reads of a step are issued whatever the step has, and the wait for a step's keys can leave those of the next one on their way (with
// branches around them it waited for both: 96 requests x 8 heads x 6144 rows 428 us).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_of(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}
template <bool ONCE, typename R>
__device__ __forceinline__ void fetch(R& r, __amdgpu_buffer_rsrc_t tile, int at) {
  constexpr int PAST = ONCE ? 2 : 0;                         // nt: 128 requests of 1000 to 8192 rows 371 us, without 416
  if constexpr (sizeof(r.x) == 16) r.x = __builtin_bit_cast(decltype(r.x), __builtin_amdgcn_raw_buffer_load_b128(tile, at, 0, PAST));
  else if constexpr (sizeof(r.x) == 8) r.x = __builtin_bit_cast(decltype(r.x), __builtin_amdgcn_raw_buffer_load_b64(tile, at, 0, PAST));
  else r.x = __builtin_amdgcn_raw_buffer_load_b32(tile, at, 0, PAST);
}

// Four numbers of the output from sums and the sum of weights, and the logarithm.
template <typename Q>
__device__ __forceinline__ void put_out(const PagedView& c, const PagedAttention& a, const Column& col, int head, int G, int r, int at, float m, float z, f32x4 y) {
  const int row = col.row0 + r;
  const int64_t to = (int64_t)(col.token0 + row / G) * a.Hq + head * G + row % G;
  const float inv = z == 0.f ? 0.f : 1.f / z;
  if (at == 0 && a.lse) a.lse[to] = z == 0.f ? MINUS_INF : (__builtin_amdgcn_logf(z) + m * a.scale2) * 0.69314718055994530942f;
  if constexpr (std::is_same<Q, float>::value)
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to * c.d + at) = y * inv;
  else
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + to * c.d + at) = u32x2{pack2(y[0] * inv, y[1] * inv), pack2(y[2] * inv, y[3] * inv)};
}

// a / b of numbers that are not negative, in 32 bits where they fit (64 take a hundred instructions).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (uint64_t)(a | b) >> 32 ? (int64_t)((uint64_t)a / (uint64_t)b) : (int64_t)((uint32_t)a / (uint32_t)b);
}

// Where a share begins.
struct Found {
  Request r;
  int request, head, tile, turn;
};

// Partial sums m (a score, not scaled), z and y of score rows, joined.
__device__ __forceinline__ void join(float& m, float& z, f32x4& y, float m2, float z2, f32x4 y2, float scale2) {
  const float top = fmaxf(m, m2);
  const float by = m == top ? 1.f : __builtin_amdgcn_exp2f((m - top) * scale2), by2 = m2 == top ? 1.f : __builtin_amdgcn_exp2f((m2 - top) * scale2);
  m = top;
  z = z * by + z2 * by2;
  y = y * by + y2 * by2;
}

// Written through to the device's memory, and read from there.
__device__ __forceinline__ void store_pair(void* p, float a, float b) {
  __hip_atomic_store(static_cast<unsigned long long*>(p), (unsigned long long)__float_as_uint(b) << 32 | __float_as_uint(a), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 load_pair(const void* p) {
  const unsigned long long v = __hip_atomic_load(static_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return f32x2{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}

// Where a workgroup's share of a call stands.  All keys of all columns are a line of turns (of TURN keys), request after request, of each its heads, of each its
// tiles, of each the turns of the request's rows (a column of a request's earlier tokens has turns in which it sees nothing); shares differ by a turn at most.
struct Share {
  Request req;
  int request, head, turn, shares, more;                     // turn: in the column; more: shares that have a turn more than the others
  int64_t tile, left, each, begin;                           // left: turns of the share from here on; each: of a share; begin: of the column on the line
  __device__ int place() const { return 2 * blockIdx.x + (turn == 0); }      // of the range's partial results
  __device__ int share_of(int64_t x) const {
    const int64_t longer = (each + 1) * more;
    return (int)(x < longer ? quotient(x, each + 1) : more + quotient(x - longer, each));
  }
};
template <int TURN> __device__ __forceinline__ int turns_of(const Request& r) { return r.held / TURN + (r.held % TURN != 0 || r.held == 0); }
template <int WAVES> struct ShareScan {
  int64_t waves[WAVES][2];
  Found found;
};
// The workgroup's first range, or false if it has none.
template <int THREADS, int TURN>
__device__ __forceinline__ bool first_range(const PagedView& c, const PagedAttention& a, int G, const AttPlan& p, ShareScan<THREADS / 64>& scan, Share& s) {
  const int H = c.Hkv;
  s.turn = s.more = s.shares = 0;
  s.left = 1;
  s.each = s.begin = 0;
  if (!p.shares) {
    const int slot = blockIdx.x / H;
    s.head = blockIdx.x % H;
    s.request = find_request(a, G, p.tile, slot);
    s.tile = slot - first_column(a, G, p.tile, s.request);
    s.req = request_of(a, c.block_rows, s.request);
    return true;
  }
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int per = (a.n + THREADS - 1) / THREADS, i0 = (int)min((int64_t)a.n, (int64_t)threadIdx.x * per), i1 = (int)min((int64_t)a.n, (int64_t)i0 + per);
  int64_t mine = 0, tiles = 0;
  for (int i = i0; i < i1; ++i) {
    const Request r = request_of(a, c.block_rows, i);
    const int64_t t = tiles_of(r, G, p.tile);
    tiles += t;
    mine += t * H * turns_of<TURN>(r);
  }
  // sums over the lanes before this one, then over the waves
  int64_t upto = mine;
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const int64_t below = __shfl_up(upto, m);
    if (lane >= m) upto += below;
    tiles += __shfl_xor(tiles, m);
  }
  if (lane == 63) {
    scan.waves[wave][0] = upto;
    scan.waves[wave][1] = tiles;
  }
  if (threadIdx.x == 0) scan.found.request = -1;
  __syncthreads();
  int64_t before = upto - mine, total = 0, all_tiles = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) before += scan.waves[w][0];
    total += scan.waves[w][0];
    all_tiles += scan.waves[w][1];
  }
  if (all_tiles > p.columns || total <= 0) return false;     // (a start that makes no sense)
  s.shares = (int)min((int64_t)p.shares, total);
  const int w = blockIdx.x;
  if (w >= s.shares) return false;
  s.each = quotient(total, s.shares);
  s.more = (int)(total - s.each * s.shares);
  const int64_t x0 = s.each * w + min(w, s.more);
  s.left = s.each + (w < s.more);
  if (x0 >= before && x0 < before + mine) {
    int64_t at = before;
    for (int i = i0; i < i1; ++i) {
      const Request r = request_of(a, c.block_rows, i);
      const int turns = turns_of<TURN>(r), tiles_here = tiles_of(r, G, p.tile);
      const int64_t all = (int64_t)turns * H * tiles_here;
      if (x0 < at + all) {
        const int64_t column = quotient(x0 - at, turns);
        const int turn_at = (int)(x0 - at - column * turns), head_at = (int)column / tiles_here;        // (columns of a request: less than 2^31)
        scan.found = Found{r, i, head_at, (int)column - head_at * tiles_here, turn_at};
        break;
      }
      at += all;
    }
  }
  __syncthreads();
  if (scan.found.request < 0) return false;
  s.req = Request{uniform(scan.found.r.token0), uniform(scan.found.r.tokens), uniform(scan.found.r.held)};
  s.request = uniform(scan.found.request);
  s.head = uniform(scan.found.head);
  s.tile = uniform(scan.found.tile);
  s.turn = uniform(scan.found.turn);
  s.begin = x0 - s.turn;
  return true;
}
// The next column of the share, or false at its end.
template <int TURN>
__device__ __forceinline__ bool next_column(const PagedView& c, const PagedAttention& a, int G, int tile, int turns, int turns_here, Share& s) {
  s.left -= turns_here;
  if (s.left <= 0) return false;
  s.begin += turns;
  s.turn = 0;
  if (++s.tile < tiles_of(s.req, G, tile)) return true;
  s.tile = 0;
  if (++s.head < c.Hkv) return true;
  s.head = 0;
  do {
    if (++s.request >= a.n) return false;
    s.req = request_of(a, c.block_rows, s.request);
  } while (s.req.tokens == 0);
  return true;
}

// The workgroup has stored its range of a column: joins the ranges if it finds that all of them are there.  U ranges are asked for at a time; lds: room for THREADS * 6 numbers.
template <typename Q, int THREADS, int U>
__device__ __forceinline__ void join_ranges(const PagedView& c, const PagedAttention& a, const Partials& part, const Share& s, const Column& col, int G, int tile, int turns,
                                            float* lds) {
  const int first = s.share_of(s.begin), count = s.share_of(s.begin + turns - 1) - first + 1;
  const auto place_of = [&](int k) { return 2 * (first + k) + (k == 0); };
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (what this wave stored has arrived)
  __syncthreads();
  if (threadIdx.x == 0) __hip_atomic_store(part.marks + s.place(), part.nonce, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  bool all = true;
  for (int k = threadIdx.x; k < count; k += THREADS)
    all &= __hip_atomic_load(part.marks + place_of(k), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == part.nonce;
  if (!__syncthreads_and(all)) return;
  for (int k = threadIdx.x; k < count; k += THREADS) __hip_atomic_store(part.marks + place_of(k), 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // four channels of a row a thread, and as many groups of ranges as there are threads for
  const int per = c.d / 4, items = col.rows * per, groups = max(1, min(count, THREADS / items));
  f32x2* const lds_mz = reinterpret_cast<f32x2*>(lds + 4 * THREADS);
  for (int i0 = 0; i0 < items; i0 += groups > 1 ? items : THREADS) {
    const int grp = groups > 1 ? threadIdx.x / items : 0, item = groups > 1 ? threadIdx.x % items : i0 + threadIdx.x;
    const int r = item / per, at = (item - r * per) * 4;
    float top = MINUS_INF, z = 0.f;
    f32x4 y{};
    if (item < items && grp < groups) {
      for (int k = grp; k < count; k += U * groups) {
        f32x2 mz[U], s0[U], s1[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t row = (int64_t)place_of(min(k + u * groups, count - 1)) * tile + r;
          mz[u] = load_pair(part.mz + row);
          s0[u] = load_pair(part.sums + row * c.d + at);
          s1[u] = load_pair(part.sums + row * c.d + at + 2);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (k + u * groups < count) join(top, z, y, mz[u][0], mz[u][1], f32x4{s0[u][0], s0[u][1], s1[u][0], s1[u][1]}, a.scale2);
      }
    }
    if (groups > 1) {
      *reinterpret_cast<f32x4*>(lds + 4 * threadIdx.x) = y;
      lds_mz[threadIdx.x] = f32x2{top, z};
      __syncthreads();
      for (int k = 1; item < items && grp == 0 && k < groups; ++k)
        join(top, z, y, lds_mz[k * items + item][0], lds_mz[k * items + item][1], *reinterpret_cast<const f32x4*>(lds + 4 * (k * items + item)), a.scale2);
    }
    if (grp == 0 && item < items) put_out<Q>(c, a, col, s.head, G, r, at, top, z, y);
  }
}

}  // namespace

}  // namespace laq
