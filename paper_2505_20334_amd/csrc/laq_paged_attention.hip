// Attention over the paged cache of 32, 16 or 8 bits (include/laq_cache.h: laq_cache_attention).
//
// A column is a KV head of a request and a tile of its score rows (row r = query head r % G of the group of the request's token r / G).  A workgroup has
// a range of a column's keys; its waves take 16 * KT keys each in turn, every wave for all rows of the tile, with its own reference m, sum z and sums O
// (one pass, exponentials of s - m; m moves only when a score is more than 8 above it, so that the usual step has no maximum over lanes).
// The waves are folded at the end through LDS, the ranges of a column by a second launch, in a fixed order.
//
// No LDS on the way of K and V.  Products have the keys as the first operand's rows, so that a lane has four keys of one score row (column n =
// lane % 16, keys 4g .. 4g + 3 of a tile for lane group g = lane / 16), and all that belongs to a score row lies in lanes n, n + 16, n + 32, n + 48:
//   S^T = K Q^T   a lane reads pieces of one key row, in the order of the operand (the sum over channels may take them in any order, Q the same)
//   O^T = V^T P^T P^T is where S^T left it: a lane group's keys are, by definition, its part of the keys summed over.  bf16 (16 x 16 x 32): a lane needs
//                 eight keys of one channel; it reads eight channels of its eight keys, and a permutation of 8 x 8 numbers in registers, two a
//                 instruction, makes the operands of eight products.  fp32 (16 x 16 x 4): one key a lane, so the pieces are operands as they are
// A lane's pieces of V are VN channels: its product row m of product e of piece h is channel (16 h + m) VN + e.
#include <type_traits>

#include "laq_paged.h"

namespace laq {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int ATT_WAVES = 4, ATT_THREADS = 64 * ATT_WAVES;
constexpr int JOIN_THREADS = 256;
constexpr float MINUS_INF = -__builtin_inff();

__device__ __forceinline__ uint32_t pack2(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2)); }
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 acc) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, acc, 0, 0, 0); }

// How the launch is cut, from what the host knows.
struct AttPlan {
  int32_t parts, part_rows;              // a column in parts of part_rows keys, `parts` at most (the last one takes what is left)
  int32_t tile;                          // score rows of a column
  int32_t slots;                         // columns of a KV head over all requests, at most
};

// Where the columns of a request begin: a request of R score rows has ceil(R / tile) columns, and floor(R' / tile) + i, with R' score rows and i requests
// before it, leaves at least that many between one request and the next.
__device__ __forceinline__ int64_t first_column(const PagedAttention& a, int G, int tile, int i) {
  return a.start ? (int64_t)a.start[i] * G / tile + i : (int64_t)i * ((G + tile - 1) / tile);
}

// What a column is.
struct Column {
  int request, row0, rows;               // its first score row in the request, and their number (0: no such column)
  int token0, tokens;                    // of the request
  int held;                              // rows of the cache
  __device__ int last(int row, int G) const { return held - tokens + (row0 + row) / G; }      // the last key that a score row sees
  __device__ int keys(int G) const { return rows ? max(0, last(rows - 1, G) + 1) : 0; }
};
__device__ __forceinline__ Column find_column(const PagedAttention& a, int block_rows, int G, int tile, int slot) {
  Column c{0, 0, 0, 0, 1, 0};
  if (a.start) {
    // the last request that begins at `slot` or before it: 64 looked at at a time
    int lo = 0, n = a.n;
    const int lane = threadIdx.x & 63;
    while (n > 1) {
      const int step = (n + 63) / 64, i = lo + lane * step;
      const bool before = lane * step < n && first_column(a, G, tile, i) <= slot;
      const int k = __popcll(__ballot(before)) - 1;
      const int at = max(k, 0) * step;
      lo += at;
      n = min(step, n - at);
      if (n < 1) n = 1;
    }
    c.request = __builtin_amdgcn_readfirstlane(min(lo, a.n - 1));
    const int64_t t0 = a.start[c.request], t1 = a.start[c.request + 1];
    if (t0 < 0 || t1 <= t0 || t1 > a.n_tokens) return c;
    c.token0 = (int)t0;
    c.tokens = (int)(t1 - t0);
  } else {
    c.request = slot / ((G + tile - 1) / tile);
    if (c.request >= a.n) return c;
    c.token0 = c.request;
  }
  const int64_t row0 = (slot - first_column(a, G, tile, c.request)) * tile, all = (int64_t)c.tokens * G;
  if (row0 < 0 || row0 >= all) return c;
  c.row0 = (int)row0;
  c.rows = (int)min((int64_t)tile, all - row0);
  c.held = max(0, min(a.rows[c.request], a.blocks_per_inst * block_rows));
  return c;
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
__device__ __forceinline__ f32x4 floats(const Raw<float, 4>& r, float) { return __builtin_bit_cast(f32x4, r.x); }
__device__ __forceinline__ f32x4 floats(const Raw<uint16_t, 4>& r, float) {
  return __builtin_bit_cast(f32x4, (u32x4{r.x[0] << 16, r.x[0] & 0xffff0000u, r.x[1] << 16, r.x[1] & 0xffff0000u}));
}
__device__ __forceinline__ f32x4 floats(const Raw<E4m3, 4>& r, float s) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(r.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(r.x, true);
  return f32x4{a[0] * s, a[1] * s, b[0] * s, b[1] * s};
}

// A number of a row of V.
__device__ __forceinline__ float number(const float* row, int i, uint32_t) { return row[i]; }
__device__ __forceinline__ float number(const uint16_t* row, int i, uint32_t) { return __uint_as_float((uint32_t)row[i] << 16); }
__device__ __forceinline__ float number(const E4m3* row, int i, uint32_t scale) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(row[i].x, false);
  return a[0] * e4m3_scale_value(scale);
}

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
// Q: the queries' numbers (and what the products are made in), E: the cache's, D: head sizes up to D, NT: 16 score rows NT times.
template <typename Q, typename E, int D, int NT>
struct Kinds {
  static constexpr bool F32 = std::is_same<Q, float>::value, SCALED = std::is_same<E, E4m3>::value;
  static constexpr int KT = F32 ? 1 : 2;                     // tiles of 16 keys a step
  static constexpr int KN = F32 ? 4 : 8, KP = D / (4 * KN);  // numbers of a piece of K; pieces of a lane's key row
  static constexpr int VN = F32 || D == 64 ? 4 : 8, VP = D / (16 * VN);
  static constexpr int OT = D / 16;                          // output tiles
  static constexpr int PAD = D + 4;
};

// The keys of a step as they came from memory.
template <typename K, typename E>
struct StepKeys {
  Raw<E, K::KN> k[K::KT][K::KP];
  Raw<E, K::VN> v[K::KT][4][K::VP];
  uint32_t ks[K::KT], vs[K::KT];                             // SCALED: of this lane's key row; of its four keys of V
  bool there[K::KT];
};

// Partial results of the ranges of a column: [slot][head][part][tile rows] of m (as a score, not scaled) and z, and as many rows of d sums.
struct Partials {
  float2* mz;
  float* sums;
};

template <typename Q, typename E, int D, int NT>
__global__ __launch_bounds__(ATT_THREADS) void paged_attention_kernel(PagedView c, PagedAttention a, AttPlan p, Partials part) {
  using K = Kinds<Q, E, D, NT>;
  const int H = c.Hkv, G = a.Hq / H;
  const int head = blockIdx.x % H, pi = blockIdx.x / H % p.parts, slot = blockIdx.x / H / p.parts;
  const Column col = find_column(a, c.block_rows, G, p.tile, slot);
  const int keys = col.keys(G), from = pi * p.part_rows;
  const bool cut = p.parts > 1 && keys > p.part_rows;        // this column is in parts
  if (col.rows == 0 || (pi > 0 && from >= keys)) return;
  const int to = pi == p.parts - 1 ? keys : min(keys, from + p.part_rows);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;

  // the score rows of this lane's columns
  int last[NT];
  u32x4 q[NT][K::KP];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = 16 * t + n;
    const bool on = r < col.rows;
    last[t] = on ? col.last(r, G) : 0x7fffffff;
    const int rr = col.row0 + (on ? r : 0);
    const Q* src = static_cast<const Q*>(a.q.x) + (int64_t)(col.token0 + rr / G) * a.q.token + (int64_t)(head * G + rr % G) * a.q.head;
#pragma unroll
    for (int i = 0; i < K::KP; ++i) {
      const int at = (4 * i + g) * K::KN;
      q[t][i] = on && at < c.d ? *reinterpret_cast<const u32x4*>(src + at) : u32x4{};
    }
  }
  const int first_last = col.last(0, G);                     // all rows see the keys up to here

  f32x4 o[NT][K::OT];
  float m[NT], z[NT], above[NT], less[NT];                   // reference; sum; the score that moves the reference; what is subtracted, scaled
  const float margin = 8.f / a.scale2;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m[t] = above[t] = MINUS_INF;
    z[t] = less[t] = 0.f;
#pragma unroll
    for (int i = 0; i < K::OT; ++i) o[t][i] = f32x4{};
  }

  bool odd = false;                                          // an infinity or a NaN in V that not every row sees

  // where the lane's pieces lie behind a tile's first row (channels beyond d: those of the row's beginning, for nobody)
  int32_t k_at[K::KP], v_at[K::VP];
#pragma unroll
  for (int i = 0; i < K::KP; ++i) {
    const int at = (4 * i + g) * K::KN;
    k_at[i] = (int32_t)(n * c.row) + (at < c.d ? at : 0);
  }
#pragma unroll
  for (int i = 0; i < K::VP; ++i) {
    const int at = (16 * i + n) * K::VN;
    v_at[i] = (int32_t)(4 * g * c.row) + (at < c.d ? at : 0);
  }
  const int32_t row = (int32_t)c.row;
  const E *kx = static_cast<const E*>(c.k.x) + head * c.head, *vx = static_cast<const E*>(c.v.x) + head * c.head;
  typedef __attribute__((address_space(4))) const int32_t* ConstTable;
  const ConstTable table = (ConstTable)(unsigned long long)(a.table + (int64_t)col.request * a.blocks_per_inst);

  // this wave's steps: keys from + (wave + 4 i) * 16 KT on; its place in the blocks moves with it
  constexpr int STEP = 16 * K::KT;
  const auto load = [&](int key, StepKeys<K, E>& s) {
#pragma unroll
    for (int kt = 0; kt < K::KT; ++kt) {
      const uint32_t at = (uint32_t)key + 16 * kt;
      const int page = (int)(at / (uint32_t)c.block_rows), off = (int)(at - (uint32_t)page * c.block_rows);
      const int block = 16 * kt < to - key ? table[page] : -1;
      s.there[kt] = block >= 0 && block < c.n_blocks;
      if (s.there[kt]) {
        const int64_t base = block * c.block + (int64_t)off * c.row;
        const E *kb = kx + base, *vb = vx + base;
#pragma unroll
        for (int i = 0; i < K::KP; ++i) s.k[kt][i] = *reinterpret_cast<const Raw<E, K::KN>*>(kb + k_at[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < K::VP; ++i) s.v[kt][j][i] = *reinterpret_cast<const Raw<E, K::VN>*>(vb + v_at[i] + j * row);
        if constexpr (K::SCALED) {
          const int64_t sc = ((int64_t)block * H + head) * c.block_rows + off;
          s.ks[kt] = c.k.scales[sc + n];
          s.vs[kt] = *reinterpret_cast<const uint32_t*>(c.v.scales + sc + 4 * g);
        }
      } else {
#pragma unroll
        for (int i = 0; i < K::KP; ++i) clear(s.k[kt][i]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < K::VP; ++i) clear(s.v[kt][j][i]);
        s.ks[kt] = s.vs[kt] = 0;
      }
    }
  };

  const auto scale_of_v = [&](const StepKeys<K, E>& s, int kt, int j) { return e4m3_scale_value(s.vs[kt] >> (8 * j) & 255u); };
  const auto compute = [&](int key, StepKeys<K, E>& s) {
    f32x4 x[NT][K::KT];
#pragma unroll
    for (int kt = 0; kt < K::KT; ++kt) {
#pragma unroll
      for (int t = 0; t < NT; ++t) x[t][kt] = f32x4{};
      const float ks = K::SCALED ? e4m3_scale_value(s.ks[kt]) : 1.f;
#pragma unroll
      for (int i = 0; i < K::KP; ++i) {
        if constexpr (K::F32) {
          f32x4 k = floats(s.k[kt][i], ks);
          if (c.d != D && (4 * i + g) * K::KN >= c.d) k = f32x4{};
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[t][kt] = mfma(k[e], __uint_as_float(q[t][i][e]), x[t][kt]);
        } else {
          u32x4 k = pairs(s.k[kt][i], ks);
          if (c.d != D && (4 * i + g) * K::KN >= c.d) k = u32x4{};
#pragma unroll
          for (int t = 0; t < NT; ++t) x[t][kt] = mfma(k, q[t][i], x[t][kt]);
        }
      }
    }
    bool all_there = true;
#pragma unroll
    for (int kt = 0; kt < K::KT; ++kt) all_there &= s.there[kt];
    const bool edge = !all_there || key > first_last - (STEP - 1);   // a key that not every row sees
    const int left = to - key;                                       // (keys of the step as far as `left`; sums with key could pass 2^31)
    if (edge) {
#pragma unroll
      for (int kt = 0; kt < K::KT; ++kt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int at = 16 * kt + 4 * g + j;
          // (keys behind this range belong to nobody here)
#pragma unroll
          for (int t = 0; t < NT; ++t)
            if (!s.there[kt] || at >= left || at > last[t] - key) x[t][kt][j] = MINUS_INF;
        }
    }
    // the reference moves where a score is far above it
    bool far = false;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int kt = 0; kt < K::KT; ++kt)
#pragma unroll
        for (int j = 0; j < 4; ++j) far |= x[t][kt][j] > above[t];
    if (__any(far)) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float most = m[t];
#pragma unroll
        for (int kt = 0; kt < K::KT; ++kt)
#pragma unroll
          for (int j = 0; j < 4; ++j) most = fmaxf(most, x[t][kt][j]);
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        if (most > m[t]) {
          const float by = m[t] == MINUS_INF ? 0.f : __builtin_amdgcn_exp2f((m[t] - most) * a.scale2);
          m[t] = most;
          above[t] = most + margin;
          less[t] = most * a.scale2;
          z[t] *= by;
#pragma unroll
          for (int i = 0; i < K::OT; ++i) o[t][i] *= by;
        }
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int kt = 0; kt < K::KT; ++kt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][kt][j], a.scale2, -less[t]));
          x[t][kt][j] = w;
          z[t] += w;
        }
    // V of keys that some rows do not see: a weight of 0 does not keep an infinity or a NaN out.  They are 0 here, and what rows that see them get is
    // added at the end.  Nothing of keys that nobody sees here
    if (edge) {
#pragma unroll
      for (int kt = 0; kt < K::KT; ++kt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int at = 16 * kt + 4 * g + j;
          if (at > first_last - key) {
            const uint32_t vs = K::SCALED ? s.vs[kt] >> (8 * j) & 255u : 0u;
            bool bad = false;
#pragma unroll
            for (int i = 0; i < K::VP; ++i) bad |= has_odd(s.v[kt][j][i], vs);
            odd |= bad && at < left;
            const bool none = at >= left || vs == 255u;
#pragma unroll
            for (int i = 0; i < K::VP; ++i) {
              if (none) clear(s.v[kt][j][i]);
              else drop_odd(s.v[kt][j][i]);
            }
            if (K::SCALED && none) s.vs[kt] &= ~(255u << (8 * j));
          }
        }
    }
    if constexpr (K::F32) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < K::VP; ++i) {
          const f32x4 v = floats(s.v[0][j][i], K::SCALED ? scale_of_v(s, 0, j) : 1.f);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int t = 0; t < NT; ++t) o[t][i * 4 + e] = mfma(v[e], x[t][0][j], o[t][i * 4 + e]);
        }
    } else {
      u32x4 w[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t)
        w[t] = u32x4{pack2(x[t][0][0], x[t][0][1]), pack2(x[t][0][2], x[t][0][3]), pack2(x[t][1][0], x[t][1][1]), pack2(x[t][1][2], x[t][1][3])};
#pragma unroll
      for (int i = 0; i < K::VP; ++i) {
        // [key][channel pair] to [channel][key pair]
        using P = decltype(pairs(s.v[0][0][0], 1.f));
        P v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = pairs(s.v[j / 4][j % 4][i], K::SCALED ? scale_of_v(s, j / 4, j % 4) : 1.f);
#pragma unroll
        for (int e = 0; e < K::VN; ++e) {
          u32x4 f;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            f[j] = __builtin_amdgcn_perm(v[2 * j + 1][e / 2], v[2 * j][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int t = 0; t < NT; ++t) o[t][i * K::VN + e] = mfma(f, w[t], o[t][i * K::VN + e]);
        }
      }
    }
  };

  // two steps at a time: one's keys are on their way while the other's are used
  {
    StepKeys<K, E> s0, s1;
    int key = to - from > wave * STEP ? from + wave * STEP : to;
    constexpr int TURN = STEP * ATT_WAVES;
    if (key < to) load(key, s0);
    while (key < to) {
      if (to - key > TURN) load(key + TURN, s1);
      compute(key, s0);
      if (to - key <= TURN) break;
      key += TURN;
      if (to - key > TURN) load(key + TURN, s0);
      compute(key, s1);
      if (to - key <= TURN) break;
      key += TURN;
    }
  }

  // the waves' sums, score rows of 16 at a time
  __shared__ float sums[ATT_WAVES][16][K::PAD];
  __shared__ float2 marks[ATT_WAVES][16];
  __shared__ bool odds[ATT_WAVES];
  const bool wave_odd = __any(odd);
  if (lane == 0) odds[wave] = wave_odd;
  const int64_t place = (((int64_t)slot * H + head) * p.parts + pi) * p.tile;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float zt = z[t];
    zt += __shfl_xor(zt, 16);
    zt += __shfl_xor(zt, 32);
    if (t) __syncthreads();
    if (g == 0) marks[wave][n] = float2{m[t], zt};
#pragma unroll
    for (int i = 0; i < K::VP; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < K::VN; ++e) sums[wave][n][(16 * i + 4 * g + j) * K::VN + e] = o[t][i * K::VN + e][j];
    __syncthreads();
    constexpr int EACH = 4, PER = D / EACH;
    for (int i = threadIdx.x; i < 16 * PER; i += ATT_THREADS) {
      const int rr = i / PER, at = i % PER * EACH, r = 16 * t + rr;
      if (r >= col.rows || at >= c.d) continue;
      float top = MINUS_INF, Z = 0.f;
#pragma unroll
      for (int w = 0; w < ATT_WAVES; ++w) top = fmaxf(top, marks[w][rr].x);
      f32x4 y{};
#pragma unroll
      for (int w = 0; w < ATT_WAVES; ++w) {
        const float2 mz = marks[w][rr];
        // (a wave without keys: 0, also where all are; an infinite or undefined score makes a NaN of z already)
        const float by = mz.x == MINUS_INF ? 0.f : mz.x == top ? 1.f : __builtin_amdgcn_exp2f((mz.x - top) * a.scale2);
        Z += mz.x == MINUS_INF && mz.y == mz.y ? 0.f : by == 0.f && mz.y != mz.y ? mz.y : mz.y * by;
#pragma unroll
        for (int e = 0; e < EACH; ++e) y[e] += mz.x == MINUS_INF ? 0.f : sums[w][rr][at + e] * by;
      }
      bool any_odd = false;
#pragma unroll
      for (int w = 0; w < ATT_WAVES; ++w) any_odd |= odds[w];
      if (any_odd) {
        const int upto = min(to - 1, col.last(r, G));
        for (int key = max(from, first_last + 1); key <= upto; ++key) {
          const int page = (int)((uint32_t)key / (uint32_t)c.block_rows), off = key - page * c.block_rows, block = table[page];
          if (block < 0 || block >= c.n_blocks) continue;
          const E* v = vx + block * c.block + (int64_t)off * c.row;
          const uint32_t vs = K::SCALED ? c.v.scales[((int64_t)block * H + head) * c.block_rows + off] : 0u;
          for (int e = 0; e < EACH; ++e) {
            const float f = number(v, at + e, vs);
            if (f - f != 0.f) y[e] += f;
          }
        }
      }
      if (cut) {
        if (at == 0) part.mz[place + r] = float2{top, Z};
        *reinterpret_cast<f32x4*>(part.sums + (place + r) * c.d + at) = y;
        continue;
      }
      const int row_in = col.row0 + r;
      const int64_t to_row = (int64_t)(col.token0 + row_in / G) * a.Hq + head * G + row_in % G;
      const float inv = Z == 0.f ? 0.f : 1.f / Z;
      if (at == 0 && a.lse) a.lse[to_row] = Z == 0.f ? MINUS_INF : (__builtin_amdgcn_logf(Z) + top * a.scale2) * 0.69314718055994530942f;
      if constexpr (K::F32) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to_row * c.d + at) = y * inv;
      } else {
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + to_row * c.d + at) = u32x2{pack2(y[0] * inv, y[1] * inv), pack2(y[2] * inv, y[3] * inv)};
      }
    }
  }
}

// The parts of a score row, in their order: a workgroup has one row, its threads four channels each of every eighth (or so) part.
template <typename Q>
__global__ __launch_bounds__(JOIN_THREADS) void paged_join_kernel(PagedView c, PagedAttention a, AttPlan p, Partials part) {
  const int H = c.Hkv, G = a.Hq / H;
  const int r = blockIdx.x % p.tile, head = blockIdx.x / p.tile % H, slot = blockIdx.x / p.tile / H;
  const Column col = find_column(a, c.block_rows, G, p.tile, slot);
  const int keys = col.keys(G);
  if (r >= col.rows || keys <= p.part_rows) return;
  const int parts = min(p.parts, (keys + p.part_rows - 1) / p.part_rows);
  __shared__ f32x4 sums[JOIN_THREADS];
  __shared__ float zs[JOIN_THREADS];
  const int lanes = c.d / 4, groups = JOIN_THREADS / lanes, mine = threadIdx.x / lanes, at = threadIdx.x % lanes * 4;
  const int64_t place = ((int64_t)slot * H + head) * p.parts * p.tile + r;
  float top = MINUS_INF;
  for (int i = 0; i < parts; ++i) top = fmaxf(top, part.mz[place + (int64_t)i * p.tile].x);
  f32x4 y{};
  float Z = 0.f;
  if (mine < groups) {
    for (int i = mine; i < parts; i += groups) {
      const int64_t row = place + (int64_t)i * p.tile;
      const float2 mz = part.mz[row];
      const f32x4 v = *reinterpret_cast<const f32x4*>(part.sums + row * c.d + at);
      const float by = mz.x == MINUS_INF ? 0.f : mz.x == top ? 1.f : __builtin_amdgcn_exp2f((mz.x - top) * a.scale2);
      Z += by == 0.f ? (mz.y != mz.y ? mz.y : 0.f) : mz.y * by;
      y += v * by;
    }
  }
  sums[threadIdx.x] = y;
  zs[threadIdx.x] = Z;
  __syncthreads();
  if (mine != 0) return;
  for (int i = 1; i < groups; ++i) {
    y += sums[i * lanes + threadIdx.x];
    Z += zs[i * lanes + threadIdx.x];
  }
  const int row_in = col.row0 + r;
  const int64_t to_row = (int64_t)(col.token0 + row_in / G) * a.Hq + head * G + row_in % G;
  const float inv = Z == 0.f ? 0.f : 1.f / Z;
  if (at == 0 && a.lse) a.lse[to_row] = Z == 0.f ? MINUS_INF : (__builtin_amdgcn_logf(Z) + top * a.scale2) * 0.69314718055994530942f;
  if constexpr (std::is_same<Q, float>::value) {
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + to_row * c.d + at) = y * inv;
  } else {
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + to_row * c.d + at) = u32x2{pack2(y[0] * inv, y[1] * inv), pack2(y[2] * inv, y[3] * inv)};
  }
}

// ---- the host's part -------------------------------------------------------------------------

constexpr int64_t MOST_PARTS = 4096;      // of a call, beside one of every column

int tiles_of_rows(int dtype, int d, int n, int64_t n_tokens, int G) {
  const int64_t rows = (n_tokens + n - 1) / n * G;                   // of a request, on average
  const int most = dtype == LAQ_F32 || d > 128 ? 2 : 4;
  return rows <= 16 ? 1 : rows <= 32 || most == 2 ? 2 : 4;
}

AttPlan plan_of(const PagedView& c, int Hq, int dtype, int n, int64_t n_tokens, bool has_start, int max_rows, bool may_cut) {
  const int G = Hq / c.Hkv;
  AttPlan p;
  p.tile = 16 * tiles_of_rows(dtype, c.d, n, n_tokens, G);
  const int64_t slots = has_start ? n_tokens * G / p.tile + n : (int64_t)n * ((G + p.tile - 1) / p.tile);
  p.slots = (int32_t)(slots < 0x7fffffff ? slots : 0x7fffffff);
  p.parts = 1;
  p.part_rows = 0x7fffffff;
  if (!may_cut) return p;
  const int64_t columns = slots * c.Hkv;
  // as many parts as keep the device busy and a workspace small, none shorter than two turns of a workgroup
  int64_t rows = ((int64_t)max_rows * columns / MOST_PARTS + 127) / 128 * 128;
  if (rows < 256) rows = 256;
  if (max_rows > rows) {
    p.part_rows = (int32_t)rows;
    p.parts = (int32_t)((max_rows + rows - 1) / rows);
  }
  return p;
}

struct Bytes { size_t mz, sums; };
Bytes bytes_of(const PagedView& c, const AttPlan& p) {
  if (p.parts == 1) return Bytes{0, 0};
  const size_t rows = (size_t)p.slots * c.Hkv * p.parts * p.tile;
  return Bytes{(rows * sizeof(float2) + 255) / 256 * 256, rows * c.d * sizeof(float)};
}

template <typename Q, typename E, int D>
hipError_t start_attention(const PagedView& c, const PagedAttention& a, const AttPlan& p, const Partials& part, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)p.slots * c.Hkv * p.parts));
  switch (p.tile) {
    case 16: hipLaunchKernelGGL((paged_attention_kernel<Q, E, D, 1>), grid, dim3(ATT_THREADS), 0, st, c, a, p, part); break;
    case 32: hipLaunchKernelGGL((paged_attention_kernel<Q, E, D, 2>), grid, dim3(ATT_THREADS), 0, st, c, a, p, part); break;
    default:
      if constexpr (!std::is_same<Q, float>::value && D <= 128)
        hipLaunchKernelGGL((paged_attention_kernel<Q, E, D, 4>), grid, dim3(ATT_THREADS), 0, st, c, a, p, part);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts == 1) return e;
  hipLaunchKernelGGL((paged_join_kernel<Q>), dim3((unsigned)((int64_t)p.slots * c.Hkv * p.tile)), dim3(JOIN_THREADS), 0, st, c, a, p, part);
  return hipGetLastError();
}

template <typename Q, typename E>
hipError_t by_size(const PagedView& c, const PagedAttention& a, const AttPlan& p, const Partials& part, hipStream_t st) {
  if (c.d <= 64) return start_attention<Q, E, 64>(c, a, p, part, st);
  if (c.d <= 128) return start_attention<Q, E, 128>(c, a, p, part, st);
  return start_attention<Q, E, 256>(c, a, p, part, st);
}

}  // namespace

size_t paged_attention_bytes(const PagedView& c, int Hq, int dtype, int n, int64_t n_tokens, int max_rows) {
  const AttPlan with = plan_of(c, Hq, dtype, n, n_tokens, true, max_rows, true), without = plan_of(c, Hq, dtype, n, n_tokens, false, max_rows, true);
  const Bytes x = bytes_of(c, with), y = bytes_of(c, without);
  return x.mz + x.sums > y.mz + y.sums ? x.mz + x.sums : y.mz + y.sums;
}

bool paged_attention_fits(const PagedView& c, int dtype, const PagedAttention& a, bool cut) {
  const AttPlan p = plan_of(c, a.Hq, dtype, a.n, a.n_tokens, a.start != nullptr, a.max_rows, cut);
  const int64_t columns = (int64_t)p.slots * c.Hkv;
  return columns * p.parts < (1 << 24) && (p.parts == 1 || columns * p.tile < (1 << 24));
}

hipError_t launch_paged_attention(const PagedView& c, int dtype, const PagedAttention& a, void* ws, hipStream_t st) {
  const AttPlan p = plan_of(c, a.Hq, dtype, a.n, a.n_tokens, a.start != nullptr, a.max_rows, ws != nullptr);
  const Bytes b = bytes_of(c, p);
  const Partials part{static_cast<float2*>(ws), reinterpret_cast<float*>(static_cast<char*>(ws) + b.mz)};
  if (dtype == LAQ_BF16)
    return c.type == LAQ_BF16 ? by_size<uint16_t, uint16_t>(c, a, p, part, st) : by_size<uint16_t, E4m3>(c, a, p, part, st);
  switch (c.type) {
    case LAQ_F32: return by_size<float, float>(c, a, p, part, st);
    case LAQ_BF16: return by_size<float, uint16_t>(c, a, p, part, st);
    default: return by_size<float, E4m3>(c, a, p, part, st);
  }
}

}  // namespace laq
