// Attention over the paged 4-bit cache (include/laq_fp4.h: laq_fp4_attention).
//
// A column is a KV head of a request and a tile of its score rows (row r = query head r % G of the group of the request's token r / G).  A
// workgroup has a range of a column's keys, in turns of 64 * KT: its four waves take 16 * KT keys of a turn each, every wave for all rows of the
// tile, with its own reference m, sum z and sums O (one pass, exponentials of s - m; m moves only when a score is more than 8 above it, so that
// the usual step has no maximum over lanes); they are folded at the end through LDS, the ranges of a column by the workgroup that finds all of
// them finished, in a fixed order.
//
// How the ranges lie: long calls of several requests with a token each are shared out evenly, all turns of all columns (fp4_attention_shares),
// since the lengths, which the host does not know, are as unequal as requests are.  Other calls: equal parts of the longest request that the
// host expects, where there would be too few workgroups otherwise (fp4_attention_parts).
//
// Bound: single tokens, the cache's bytes (68 a row of d = 128, K and V each): 96 x 8 heads x 6144 rows 6.3 TB/s, 128 x 8 heads x 2048 to 8192
// rows 5.7 TB/s; the vector units are busy a third of the time.  Chunks of a prompt, the vector units beside the matrix cores (exponentials,
// conversions, packing): 4 x 512 tokens x 32 heads over 2100 to 8704 rows 212 us, 880 TFLOP/s, vector units busy 50 % of the time, matrix cores 34 %.
//
// Products are 16 x 16 x 32 bf16 with the keys as the first operand's rows, so that a lane has four keys of one score row (column n = lane % 16)
// and all that belongs to a row lies in lanes n, n + 16, n + 32, n + 48:
//   S^T = K Q^T   codes go from memory to the operand's registers, converted eight numbers in four instructions with the scale applied: exact, no LDS.
//                 A lane reads one contiguous piece of a key row (the sum over channels may take them in any order, Q the same)
//   O^T = V^T P^T P^T is where S^T left it: the lane's four keys of two tiles are eight of the 32 summed over.  V^T needs eight keys of one channel in a
//                 lane: rows are converted like K's, written to LDS and read back transposed (the LDS's own transposing read)
//
// fp32: q as the sum of three bf16 (their rows brought to about 2^-20 by a power of two), weights too; K and V are exact in bf16.
//
// A V that stands for NaN must not reach rows that do not see it (0 * NaN): only in steps whose keys not every row sees, where such
// a block is, V has 0 there and a second product of ones tells which sums it belongs to.
#include <atomic>
#include <chrono>
#include <type_traits>

#include "laq_fp4_codes.h"
#include "laq_products.h"

namespace laq {

namespace {

constexpr int ATT_THREADS = 256, ATT_WAVES = 4;
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2)); }

// How the launch is cut, from what the host knows.
struct AttPlan {
  int32_t parts, part_rows;              // several tokens: a column in parts of part_rows, `parts` at most (the last one takes what is left)
  int32_t tiles_per;                     // a token each: tiles of a request
  int32_t ws_rows;                       // rows of a tile that can be there
  int32_t adv_blocks, adv_tiles;         // what a turn moves a position (block, key tile in it) by
};

template <int FROM, int TO, typename F>
__device__ __forceinline__ void for_groups(F&& f) {
  if constexpr (FROM < TO) {
    f(std::integral_constant<int, FROM>{});
    for_groups<FROM + 1, TO>(f);
  }
}

// A lane of quarter h has the numbers 8 D32 h .. of a row, in D32 groups of eight: one piece of memory.
template <int D32> __device__ __forceinline__ int channel_of(int t, int h) { return 8 * (h * D32 + t); }

// A lane's codes and scales of a key row.  Group t lies in scale block (h D32 + t) / 4; a quarter touches NS of these, and reads NS from first_scale() on.
template <int D32>
struct KeyPiece {
  static constexpr int NS = D32 == 7 ? 3 : D32 == 3 || D32 >= 5 ? 2 : 1;
  uint32_t c[D32];
  uint32_t s[NS];
  static constexpr __host__ __device__ int first_scale(int h) { return h * D32 / 4 < D32 - NS ? h * D32 / 4 : D32 - NS; }
  static constexpr __host__ __device__ int scale_of(int t, int h) { return (h * D32 + t) / 4 - first_scale(h); }
  // the quarters, a bit each, whose group t has the lane's scale i or a later one: none or all where head sizes fit the pieces
  static constexpr __host__ __device__ int quarters(int t, int i) {
    int q = 0;
    for (int h = 0; h < 4; ++h) q |= scale_of(t, h) >= i ? 1 << h : 0;
    return q;
  }
  // (all are read before one is chosen: a choice between places in memory keeps them there; d = 224, 64 requests of 8192 to 1000 rows 235 : 124 us)
  template <int T>
  __device__ __forceinline__ uint32_t scale(int h) const {
    const uint32_t s1 = s[NS > 1 ? 1 : 0], s2 = s[NS > 2 ? 2 : 0];
    uint32_t x = s[0];
    if constexpr (NS > 1) {
      constexpr int Q = quarters(T, 1);
      x = Q == 15 ? s1 : Q == 0 ? x : Q >> h & 1 ? s1 : x;
    }
    if constexpr (NS > 2) {
      constexpr int Q = quarters(T, 2);
      x = Q == 15 ? s2 : Q == 0 ? x : Q >> h & 1 ? s2 : x;
    }
    return x;
  }
  // codes, scales: of the tile's first row (uniform); the offsets: of this lane's.  ONCE: rows that one workgroup reads, past the caches
  // (96 requests x 6144 rows x 8 heads, 641 MB: 112 us, 126 without; with 32 tiles of a request that read the same rows 288 against 267)
  template <bool ONCE, int N>
  static __device__ __forceinline__ void words(const uint8_t* p, uint32_t* to) {
    typedef uint32_t vec __attribute__((ext_vector_type(N == 1 ? 2 : N), aligned(4)));
    if constexpr (N == 1) {
      to[0] = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p)) : *reinterpret_cast<const uint32_t*>(p);
    } else {
      vec w;
      if constexpr (ONCE) w = __builtin_nontemporal_load(reinterpret_cast<const vec*>(p));
      else w = *reinterpret_cast<const vec*>(p);
#pragma unroll
      for (int i = 0; i < N; ++i) to[i] = w[i];
    }
  }
  template <bool ONCE>
  __device__ __forceinline__ void read(const uint8_t* codes, const uint8_t* scales, uint32_t code_at, uint32_t scale_at) {
    words<ONCE, (D32 < 4 ? D32 : 4)>(codes + code_at, c);
    if constexpr (D32 > 4) words<ONCE, D32 - 4>(codes + code_at + 16, c + 4);
#pragma unroll
    for (int i = 0; i < NS; ++i) s[i] = scales[scale_at + i];
  }
  template <int T>
  __device__ __forceinline__ u32x4 group(int h) const { return __builtin_bit_cast(u32x4, fp4_to_bf16(c[T], fp4_scale_value(scale<T>(h)))); }
  // which groups stand for NaN; those are 0 then
  __device__ __forceinline__ uint32_t take_nan(int h) {
    uint32_t found = 0;
    for_groups<0, D32>([&](auto t) {
      if (scale<t()>(h) == 255u) {
        found |= 1u << t();
        c[t()] = 0;
      }
    });
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (s[i] == 255u) s[i] = 127;
    return found;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < D32; ++t) c[t] = 0;
#pragma unroll
    for (int i = 0; i < NS; ++i) s[i] = 127;
  }
};

// A tile's request and rows.
struct AttTile {
  int inst, token0, T;                   // request, its first token, its tokens
  int first_row, n_rows;                 // score rows of this tile among the request's T * G
  int held;                              // rows of the cache
  int seen_min, seen_max;                // rows that the first and the last score row see
};
// The rows that score row r of the request sees.
__device__ __forceinline__ int rows_seen(const AttTile& t, int r, int G) { return min(max(t.held - t.T + r / G + 1, 0), t.held); }

__device__ __forceinline__ int rows_held(const Fp4View& c, const Fp4Attention& a, int rows) {
  return (int)min((long long)max(rows, 0), (long long)a.blocks_per_inst * c.block_rows);
}

// Tile `tile` of the batch.
template <int TR>
__device__ __forceinline__ bool find_tile(const Fp4View& c, const Fp4Attention& a, const AttPlan& p, int tile, int G, AttTile* out) {
  int tin;
  if (!a.start) {
    out->inst = out->token0 = tile / p.tiles_per;
    out->T = 1;
    tin = tile - out->inst * p.tiles_per;
  } else {
    // request i has the tiles from start[i] * G / TR + i on: never fewer than it needs
    const auto start = [&](int i) { return min(max(a.start[i], 0), (int)a.n_tokens); };
    int lo = 0, hi = a.n;
    // 64 requests at a time: a trip to memory instead of six
    while (hi - lo > 1) {
      const int step = (hi - lo + 63) / 64, i = lo + (int)(threadIdx.x & 63) * step;
      const bool before = i < hi && (int)((uint32_t)(start(i) * G) / TR) + i <= tile;
      const unsigned long long found = __ballot(before) | 1;
      lo += (63 - __builtin_clzll(found)) * step;
      hi = min(lo + step, hi);
    }
    out->inst = lo;
    out->token0 = start(lo);
    out->T = max(start(lo + 1) - out->token0, 0);
    tin = tile - ((int)((uint32_t)(out->token0 * G) / TR) + lo);
    if (tin < 0) return false;           // (a `start` that does not begin with 0)
  }
  out->first_row = tin * TR;
  out->n_rows = min(out->T * G - out->first_row, TR);
  if (out->n_rows <= 0) return false;
  out->held = rows_held(c, a, a.rows[out->inst]);
  out->seen_min = rows_seen(*out, out->first_row, G);
  out->seen_max = rows_seen(*out, out->first_row + out->n_rows - 1, G);
  return true;
}

// Eight numbers of a query row as the operand's parts.
template <typename T> constexpr int PARTS_OF = is_f32(T()) ? 3 : 1;

template <typename T, int D32, int RT>
__device__ __forceinline__ void read_queries(const Fp4Attention& a, const AttTile& tl, int kv, int G, int lane, u32x4 (&q)[RT][D32][PARTS_OF<T>],
                                             float (&factor)[is_f32(T()) ? RT : 1]) {
  const int n = lane & 15, h = lane >> 4;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = rt * 16 + n, row = tl.first_row + r;
    const bool there = r < tl.n_rows;
    const int t = row / G, g = row - t * G;
    const T* src = static_cast<const T*>(a.q) + (int64_t)(tl.token0 + (there ? t : 0)) * a.stride_token + (int64_t)(kv * G + (there ? g : 0)) * a.stride_head;
    if constexpr (is_f32(T())) {
      u32x4 x[D32][2];
      uint32_t most = 0;
#pragma unroll
      for (int g8 = 0; g8 < D32; ++g8)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          x[g8][j] = u32x4{0, 0, 0, 0};
          if (there) x[g8][j] = *reinterpret_cast<const u32x4*>(src + channel_of<D32>(g8, h) + 4 * j);
#pragma unroll
          for (int i = 0; i < 4; ++i) most = max(most, x[g8][j][i] & 0x7fffffffu);
        }
      most = max(most, (uint32_t)__shfl_xor((int)most, 16));
      most = max(most, (uint32_t)__shfl_xor((int)most, 32));
      // the largest of the row to 2^-20 .. 2^-19 (from 2^40 on: times 2^-60, so that the factor stays a number): no part is too small for bf16, no sum of
      // products overflows before the logit does
      const int e = (int)(most >> 23), shift = most >= 0x7f800000u || most == 0 ? 0 : max(107 - e, -60);
      factor[rt] = fmaxf(ldexpf(a.scale2, -shift), 0x1p-126f);           // (not 0, as below)
#pragma unroll
      for (int g8 = 0; g8 < D32; ++g8) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[g8][j][i] = __float_as_uint(ldexpf(__uint_as_float(x[g8][j][i]), shift));
        const Split s = split8(x[g8][0], x[g8][1]);
#pragma unroll
        for (int pl = 0; pl < 3; ++pl) q[rt][g8][pl] = s.p[pl];
      }
    } else {
#pragma unroll
      for (int g8 = 0; g8 < D32; ++g8) {
        q[rt][g8][0] = u32x4{0, 0, 0, 0};
        if (there) q[rt][g8][0] = *reinterpret_cast<const u32x4*>(src + channel_of<D32>(g8, h));
      }
    }
  }
}

// The sum of eight weights' parts: four of one key tile, four of the next.  bf16: one part, rounded as the operand has it.  A result is then 0.0023 of its size
// from 64 bits, 0.0017 of which its own rounding makes; a second part would double the products with V for the rest.
template <typename T>
__device__ __forceinline__ void split_weights(const f32x4& a, const f32x4& b, u32x4 (&p)[PARTS_OF<T>]) {
  if constexpr (is_f32(T())) {
    const Split s = split8(__builtin_bit_cast(u32x4, a), __builtin_bit_cast(u32x4, b));
#pragma unroll
    for (int i = 0; i < 3; ++i) p[i] = s.p[i];
  } else {
    p[0] = u32x4{pack2(a[0], a[1]), pack2(a[2], a[3]), pack2(b[0], b[1]), pack2(b[2], b[3])};
  }
}

template <typename T> __device__ __forceinline__ void put8(T* p, const float (&x)[8]) {
  if constexpr (is_f32(T())) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
  }
}

// The ranges of cut columns: a slot of the workspace has sums[slot][ws_rows][d], and per row two words marks[slot][ws_rows][2]: the
// launch's nonce with the reference, and with the sum of weights.
struct AttParts {
  unsigned long long* marks;
  float* sums;
  uint32_t nonce;                        // a number that no other recent launch of the process has
};
// Range s of `count` of a column: slots first, then second, second + step, ...
struct AttColumn {
  int s, count;
  size_t first, second;
  int step;
  __device__ __forceinline__ size_t slot(int i) const { return i == 0 ? first : second + (size_t)(i - 1) * step; }
};
// Written through to the device's memory, and read from there.
__device__ __forceinline__ void store_pair(void* p, uint32_t a, uint32_t b) {
  __hip_atomic_store(static_cast<unsigned long long*>(p), (unsigned long long)b << 32 | a, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint2 load_pair(const void* p) {
  const unsigned long long v = __hip_atomic_load(static_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_uint2((uint32_t)v, (uint32_t)(v >> 32));
}
__device__ __forceinline__ void stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

constexpr float LN2 = 0.69314718055994530942f;
// Where score row `row` of the tile goes: its number among the rows of out and lse.
__device__ __forceinline__ size_t out_row(const Fp4Attention& a, const AttTile& tl, int kv, int G, int row) {
  const int global = tl.first_row + row, token = global / G;
  return (size_t)(tl.token0 + token) * a.Hq + kv * G + (global - token * G);
}

// Folds the ranges of a column, in their order, if all of them are finished (decode attention's way, laq_decode.hip): every range sets its marks
// after its sums have been written and then looks at the marks of all.  Whoever finds all of them set clears them, so that a captured
// launch, whose nonce is the same every time, never finds its own old ones; whatever else lies in the workspace is an unfinished range.
// `sm`: room for FOLD marks.  Several workgroups may find all of them set.  Where the marks fit, each has its copy from before anybody clears, and all write
// the same values.  Where they do not, the fold reads them again, and one alone folds: the one that takes the column's first mark away.
template <typename T, int FOLD>
__device__ void fold_ranges(const Fp4View& c, const Fp4Attention& a, const AttPlan& p, const AttTile& tl, const AttParts& pa, const AttColumn& col, int kv,
                            int G, float2* sm) {
  const int tid = threadIdx.x, R = tl.n_rows;
  bool all = true;
  for (int i = tid; i < col.count * R; i += ATT_THREADS) {
    const unsigned long long* mark = pa.marks + (col.slot(i / R) * p.ws_rows + i % R) * 2;
    const uint2 m = load_pair(mark), z = load_pair(mark + 1);
    all = all && m.x == pa.nonce && z.x == pa.nonce;
    if (i < FOLD) sm[i] = float2{__uint_as_float(m.y), __uint_as_float(z.y)};
  }
  if (!__syncthreads_and(all)) return;
  const int pairs = c.d / 2, at_once = FOLD / R;           // ranges whose marks fit
  const bool again = col.count > at_once;
  uint32_t taken_ref = 0;                                  // thread 0: what the mark that it took away held
  if (again) {
    bool taken = false;
    if (tid == 0) {
      const unsigned long long was = __hip_atomic_exchange(pa.marks + col.slot(0) * p.ws_rows * 2, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      taken = (uint32_t)was == pa.nonce;
      taken_ref = (uint32_t)(was >> 32);
    }
    if (!__syncthreads_or(taken)) return;
  }
  // EU pairs of channels of a thread at a time, so that enough loads are under way: 16
  auto fold = [&](auto EUC) {
    constexpr int EU = decltype(EUC)::value;
    for (int e0 = tid; e0 < (R * pairs + ATT_THREADS - 1) / ATT_THREADS * ATT_THREADS; e0 += ATT_THREADS * EU) {
      int row[EU], ch[EU];
      float M[EU], Z[EU], x[EU], y[EU];
#pragma unroll
      for (int u = 0; u < EU; ++u) {
        const int e = min(e0 + u * ATT_THREADS, R * pairs - 1);
        row[u] = e / pairs;
        ch[u] = (e - row[u] * pairs) * 2;
        M[u] = -INFINITY;
        Z[u] = x[u] = y[u] = 0.f;
      }
      for (int s0 = 0; s0 < col.count; s0 += at_once) {
        const int n = min(at_once, col.count - s0);
        if (again) {
          __syncthreads();
          for (int i = tid; i < n * R; i += ATT_THREADS) {
            const unsigned long long* mark = pa.marks + (col.slot(s0 + i / R) * p.ws_rows + i % R) * 2;
            sm[i] = float2{__uint_as_float(s0 + i == 0 ? taken_ref : load_pair(mark).y), __uint_as_float(load_pair(mark + 1).y)};
          }
          __syncthreads();
        }
        float ref[EU];
#pragma unroll
        for (int u = 0; u < EU; ++u) {
          float top = M[u];
          for (int s = 0; s < n; ++s) top = fmaxf(top, sm[s * R + row[u]].x);
          ref[u] = top == -INFINITY ? 0.f : top;
          const float w = M[u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M[u] - ref[u]);
          M[u] = top;
          Z[u] *= w;
          x[u] *= w;
          y[u] *= w;
        }
#pragma unroll(16 / EU)
        for (int s = 0; s < n; ++s) {
          const float* from = pa.sums + col.slot(s0 + s) * p.ws_rows * c.d;
#pragma unroll
          for (int u = 0; u < EU; ++u) {
            const float2 mz = sm[s * R + row[u]];
            const uint2 o = load_pair(from + row[u] * c.d + ch[u]);
            const float w = __builtin_amdgcn_exp2f(mz.x - ref[u]);
            Z[u] = fmaf(mz.y, w, Z[u]);
            x[u] = fmaf(__uint_as_float(o.x), w, x[u]);
            y[u] = fmaf(__uint_as_float(o.y), w, y[u]);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < EU; ++u) {
        if (e0 + u * ATT_THREADS >= R * pairs) break;
        const float part_of = Z[u] == 0.f ? 0.f : 1.f / Z[u], vx = x[u] * part_of, vy = y[u] * part_of;
        const size_t to = out_row(a, tl, kv, G, row[u]);
        if constexpr (is_f32(T())) *reinterpret_cast<float2*>(static_cast<T*>(a.out) + to * c.d + ch[u]) = float2{vx, vy};
        else *reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + to * c.d + ch[u]) = pack2(vx, vy);
        if (a.lse && ch[u] == 0) a.lse[to] = Z[u] == 0.f ? -INFINITY : (M[u] + __builtin_amdgcn_logf(Z[u])) * LN2;
      }
    }
  };
  if (R * pairs <= ATT_THREADS) fold(std::integral_constant<int, 1>{});
  else fold(std::integral_constant<int, 4>{});
  if (again) __syncthreads();                              // (this workgroup, the only one to fold, reads the marks until here)
  for (int i = tid; i < col.count * R; i += ATT_THREADS) {
    unsigned long long* mark = pa.marks + (col.slot(i / R) * p.ws_rows + i % R) * 2;
    store_pair(mark, 0, 0);
    store_pair(mark + 1, 0, 0);
  }
}

// A call's arguments.  Kernels read them where they are needed, from the launch's own argument memory through the scalar cache: kept in registers from their first
// use to their last, they and what a step computes are more than the 102 scalar registers hold, and a step then fetches spilled ones back one instruction each.
struct AttCall {
  Fp4View c;
  Fp4Attention a;
  AttPlan p;
  AttParts pa;
};
typedef __attribute__((address_space(4))) const AttCall* AttCallPtr;
__device__ __forceinline__ AttCallPtr att_call() { return (AttCallPtr)__builtin_amdgcn_kernarg_segment_ptr(); }
// The same, to be read anew.
__device__ __forceinline__ const AttCall& anew(AttCallPtr call) {
  asm volatile("" : "+s"(call));
  return *(const AttCall*)call;
}

template <int D32, int RT>
struct AttLds {
  static constexpr int CG = D32 < 4 ? D32 : 4, CHUNKS = (D32 + 3) / 4;        // groups of a chunk of V's channels (32 columns each), chunks
  static constexpr int STRIDE = CG * 64 + 32;                                  // bytes of a key's row of a chunk
  static constexpr int OSTRIDE = CG * 32 + 4;                                  // floats of a row's sums
  static constexpr int V_BYTES = 32 * STRIDE, O_BYTES = 16 * OSTRIDE * 4;
  static constexpr int WAVE_BYTES = V_BYTES > O_BYTES ? V_BYTES : O_BYTES;
  __align__(16) unsigned char wave[ATT_WAVES][WAVE_BYTES];
  float m[ATT_WAVES][16 * RT], z[ATT_WAVES][16 * RT];
};

// The key tiles first .. end - 1 of a column.  EARLY_V: the next step's rows of V are asked for as soon as this step's are in LDS, not after their
// products: 256 requests x 1024 rows 54.5 : 53.5 us, 64 of 2048 to 100 24.2 : 22.8; but where all places are taken for long 102 : 108 (96 x 6144),
// unless registers leave few places: 64 of 8192 to 1000, d = 160 105 : 98, fp32 and 32 of d = 256 121 : 112, bf16 of d = 192 to 256 the same.
template <typename T, int D32, int RT, int KT, bool ONCE, bool EARLY_V>
__device__ __forceinline__ void attend(AttCallPtr call, const AttTile& tl, int kv, int G, int first, int end, const AttColumn& col, AttLds<D32, RT>& sh) {
  const AttCall& k = anew(call);
  const Fp4View& c = k.c;
  const Fp4Attention& a = k.a;
  const AttPlan& p = k.p;
  using Lds = AttLds<D32, RT>;
  constexpr int NP = PARTS_OF<T>, CG = Lds::CG, CHUNKS = Lds::CHUNKS, STRIDE = Lds::STRIDE, OSTRIDE = Lds::OSTRIDE;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, h = lane >> 4;
  u32x4 q[RT][D32][NP];
  // the factor of the products: of all rows, but where rows are brought to a magnitude (fp32)
  float row_factor[is_f32(T()) ? RT : 1];
  read_queries<T, D32, RT>(a, tl, kv, G, lane, q, row_factor);
  const float factor_of_all = fmaxf(a.scale2, 0x1p-126f);        // (not 0: a masked product is -infinity)
  auto factor = [&](int rt) {
    if constexpr (is_f32(T())) return row_factor[rt];
    else return factor_of_all;
  };

  // rows of the cache that row n of tile rt sees (few steps ask)
  auto row_sees = [&](int rt) { return rows_seen(tl, tl.first_row + min(rt * 16 + n, tl.n_rows - 1), G); };

  // this wave's position: key tile `at`, in block `block` of the request its tile `in_block`
  const int per_block = c.block_rows / 16;
  int at = first + wave * KT, block = at / per_block, in_block = at - block * per_block;
  typedef __attribute__((address_space(4))) const int32_t* ConstTable;
  const ConstTable table = (ConstTable)(unsigned long long)(a.table + (size_t)tl.inst * a.blocks_per_inst);
  const uint8_t *kc = c.k.codes + kv * c.head, *ks = c.k.scales + kv * c.scale_head, *vc = c.v.codes + kv * c.head, *vs = c.v.scales + kv * c.scale_head;
  const uint32_t code_at = n * (uint32_t)c.row + h * 4 * D32, scale_at = n * (uint32_t)c.scale_row + KeyPiece<D32>::first_scale(h);

  KeyPiece<D32> kp[KT], vp[KT];
  int64_t code_base[KT], scale_base[KT];
  uint32_t there = 0, there_v = 0;       // a bit for each tile of the step whose rows are there
  // Block numbers are asked for a step ahead, so that their way does not lie in front of the codes'.  (Addresses of products of 32 bits: what is scalar in a step
  // takes a third of its instructions.)
  int number[KT];
  const int last_block = max(tl.held - 1, 0) / c.block_rows;
  const bool straddles = per_block % KT != 0;              // a step's tiles may lie in several blocks
  const uint32_t tile_codes = (uint32_t)c.row * 16, tile_scales = (uint32_t)c.scale_row * 16;
  auto ask = [&](int b, int r) {
    number[0] = table[min(b, last_block)];
    if (straddles) {
#pragma unroll
      for (int i = 1; i < KT; ++i) {
        if (++r == per_block) {
          r = 0;
          ++b;
        }
        number[i] = table[min(b, last_block)];
      }
    }
  };
  auto locate = [&] {                    // the tiles of the step at `at`, whose block numbers have been asked for
    // (tiles beyond the end are those of the last block: read, and not there)
    auto place = [&](int i, int r) {
      const bool good = (uint32_t)number[i] < (uint32_t)c.n_blocks;
      const uint32_t num = good ? number[i] : 0;
      code_base[i] = (uint64_t)num * (uint32_t)c.block + (uint64_t)(uint32_t)r * tile_codes;
      scale_base[i] = (uint64_t)num * (uint32_t)c.scale_block + (uint64_t)(uint32_t)r * tile_scales;
      return good;
    };
    const int left = min(end - at, KT);  // tiles
    const bool good = place(0, in_block);
    if (straddles) {
      there = good;
      int r = in_block;
#pragma unroll
      for (int i = 1; i < KT; ++i) {
        if (++r == per_block) r = 0;
        there |= (uint32_t)place(i, r) << i;
      }
      there &= (1u << left) - 1;
    } else {
#pragma unroll
      for (int i = 1; i < KT; ++i) {
        code_base[i] = code_base[i - 1] + tile_codes;      // (one at a time: three tiles' distance is more than 32 bits hold)
        scale_base[i] = scale_base[i - 1] + tile_scales;
      }
      there = good ? (1u << left) - 1 : 0u;
    }
  };
  auto advance = [&] {
    at += ATT_WAVES * KT;
    block += p.adv_blocks;
    in_block += p.adv_tiles;
    if (in_block >= per_block) {
      in_block -= per_block;
      ++block;
    }
  };
  auto ask_next = [&] {                  // for the step after that at `at`
    int b = block + p.adv_blocks, r = in_block + p.adv_tiles;
    if (r >= per_block) {
      r -= per_block;
      ++b;
    }
    ask(b, r);
  };

  // of row n of each tile: the exponents' reference, the product from which on it is moved (LEEWAY beyond it: weights of up to 2^8 cost
  // nothing, and most steps then neither look for their rows' maxima across lanes nor touch the sums), this lane's share of the sum
  constexpr float LEEWAY = 8.f;
  float off[RT], limit[RT], z[RT];
  f32x4 acc[RT][CHUNKS * CG * 2];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    off[rt] = 0.f;
    limit[rt] = -INFINITY;
    z[rt] = 0.f;
#pragma unroll
    for (int i = 0; i < CHUNKS * CG * 2; ++i) acc[rt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  unsigned char* const my_lds = sh.wave[wave];
  // Rows of V are an odd number of 32 bytes apart, and rows 4 .. 7 of 8 have the halves of every 32 bytes changed: the reads (4 rows of 32 bytes by 16 lanes,
  // over 64 banks) and the writes (8 rows of 16 bytes at a time, over 32) then meet in no bank; without the change a write takes 16 cycles instead of 8.
  unsigned char* const v_write = my_lds + n * STRIDE + (h ^ (n >> 2 & 1)) * 16;
  const uint32_t v_read = (uint32_t)(4 * h + n / 4) * STRIDE + ((n & 3) * 8 ^ (h & 1) * 16);
  typedef __attribute__((address_space(3))) s16x4* LdsQuad;

  if (at < end) {
    ask(block, in_block);
    locate();
    ask_next();
    there_v = there;
#pragma unroll
    for (int i = 0; i < KT; ++i) kp[i].template read<ONCE>(kc + code_base[i], ks + scale_base[i], code_at, scale_at);
#pragma unroll
    for (int i = 0; i < KT; ++i) vp[i].template read<ONCE>(vc + code_base[i], vs + scale_base[i], code_at, scale_at);
  }
#pragma unroll 1
  while (at < end) {
    f32x4 s[RT][KT];
#pragma unroll
    for (int i = 0; i < KT; ++i) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      for_groups<0, D32>([&](auto t) {
        const u32x4 k8 = kp[i].template group<t()>(h);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int pl = 0; pl < NP; ++pl) s[rt][i] = mfma16(k8, q[rt][t()][NP - 1 - pl], s[rt][i]);
      });
    }
    const int key0 = at * 16;
    const bool masked = key0 > tl.seen_min - KT * 16 || there_v != (1u << KT) - 1;
    advance();
    if (at < end) {
      locate();
      ask_next();
#pragma unroll
      for (int i = 0; i < KT; ++i) kp[i].template read<ONCE>(kc + code_base[i], ks + scale_base[i], code_at, scale_at);
    }
    if (masked) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int seen = row_sees(rt);
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!(there_v >> i & 1) || key0 + i * 16 + 4 * h + r >= seen) s[rt][i][r] = -INFINITY;
      }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float top = s[rt][0][0];
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, s[rt][i][r]);
      if (__any(top > limit[rt])) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (top > limit[rt]) {
          const float moved = top * factor(rt), w = limit[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(off[rt] - moved);
          off[rt] = moved;
          limit[rt] = (moved + LEEWAY) / factor(rt);
          z[rt] *= w;
#pragma unroll
          for (int i = 0; i < CHUNKS * CG * 2; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[rt][i][r] *= w;
        }
      }
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[rt][i][r] = __builtin_amdgcn_exp2f(fmaf(s[rt][i][r], factor(rt), -off[rt]));
          z[rt] += s[rt][i][r];
        }
    }
    bool nan_rows = false;               // some V stands for NaN where not every row sees it
    uint32_t nan_at[KT];
    if (masked) {
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        if (!(there_v >> i & 1) || key0 + i * 16 + n >= tl.seen_max) vp[i].clear();
        nan_at[i] = vp[i].take_nan(h);
        nan_rows |= nan_at[i] != 0;
      }
      nan_rows = __any(nan_rows);
    }
#pragma unroll
    for (int j = 0; j < KT; j += 2) {
      u32x4 w[RT][NP];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) split_weights<T>(s[rt][j], s[rt][j + 1], w[rt]);
      // chunk ch of two tiles of V to LDS; with ONES, 1 where it stands for NaN and else 0
      auto stage = [&](auto ch, bool ones) {
        constexpr int first = ch() * CG, beyond = first + CG < D32 ? first + CG : D32;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          for_groups<first, beyond>([&](auto t) {
            const uint32_t one = ones && nan_at[j + i] >> t() & 1 ? 0x3f803f80u : 0u;
            *reinterpret_cast<u32x4*>(v_write + i * 16 * STRIDE + (t() - first) * 64) = ones ? u32x4{one, one, one, one} : vp[j + i].template group<t()>(h);
          });
      };
      auto column = [&](int ct) {        // 32 keys of 16 columns
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)(my_lds + v_read + ct * 32));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)(my_lds + v_read + 16 * STRIDE + ct * 32));
        const uint2 x = __builtin_bit_cast(uint2, lo), y = __builtin_bit_cast(uint2, hi);
        return u32x4{x.x, x.y, y.x, y.y};
      };
      for_groups<0, CHUNKS>([&](auto CH) {
        constexpr int ch = CH();
        // (LDS operations of a wave are done in their order: only the compiler has to keep it)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        stage(CH, false);
        if (EARLY_V && ch == CHUNKS - 1 && at < end) {
#pragma unroll
          for (int i = j; i < j + 2; ++i) vp[i].template read<ONCE>(vc + code_base[i], vs + scale_base[i], code_at, scale_at);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int ct = 0; ct < CG * 2; ++ct) {
          if (ch * CG + ct / 2 >= D32) break;
          const u32x4 v8 = column(ct);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int pl = 0; pl < NP; ++pl) acc[rt][ch * CG * 2 + ct] = mfma16(v8, w[rt][NP - 1 - pl], acc[rt][ch * CG * 2 + ct]);
        }
        if (__builtin_expect(nan_rows, 0)) {
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          stage(CH, true);
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            u32x4 sees;
            const int seen = row_sees(rt);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int tile_of = j + x / 2, key = key0 + tile_of * 16 + 4 * h + (x & 1) * 2;
              const bool in = there_v >> tile_of & 1;
              sees[x] = (in && key < seen ? 0x3f80u : 0u) | (in && key + 1 < seen ? 0x3f800000u : 0u);
            }
#pragma unroll
            for (int ct = 0; ct < CG * 2; ++ct) {
              if (ch * CG + ct / 2 >= D32) break;
              const f32x4 count = mfma16(column(ct), sees, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (count[r] > 0.f) acc[rt][ch * CG * 2 + ct][r] = NAN;
            }
          }
        }
      });
    }
    if (!EARLY_V && at < end) {
#pragma unroll
      for (int i = 0; i < KT; ++i) vp[i].template read<ONCE>(vc + code_base[i], vs + scale_base[i], code_at, scale_at);
    }
    there_v = there;
  }

  // fold the waves, 16 rows and a chunk of channels at a time
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    z[rt] += __shfl_xor(z[rt], 16);
    z[rt] += __shfl_xor(z[rt], 32);
    if (h == 0) {
      sh.m[wave][rt * 16 + n] = limit[rt] == -INFINITY ? -INFINITY : off[rt];
      sh.z[wave][rt * 16 + n] = z[rt];
    }
  }
  __syncthreads();
  const AttCall& e = anew(call);
  const bool whole = col.count == 1;
  const size_t slot = col.slot(col.s) * e.p.ws_rows;
  auto row_sum = [&](int r, float* top) {        // over the waves, of a row
    float M = sh.m[0][r];
#pragma unroll
    for (int w = 1; w < ATT_WAVES; ++w) M = fmaxf(M, sh.m[w][r]);
    const float ref = M == -INFINITY ? 0.f : M;
    float Z = 0.f;
#pragma unroll
    for (int w = 0; w < ATT_WAVES; ++w) Z = fmaf(sh.z[w][r], __builtin_amdgcn_exp2f(sh.m[w][r] - ref), Z);
    *top = M;
    return Z;
  };
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (rt * 16 >= tl.n_rows) break;
    float M = sh.m[0][rt * 16 + n];
#pragma unroll
    for (int w = 1; w < ATT_WAVES; ++w) M = fmaxf(M, sh.m[w][rt * 16 + n]);
    const float mine = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sh.m[wave][rt * 16 + n] - M);
#pragma unroll
    for (int ch = 0; ch < CHUNKS; ++ch) {
#pragma unroll
      for (int ct = 0; ct < CG * 2; ++ct)
        if (ch * CG + ct / 2 < D32) {
          f32x4 x = acc[rt][ch * CG * 2 + ct];
#pragma unroll
          for (int r = 0; r < 4; ++r) x[r] *= mine;
          *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(my_lds) + n * OSTRIDE + ct * 16 + 4 * h) = x;
        }
      __syncthreads();
      for (int x8 = threadIdx.x; x8 < 16 * CG * 4; x8 += ATT_THREADS) {       // eight columns of a row: group t, quarter hh
        const int r = x8 / (CG * 4), t = x8 % (CG * 4) / 4, hh = x8 & 3, row = rt * 16 + r;
        if (row < tl.n_rows && ch * CG + t < D32) {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
          for (int w = 0; w < ATT_WAVES; ++w)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] += reinterpret_cast<const float*>(sh.wave[w])[r * OSTRIDE + t * 32 + hh * 8 + i];
          const int channel = channel_of<D32>(ch * CG + t, hh);
          if (whole) {
            float top;
            const float Z = row_sum(row, &top), part_of = Z == 0.f ? 0.f : 1.f / Z;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] *= part_of;
            put8(static_cast<T*>(e.a.out) + out_row(e.a, tl, kv, G, row) * e.c.d + channel, x);
          } else {
#pragma unroll
            for (int i = 0; i < 8; i += 2) store_pair(e.pa.sums + (slot + row) * e.c.d + channel + i, __float_as_uint(x[i]), __float_as_uint(x[i + 1]));
          }
        }
      }
      __syncthreads();
    }
  }
  if (!whole) {
    stores_done();
    __syncthreads();
  }
  for (int row = threadIdx.x; row < tl.n_rows; row += ATT_THREADS) {
    float top;
    const float Z = row_sum(row, &top);
    if (!whole) {
      store_pair(e.pa.marks + (slot + row) * 2, e.pa.nonce, __float_as_uint(top));
      store_pair(e.pa.marks + (slot + row) * 2 + 1, e.pa.nonce, __float_as_uint(Z));
      stores_done();
    } else if (e.a.lse) {
      e.a.lse[out_row(e.a, tl, kv, G, row)] = Z == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(Z)) * LN2;
    }
  }
  if (whole) return;
  __syncthreads();
  fold_ranges<T, (int)sizeof sh.wave / 8>(e.c, e.a, e.p, tl, e.pa, col, kv, G, reinterpret_cast<float2*>(sh.wave[0]));
}

// Several tokens of a request, and calls that are not cut: a workgroup per part of a column.
template <typename T, int D32, int RT, int KT, bool ONCE>
__global__ __launch_bounds__(ATT_THREADS, (RT > 1 && D32 <= 5 ? 2 : 1)) void fp4_attention_parts(AttCall) {
  __shared__ AttLds<D32, RT> sh;
  const AttCallPtr call = att_call();
  const AttCall& k = anew(call);
  const Fp4View& c = k.c;
  const Fp4Attention& a = k.a;
  const AttPlan& p = k.p;
  const int G = a.Hq / c.Hkv, kv = blockIdx.x % c.Hkv, rest = blockIdx.x / c.Hkv, part = rest % p.parts, tile = rest / p.parts;
  AttTile tl;
  if (!find_tile<16 * RT>(c, a, p, tile, G, &tl)) return;
  // (lengths come up to 2^31 - 16, and a part of all of them is as long: their sum is none of an int)
  const int parts = min(p.parts, max((int)(((uint32_t)tl.seen_max + (uint32_t)p.part_rows - 1) / (uint32_t)p.part_rows), 1));
  if (part >= parts) return;
  const size_t slot = ((size_t)tile * c.Hkv + kv) * p.parts;
  attend<T, D32, RT, KT, ONCE, true>(call, tl, kv, G, part * p.part_rows / 16, part == parts - 1 ? (tl.seen_max + 15) / 16 : (part + 1) * p.part_rows / 16,
                               AttColumn{part, parts, slot, slot + 1, 1}, sh);
}

// One token each: the turns of all columns, request by request, are shared out evenly among the workgroups.  A share may end one column, have
// others whole and begin another, so a workgroup leaves at most two ranges for others to fold: slot 2w what it begins with, 2w + 1 what it ends with.
// A column counts COLUMN_TURNS more than it has, for what beginning and folding it takes.
// SHARES_PER_UNIT: workgroups that a compute unit holds, four waves to each, by the registers that a variant is given (bf16, d = 64: four
// spill, 64 requests of 8192 to 1000 rows 54 us, three 47).
constexpr int SHARE_MOST_REQUESTS = 1024;
constexpr int COLUMN_TURNS = 1;
template <typename T, int D32>
constexpr int SHARES_PER_UNIT = is_f32(T()) ? (D32 <= 2 ? 3 : D32 <= 6 ? 2 : 1) : D32 <= 5 ? 3 : 2;
template <typename T, int D32, int KT, bool ONCE>
__global__ __launch_bounds__(ATT_THREADS, (SHARES_PER_UNIT<T, D32>)) void fp4_attention_shares(AttCall) {
  constexpr int TURN = ATT_WAVES * KT * 16, PER = SHARE_MOST_REQUESTS / ATT_THREADS;
  __shared__ AttLds<D32, 1> sh;
  __shared__ int held[SHARE_MOST_REQUESTS];
  __shared__ int wave_turns[ATT_WAVES], begin_before, begin_inst;
  const AttCallPtr call = att_call();
  const AttCall& k = anew(call);
  const Fp4View& c = k.c;
  const Fp4Attention& a = k.a;
  const int tiles_per = k.p.tiles_per, G = a.Hq / c.Hkv, tid = threadIdx.x, lane = tid & 63, columns = c.Hkv * tiles_per;
  const auto turns_of = [](int rows) { return max(rows - 1, 0) / TURN + 1 + COLUMN_TURNS; };
  int mine = 0;                          // (the launch sees to it that the sum of all is one)
  const int per = (a.n + ATT_THREADS - 1) / ATT_THREADS;
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    const int i = tid * per + x;
    if (x < per && i < a.n) {
      held[i] = rows_held(c, a, a.rows[i]);
      mine += turns_of(held[i]) * columns;
    }
  }
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int y = __shfl_up(upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 63) wave_turns[tid >> 6] = upto;
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int w = 0; w < ATT_WAVES; ++w) {
    if (w < tid >> 6) upto += wave_turns[w];
    all += wave_turns[w];
  }
  // shares of q + 1 turns, `more` of them, and of q
  all = __builtin_amdgcn_readfirstlane(all);
  const int shares = min((int)gridDim.x, all), w = blockIdx.x, q = all / shares, more = all - q * shares;
  if (w >= shares) return;
  int at = w * q + min(w, more);
  const int stop = at + q + (w < more ? 1 : 0);
  const auto share_of = [&](int turn) {
    const int longer = more * (q + 1);
    return turn < longer ? turn / (q + 1) : more + (turn - longer) / q;
  };
  if (at >= upto - mine && at < upto) {
    int before = upto - mine, i = tid * per;
    while (at >= before + turns_of(held[i]) * columns) before += turns_of(held[i++]) * columns;
    begin_inst = i;
    begin_before = before;
  }
  __syncthreads();
  int inst = __builtin_amdgcn_readfirstlane(begin_inst), before = __builtin_amdgcn_readfirstlane(begin_before);
#pragma unroll 1
  while (at < stop) {
    const int rows = __builtin_amdgcn_readfirstlane(held[inst]), turns = turns_of(rows);
    const int column = __builtin_amdgcn_readfirstlane((at - before) / turns), t0 = at - before - column * turns;
    const int t1 = min(turns, t0 + stop - at), kv = __builtin_amdgcn_readfirstlane(column / tiles_per), tile = column - kv * tiles_per;
    AttTile tl;
    tl.inst = tl.token0 = inst;
    tl.T = 1;
    tl.first_row = tile * 16;
    tl.n_rows = min(G - tl.first_row, 16);
    tl.held = tl.seen_min = tl.seen_max = rows;
    if (t1 > COLUMN_TURNS) {
      const int begin = at - t0, s0 = __builtin_amdgcn_readfirstlane(share_of(begin + COLUMN_TURNS));
      const int s1 = __builtin_amdgcn_readfirstlane(share_of(begin + turns - 1));
      attend<T, D32, 1, KT, ONCE, (D32 > 4)>(call, tl, kv, G, max(t0 - COLUMN_TURNS, 0) * (TURN / 16), min((t1 - COLUMN_TURNS) * (TURN / 16), (rows + 15) / 16),
                                  AttColumn{w - s0, s1 - s0 + 1, (size_t)2 * s0 + 1, (size_t)2 * (s0 + 1), 2}, sh);
      __syncthreads();
    }
    at += t1 - t0;
    if (at - before >= turns * columns) {
      before += turns * columns;
      ++inst;
    }
  }
}

struct AttLaunch {
  AttPlan plan;
  int row_tiles, key_tiles;              // RT, KT
  bool shares, once;
  long long workgroups;
  size_t slots;                          // of the workspace
};

template <typename T>
int shares_per_unit(int d) {
  switch (d / 32) {
    case 1: return SHARES_PER_UNIT<T, 1>;
    case 2: return SHARES_PER_UNIT<T, 2>;
    case 3: return SHARES_PER_UNIT<T, 3>;
    case 4: return SHARES_PER_UNIT<T, 4>;
    case 5: return SHARES_PER_UNIT<T, 5>;
    case 6: return SHARES_PER_UNIT<T, 6>;
    case 7: return SHARES_PER_UNIT<T, 7>;
    default: return SHARES_PER_UNIT<T, 8>;
  }
}

AttLaunch plan_attention(const Fp4View& c, int Hq, int dtype, int n, int64_t n_tokens, int max_rows, bool one_each, bool cut) {
  const int G = Hq / c.Hkv;
  const long long rows_each = one_each ? G : (n_tokens * G + n - 1) / n;        // score rows of a request, on average
  AttLaunch l;
  // Tiles of 16 score rows of a workgroup.  More share what a step costs that does not depend on them (a third of its instructions with two, of
  // d = 128), but leave fewer workgroups: three from 192 rows on, with two of these a compute unit, where head sizes leave registers for it and
  // less would not let more workgroups in.  Two : three, us, 8 KV heads: 4 x 512 tokens x 4 heads over 8704 rows 243 : 211; 2 x 2048 over 8192
  // 576 : 498;  16 x 48 over 2048 43.4 : 33.9, x 100 69.3 : 63.5, x 24 27.3 : 34.6;  1 x 64 over 8192 33 : 44;  d = 64, 4 x 256 over 8192 117 : 136.
  const bool three = rows_each >= 192 && c.d > 64 && c.d <= 128 && n_tokens * G / 48 * c.Hkv >= 512;
  l.row_tiles = one_each || rows_each <= 16 || dtype == LAQ_F32 ? 1 : three ? 3 : 2;
  l.key_tiles = l.row_tiles == 1 && c.d <= 128 ? 4 : 2;
  l.once = rows_each <= 16;
  const int TR = 16 * l.row_tiles, turn = ATT_WAVES * l.key_tiles * 16;
  l.plan = AttPlan{1, 0x7fffff00, (G + TR - 1) / TR, one_each && G < TR ? G : TR, turn / c.block_rows, turn % c.block_rows / 16};
  // Columns (as many as are surely there) and the turns of the longest.  As many ranges of a column as make the sum of what they take (a turn 2 us
  // where few workgroups run) and what folding them takes (0.12 us each for sums of 512 numbers, more in proportion: one workgroup reads them all)
  // least, as long as that makes no more than two workgroups a compute unit: that many saturate the memory, and more of them only fold more.
  // (8 heads on one, 2 x 14 tokens over 21836 and 7278 rows, d = 256 93 : 57 us with the sums' size counted, d = 128 48 : 34.)
  // us, bf16, 8 heads of d = 128, with 1, 2, 4, 8, 16, 32, 64 ranges:
  //   1 x 4096 rows 37, 24, 17, 14, 12;  1 x 65536 503, 259, 136, 76, 43, 29, 28;  4 x 16384 133, 73, 42, 28, 23, 33, 42
  //   16 x 16384 140, 79, 53, 66, 67, 86, 121;  32 x 4096 41, 31, 40, 48, 59;  64 x 4096 53, 65, 67, 83, 109
  const long long tiles = one_each ? (long long)n * l.plan.tiles_per : n_tokens * G / TR + n;
  const long long columns = (one_each ? tiles : n_tokens * G / TR > n ? n_tokens * G / TR : n) * c.Hkv, turns = ((long long)max_rows + turn - 1) / turn;
  long long ranges = 1;
  const long long folded = l.plan.ws_rows * c.d > 512 ? l.plan.ws_rows * c.d : 512;
  while (ranges < turns && ranges * (ranges + 1) * folded < 16 * 512 * turns && (ranges + 1) * columns <= 512) ++ranges;
  // Long calls of one token each and several requests are shared out evenly.  us, shared out : the best equal parts, requests of that many rows, and of
  // an eighth of that to that many: 8 x 65536 106 : 97, 73 : 92 (of 8);  16 x 16384 59 : 53, 42 : 51;  32 x 16384 101 : 98, 67 : 89;
  // 64 x 4096 59 : 53, 41 : 46;  128 x 4096 109 : 101, 68 : 73;  shorter: 8 x 16384 38 : 34, 30 : 32;  8 x 4096 22 : 18, 20 : 16.
  // (A workgroup's scan of the lengths holds SHARE_MOST_REQUESTS of them; with more there are columns enough.)
  l.shares = cut && one_each && n > 1 && n <= SHARE_MOST_REQUESTS && turns >= 16 && columns * turns >= 8192;
  if (l.shares) {
    l.workgroups = 256 * (dtype == LAQ_BF16 ? shares_per_unit<uint16_t>(c.d) : shares_per_unit<float>(c.d));
    l.slots = 2 * l.workgroups;
    return l;
  }
  if (cut && ranges > 1) {
    const long long steps = (turns + ranges - 1) / ranges;
    l.plan.part_rows = (int)(steps * turn);
    l.plan.parts = (int)((turns + steps - 1) / steps);
  }
  l.workgroups = tiles * c.Hkv * l.plan.parts;
  l.slots = l.plan.parts > 1 ? l.workgroups : 0;
  return l;
}

template <typename T, int D32, int RT, int KT>
hipError_t launch_rt(const Fp4View& c, const Fp4Attention& a, const AttLaunch& l, const AttParts& pa, hipStream_t st) {
  const dim3 grid((unsigned)l.workgroups), threads(ATT_THREADS);
  const AttCall call{c, a, l.plan, pa};
  if constexpr (RT == 1) {
    if (l.shares) {
      if (l.once) hipLaunchKernelGGL((fp4_attention_shares<T, D32, KT, true>), grid, threads, 0, st, call);
      else hipLaunchKernelGGL((fp4_attention_shares<T, D32, KT, false>), grid, threads, 0, st, call);
      return hipGetLastError();
    }
    if (l.once) {
      hipLaunchKernelGGL((fp4_attention_parts<T, D32, RT, KT, true>), grid, threads, 0, st, call);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((fp4_attention_parts<T, D32, RT, KT, false>), grid, threads, 0, st, call);
  return hipGetLastError();
}

template <typename T, int D32>
hipError_t launch_d(const Fp4View& c, const Fp4Attention& a, const AttLaunch& l, const AttParts& pa, hipStream_t st) {
  if constexpr (!is_f32(T()))
    {
      if constexpr (D32 == 3 || D32 == 4)
        if (l.row_tiles == 3) return launch_rt<T, D32, 3, 2>(c, a, l, pa, st);
      if (l.row_tiles == 2) return launch_rt<T, D32, 2, 2>(c, a, l, pa, st);
    }
  return launch_rt<T, D32, 1, D32 <= 4 ? 4 : 2>(c, a, l, pa, st);
}

template <typename T>
hipError_t launch_t(const Fp4View& c, const Fp4Attention& a, const AttLaunch& l, const AttParts& pa, hipStream_t st) {
  switch (c.d / 32) {
    case 1: return launch_d<T, 1>(c, a, l, pa, st);
    case 2: return launch_d<T, 2>(c, a, l, pa, st);
    case 3: return launch_d<T, 3>(c, a, l, pa, st);
    case 4: return launch_d<T, 4>(c, a, l, pa, st);
    case 5: return launch_d<T, 5>(c, a, l, pa, st);
    case 6: return launch_d<T, 6>(c, a, l, pa, st);
    case 7: return launch_d<T, 7>(c, a, l, pa, st);
    default: return launch_d<T, 8>(c, a, l, pa, st);
  }
}

}  // namespace

size_t fp4_attention_bytes(const Fp4View& c, int Hq, int dtype, int n, int64_t n_tokens, int max_rows) {
  // (whether the tokens are one each is not known here: the larger of both)
  size_t most = 0;
  for (int one = 0; one <= (n_tokens == n ? 1 : 0); ++one) {
    const AttLaunch l = plan_attention(c, Hq, dtype, n, n_tokens, max_rows, one, true);
    const size_t bytes = l.slots * l.plan.ws_rows * (2 * sizeof(unsigned long long) + c.d * sizeof(float));
    if (bytes > most) most = bytes;
  }
  return most;
}

namespace {
// The launch of a call: not shared out where its turns are more than an int holds.
AttLaunch plan_call(const Fp4View& c, int dtype, const Fp4Attention& a, bool cut) {
  const AttLaunch l = plan_attention(c, a.Hq, dtype, a.n, a.n_tokens, a.max_rows, a.start == nullptr, cut);
  const int turn = ATT_WAVES * l.key_tiles * 16;
  const long long turns = (long long)a.blocks_per_inst * c.block_rows / turn + 1 + COLUMN_TURNS;      // of a column at most
  if (!l.shares || turns * a.n * c.Hkv * l.plan.tiles_per <= 0x7fffffff) return l;
  return plan_attention(c, a.Hq, dtype, a.n, a.n_tokens, a.max_rows, true, false);
}
}  // namespace

bool fp4_attention_fits(const Fp4View& c, int dtype, const Fp4Attention& a, bool cut) {
  return plan_call(c, dtype, a, cut).workgroups < (1ll << 32) / ATT_THREADS;
}

hipError_t launch_fp4_attention(const Fp4View& c, int dtype, const Fp4Attention& a, void* ws, hipStream_t st) {
  static std::atomic<uint32_t> launches{(uint32_t)(std::chrono::steady_clock::now().time_since_epoch().count() * 0x9E3779B97F4A7C15ull >> 32)};
  const AttLaunch l = plan_call(c, dtype, a, ws != nullptr);
  AttParts pa{static_cast<unsigned long long*>(ws), nullptr, 0};
  if (l.slots) {
    pa.sums = reinterpret_cast<float*>(pa.marks + 2 * l.slots * l.plan.ws_rows);
    do pa.nonce = launches.fetch_add(1); while (pa.nonce == 0);        // 0 is the cleared mark
  }
  return dtype == LAQ_BF16 ? launch_t<uint16_t>(c, a, l, pa, st) : launch_t<float>(c, a, l, pa, st);
}

}  // namespace laq
