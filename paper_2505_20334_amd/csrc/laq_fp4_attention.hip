// Attention over the paged 4-bit cache (include/laq_fp4.h: laq_fp4_attention).
//
// A workgroup has one KV head of a request, a tile of its score rows (row r = query head r % G of the group of the request's token r / G) and a
// part of the cache.  Its four waves take steps of 16 * KT keys in turn, every wave for all rows of the tile, each with its own running
// reference m, sum z and sums O (one pass, exponentials of s - m); they are folded at the end through LDS, the parts of a cache by
// the workgroup that finds all of them finished, in a fixed order.
//
// Products are 16 x 16 x 32 bf16 with the keys as the first operand's rows, so that a lane has four keys of one score row (column n = lane % 16) and all that
// belongs to a row lies in lanes n, n + 16, n + 32, n + 48:
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
  int32_t parts, part_rows;              // a request's rows in parts of part_rows, `parts` at most (the last one takes what is left)
  int32_t tiles_per;                     // without `start`: tiles of a request
  int32_t ws_rows;                       // rows of a tile that can be there
  int32_t adv_blocks, adv_tiles;         // what a wave's step moves a position (block, key tile in it) by
};

// Channel of number i of group t of lane quarter h: whole pieces of a row where scale blocks and pieces fit each other, else 8 of each block.
template <int D32> constexpr bool PIECES = D32 == 1 || D32 == 2 || D32 == 4 || D32 == 8;
template <int D32> __device__ __forceinline__ int channel_of(int t, int h) { return PIECES<D32> ? h * 8 * D32 + 8 * t : 32 * t + 8 * h; }

// A lane's codes and scales of a key row.
template <int D32>
struct KeyPiece {
  static constexpr int NS = !PIECES<D32> ? D32 : D32 == 8 ? 2 : 1;
  uint32_t c[D32];
  uint32_t s[NS];
  // codes, scales: of the tile's first row (uniform); the offsets: of this lane's
  __device__ __forceinline__ void read(const uint8_t* codes, const uint8_t* scales, uint32_t code_at, uint32_t scale_at) {
    if constexpr (PIECES<D32>) {
      typedef uint32_t words __attribute__((ext_vector_type(D32 == 1 ? 2 : D32)));
      if constexpr (D32 == 1) {
        c[0] = *reinterpret_cast<const uint32_t*>(codes + code_at);
      } else if constexpr (D32 == 8) {
        const u32x4 a = *reinterpret_cast<const u32x4*>(codes + code_at), b = *reinterpret_cast<const u32x4*>(codes + code_at + 16);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          c[t] = a[t];
          c[t + 4] = b[t];
        }
      } else {
        const words w = *reinterpret_cast<const words*>(codes + code_at);
#pragma unroll
        for (int t = 0; t < D32; ++t) c[t] = w[t];
      }
    } else {
#pragma unroll
      for (int t = 0; t < D32; ++t) c[t] = *reinterpret_cast<const uint32_t*>(codes + code_at + 16 * t);
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) s[i] = scales[scale_at + i];
  }
  __device__ __forceinline__ u32x4 group(int t) const { return __builtin_bit_cast(u32x4, fp4_to_bf16(c[t], fp4_scale_value(s[scale_of(t)]))); }
  static __device__ __forceinline__ int scale_of(int t) { return !PIECES<D32> ? t : D32 == 8 ? t / 4 : 0; }
  // which of its scales stand for NaN; those blocks are 0 then
  __device__ __forceinline__ uint32_t take_nan() {
    uint32_t found = 0;
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (s[i] == 255u) {
        found |= 1u << i;
        s[i] = 127;
#pragma unroll
        for (int t = 0; t < D32; ++t)
          if (scale_of(t) == i) c[t] = 0;
      }
    return found;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < D32; ++t) c[t] = 0;
#pragma unroll
    for (int i = 0; i < NS; ++i) s[i] = 127;
  }
};
// offsets of a lane's piece in a row
template <int D32> __device__ __forceinline__ uint32_t piece_codes(int h) { return PIECES<D32> ? h * 4 * D32 : 4 * h; }
template <int D32> __device__ __forceinline__ uint32_t piece_scales(int h) { return !PIECES<D32> ? 0 : h * D32 / 4; }

// A tile's request and rows.
struct AttTile {
  int inst, token0, T;                   // request, its first token, its tokens
  int first_row, n_rows;                 // score rows of this tile among the request's T * G
  int held;                              // rows of the cache
  int seen_min, seen_max;                // rows that the first and the last score row see
  int parts;
};
// The rows that score row r of the request sees.
__device__ __forceinline__ int rows_seen(const AttTile& t, int r, int G) { return min(max(t.held - t.T + r / G + 1, 0), t.held); }

template <int TR>
__device__ __forceinline__ bool find_tile(const Fp4View& c, const Fp4Attention& a, const AttPlan& p, int tile, int G, AttTile* out) {
  int tin;
  if (!a.start) {
    out->inst = tile / p.tiles_per;
    tin = tile - out->inst * p.tiles_per;
    out->token0 = out->inst;
    out->T = 1;
  } else {
    // request i has the tiles from start[i] * G / TR + i on: never fewer than it needs
    const auto start = [&](int i) { return min(max(a.start[i], 0), (int)a.n_tokens); };
    int lo = 0, hi = a.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((int)((uint32_t)(start(mid) * G) / TR) + mid <= tile) lo = mid; else hi = mid;
    }
    out->inst = lo;
    out->token0 = start(lo);
    out->T = max(start(lo + 1) - out->token0, 0);
    tin = tile - ((int)((uint32_t)(out->token0 * G) / TR) + lo);
  }
  if (tin < 0) return false;             // (a `start` that does not begin with 0)
  out->first_row = tin * TR;
  out->n_rows = min(out->T * G - out->first_row, TR);
  if (out->n_rows <= 0) return false;
  out->held = (int)min((long long)max(a.rows[out->inst], 0), (long long)a.blocks_per_inst * c.block_rows);
  out->seen_min = rows_seen(*out, out->first_row, G);
  out->seen_max = rows_seen(*out, out->first_row + out->n_rows - 1, G);
  out->parts = min(p.parts, max((out->seen_max + p.part_rows - 1) / p.part_rows, 1));
  return true;
}

// Eight numbers of a query row as the operand's parts.
template <typename T> constexpr int PARTS_OF = is_f32(T()) ? 3 : 1;

template <typename T, int D32, int RT>
__device__ __forceinline__ void read_queries(const Fp4Attention& a, const AttTile& tl, int kv, int G, int lane, u32x4 (&q)[RT][D32][PARTS_OF<T>],
                                             float (&factor)[RT]) {
  const int n = lane & 15, h = lane >> 4;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = rt * 16 + n, row = tl.first_row + r;
    const bool there = r < tl.n_rows;
    const int t = row / G, g = row - t * G;
    const T* src = static_cast<const T*>(a.q) + (int64_t)(tl.token0 + (there ? t : 0)) * a.stride_token + (int64_t)(kv * G + (there ? g : 0)) * a.stride_head;
    factor[rt] = fmaxf(a.scale2, 0x1p-126f);           // (not 0: a masked product is -infinity)
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
      factor[rt] = fmaxf(ldexpf(a.scale2, -shift), 0x1p-126f);
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

// The sum of eight weights' parts: four of one key tile, four of the next.
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

// The parts of cut caches: part s of column (tile, KV head) has sums[column][s][ws_rows][d], and per row two words
// marks[column][s][ws_rows][2]: the launch's nonce with the reference, and with the sum of weights.
struct AttParts {
  unsigned long long* marks;
  float* sums;
  uint32_t nonce;                        // a number that no other recent launch of the process has
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

// Folds the parts of a column, in their order, if all of them are finished (decode attention's way, laq_decode.hip): every part sets its marks
// after its sums have been written and then looks at the marks of all.  Whoever finds all of them set clears them, so that a captured
// launch, whose nonce is the same every time, never finds its own old ones; whatever else lies in the workspace is an unfinished part.
template <typename T>
__device__ void fold_parts(const Fp4View& c, const Fp4Attention& a, const AttPlan& p, const AttTile& tl, const AttParts& pa, size_t column, int kv, int G,
                           float* sm) {
  const int tid = threadIdx.x, S = tl.parts, R = tl.n_rows;
  unsigned long long* const marks = pa.marks + column * p.parts * p.ws_rows * 2;
  const float* const sums = pa.sums + column * p.parts * p.ws_rows * c.d;
  float *sm_m = sm, *sm_z = sm + S * R;
  bool all = true;
  for (int i = tid; i < S * R; i += ATT_THREADS) {
    const int s = i / R, r = i - s * R;
    const unsigned long long* mark = marks + ((size_t)s * p.ws_rows + r) * 2;
    const uint2 m = load_pair(mark), z = load_pair(mark + 1);
    all = all && m.x == pa.nonce && z.x == pa.nonce;
    sm_m[i] = __uint_as_float(m.y);
    sm_z[i] = __uint_as_float(z.y);
  }
  if (!__syncthreads_and(all)) return;
  for (int i = tid; i < S * R; i += ATT_THREADS) {
    unsigned long long* mark = marks + ((size_t)(i / R) * p.ws_rows + i % R) * 2;
    store_pair(mark, 0, 0);
    store_pair(mark + 1, 0, 0);
  }
  const int pairs = c.d / 2;
  for (int e = tid; e < R * pairs; e += ATT_THREADS) {
    const int r = e / pairs, col = (e - r * pairs) * 2;
    float M = -INFINITY;
    for (int s = 0; s < S; ++s) M = fmaxf(M, sm_m[s * R + r]);
    const float ref = M == -INFINITY ? 0.f : M;
    float Z = 0.f, x = 0.f, y = 0.f;
#pragma unroll 8
    for (int s = 0; s < S; ++s) {
      const float w = __builtin_amdgcn_exp2f(sm_m[s * R + r] - ref);
      const uint2 o = load_pair(sums + ((size_t)s * p.ws_rows + r) * c.d + col);
      Z = fmaf(sm_z[s * R + r], w, Z);
      x = fmaf(__uint_as_float(o.x), w, x);
      y = fmaf(__uint_as_float(o.y), w, y);
    }
    x = Z == 0.f ? 0.f : x / Z;
    y = Z == 0.f ? 0.f : y / Z;
    const size_t to = out_row(a, tl, kv, G, r);
    if constexpr (is_f32(T())) *reinterpret_cast<float2*>(static_cast<T*>(a.out) + to * c.d + col) = float2{x, y};
    else *reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + to * c.d + col) = pack2(x, y);
    if (a.lse && col == 0) a.lse[to] = Z == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(Z)) * LN2;
  }
}

template <typename T, int D32, int RT, int KT>
__global__ __launch_bounds__(ATT_THREADS) void fp4_attention_kernel(Fp4View c, Fp4Attention a, AttPlan p, AttParts pa) {
  constexpr int TR = 16 * RT, NP = PARTS_OF<T>;
  constexpr int CG = D32 < 4 ? D32 : 4, CHUNKS = (D32 + 3) / 4;        // groups of a chunk of V's channels (32 columns each), chunks
  constexpr int STRIDE = CG * 64 + 32;                                  // bytes of a key's row of a chunk in LDS
  constexpr int OSTRIDE = CG * 32 + 4;                                  // floats of a row's sums in LDS
  constexpr int V_BYTES = 32 * STRIDE, O_BYTES = 16 * OSTRIDE * 4;
  constexpr int WAVE_BYTES = V_BYTES > O_BYTES ? V_BYTES : O_BYTES;
  __shared__ __align__(16) unsigned char lds[ATT_WAVES * WAVE_BYTES];
  __shared__ float sm_m[ATT_WAVES][TR], sm_z[ATT_WAVES][TR];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, h = lane >> 4;
  const int G = a.Hq / c.Hkv, kv = blockIdx.x % c.Hkv, rest = blockIdx.x / c.Hkv, part = rest % p.parts, tile = rest / p.parts;
  AttTile tl;
  if (!find_tile<TR>(c, a, p, tile, G, &tl) || part >= tl.parts) return;

  u32x4 q[RT][D32][NP];
  float factor[RT];
  read_queries<T, D32, RT>(a, tl, kv, G, lane, q, factor);
  int seen[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) seen[rt] = rows_seen(tl, tl.first_row + min(rt * 16 + n, tl.n_rows - 1), G);

  // key tiles of this part, and this wave's position: tile `at`, in block `block` of the request its tile `in_block`
  const int first = part * p.part_rows / 16;
  const int end = part == tl.parts - 1 ? (tl.seen_max + 15) / 16 : (part + 1) * p.part_rows / 16;
  const int per_block = c.block_rows / 16;
  int at = first + wave * KT, block = at / per_block, in_block = at - block * per_block;
  typedef __attribute__((address_space(4))) const int32_t* ConstTable;
  const ConstTable table = (ConstTable)(unsigned long long)(a.table + (size_t)tl.inst * a.blocks_per_inst);
  const uint8_t *kc = c.k.codes + kv * c.head, *ks = c.k.scales + kv * c.scale_head, *vc = c.v.codes + kv * c.head, *vs = c.v.scales + kv * c.scale_head;
  const uint32_t code_at = n * (uint32_t)c.row + piece_codes<D32>(h), scale_at = n * (uint32_t)c.scale_row + piece_scales<D32>(h);

  KeyPiece<D32> kp[KT], vp[KT];
  int64_t code_base[KT], scale_base[KT];
  uint32_t there = 0, there_v = 0;       // a bit for each tile of the step whose rows are there
  auto locate = [&] {                    // the tiles of the step at `at`: one look at the table for those of a block
    int b = block, r = in_block;
    bool good = false;
    there = 0;
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      if (i == 0 || r == 0) {
        int number = -1;
        if (at + i < end) number = table[b];
        good = number >= 0 && number < c.n_blocks;
        const int64_t num = good ? number : 0, row = good ? r * 16 : 0;
        code_base[i] = num * c.block + row * c.row;
        scale_base[i] = num * c.scale_block + row * c.scale_row;
      } else {
        code_base[i] = code_base[i - 1] + (good ? 16 * c.row : 0);
        scale_base[i] = scale_base[i - 1] + (good ? 16 * c.scale_row : 0);
      }
      there |= good && at + i < end ? 1u << i : 0u;
      if (++r == per_block) {
        r = 0;
        ++b;
      }
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
  unsigned char* const my_lds = lds + wave * WAVE_BYTES;
  unsigned char* const v_write = my_lds + n * STRIDE + h * 16;
  const uint32_t v_read = (uint32_t)(4 * h + n / 4) * STRIDE + (n & 3) * 8;
  typedef __attribute__((address_space(3))) s16x4* LdsQuad;

  if (at < end) {
    locate();
    there_v = there;
#pragma unroll
    for (int i = 0; i < KT; ++i) kp[i].read(kc + code_base[i], ks + scale_base[i], code_at, scale_at);
#pragma unroll
    for (int i = 0; i < KT; ++i) vp[i].read(vc + code_base[i], vs + scale_base[i], code_at, scale_at);
  }
#pragma unroll 1
  while (at < end) {
    f32x4 s[RT][KT];
#pragma unroll
    for (int i = 0; i < KT; ++i) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < D32; ++t) {
        const u32x4 k8 = kp[i].group(t);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int pl = 0; pl < NP; ++pl) s[rt][i] = mfma16(k8, q[rt][t][NP - 1 - pl], s[rt][i]);
      }
    }
    const int key0 = at * 16;
    const bool masked = key0 + KT * 16 > tl.seen_min || there_v != (1u << KT) - 1;
    advance();
    if (at < end) {
      locate();
#pragma unroll
      for (int i = 0; i < KT; ++i) kp[i].read(kc + code_base[i], ks + scale_base[i], code_at, scale_at);
    }
    if (masked) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!(there_v >> i & 1) || key0 + i * 16 + 4 * h + r >= seen[rt]) s[rt][i][r] = -INFINITY;
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
          const float moved = top * factor[rt], w = limit[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(off[rt] - moved);
          off[rt] = moved;
          limit[rt] = (moved + LEEWAY) / factor[rt];
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
          s[rt][i][r] = __builtin_amdgcn_exp2f(fmaf(s[rt][i][r], factor[rt], -off[rt]));
          z[rt] += s[rt][i][r];
        }
    }
    bool nan_rows = false;               // some V stands for NaN where not every row sees it
    uint32_t nan_at[KT];
    if (masked) {
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        if (!(there_v >> i & 1) || key0 + i * 16 + n >= tl.seen_max) vp[i].clear();
        nan_at[i] = vp[i].take_nan();
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
      auto stage = [&](int ch, bool ones) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int t = 0; t < CG; ++t)
            if (ch * CG + t < D32) {
              const uint32_t one = ones && nan_at[j + i] >> KeyPiece<D32>::scale_of(ch * CG + t) & 1 ? 0x3f803f80u : 0u;
              *reinterpret_cast<u32x4*>(v_write + i * 16 * STRIDE + t * 64) = ones ? u32x4{one, one, one, one} : vp[j + i].group(ch * CG + t);
            }
      };
      auto column = [&](int ct) {        // 32 keys of 16 columns
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)(my_lds + v_read + ct * 32));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)(my_lds + v_read + 16 * STRIDE + ct * 32));
        const uint2 x = __builtin_bit_cast(uint2, lo), y = __builtin_bit_cast(uint2, hi);
        return u32x4{x.x, x.y, y.x, y.y};
      };
#pragma unroll
      for (int ch = 0; ch < CHUNKS; ++ch) {
        // (LDS operations of a wave are done in their order: only the compiler has to keep it)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        stage(ch, false);
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
          stage(ch, true);
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            u32x4 sees;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int tile_of = j + x / 2, key = key0 + tile_of * 16 + 4 * h + (x & 1) * 2;
              const bool in = there_v >> tile_of & 1;
              sees[x] = (in && key < seen[rt] ? 0x3f80u : 0u) | (in && key + 1 < seen[rt] ? 0x3f800000u : 0u);
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
      }
    }
    if (at < end) {
      there_v = there;
#pragma unroll
      for (int i = 0; i < KT; ++i) vp[i].read(vc + code_base[i], vs + scale_base[i], code_at, scale_at);
    }
  }

  // fold the waves, 16 rows and a chunk of channels at a time
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    z[rt] += __shfl_xor(z[rt], 16);
    z[rt] += __shfl_xor(z[rt], 32);
    if (h == 0) {
      sm_m[wave][rt * 16 + n] = limit[rt] == -INFINITY ? -INFINITY : off[rt];
      sm_z[wave][rt * 16 + n] = z[rt];
    }
  }
  __syncthreads();
  const bool whole = tl.parts == 1;
  const size_t column = (size_t)tile * c.Hkv + kv, slot = (column * p.parts + part) * p.ws_rows;
  auto row_sum = [&](int r, float* top) {        // over the waves, of a row
    float M = sm_m[0][r];
#pragma unroll
    for (int w = 1; w < ATT_WAVES; ++w) M = fmaxf(M, sm_m[w][r]);
    const float ref = M == -INFINITY ? 0.f : M;
    float Z = 0.f;
#pragma unroll
    for (int w = 0; w < ATT_WAVES; ++w) Z = fmaf(sm_z[w][r], __builtin_amdgcn_exp2f(sm_m[w][r] - ref), Z);
    *top = M;
    return Z;
  };
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (rt * 16 >= tl.n_rows) break;
    float M = sm_m[0][rt * 16 + n];
#pragma unroll
    for (int w = 1; w < ATT_WAVES; ++w) M = fmaxf(M, sm_m[w][rt * 16 + n]);
    const float mine = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm_m[wave][rt * 16 + n] - M);
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
      for (int e = threadIdx.x; e < 16 * CG * 4; e += ATT_THREADS) {       // eight columns of a row: group t, quarter hh
        const int r = e / (CG * 4), t = e % (CG * 4) / 4, hh = e & 3, row = rt * 16 + r;
        if (row < tl.n_rows && ch * CG + t < D32) {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
          for (int w = 0; w < ATT_WAVES; ++w)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] += reinterpret_cast<const float*>(lds + w * WAVE_BYTES)[r * OSTRIDE + t * 32 + hh * 8 + i];
          const int channel = channel_of<D32>(ch * CG + t, hh);
          if (whole) {
            float top;
            const float Z = row_sum(row, &top);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = Z == 0.f ? 0.f : x[i] / Z;
            put8(static_cast<T*>(a.out) + out_row(a, tl, kv, G, row) * c.d + channel, x);
          } else {
#pragma unroll
            for (int i = 0; i < 8; i += 2) store_pair(pa.sums + (slot + row) * c.d + channel + i, __float_as_uint(x[i]), __float_as_uint(x[i + 1]));
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
      store_pair(pa.marks + (slot + row) * 2, pa.nonce, __float_as_uint(top));
      store_pair(pa.marks + (slot + row) * 2 + 1, pa.nonce, __float_as_uint(Z));
      stores_done();
    } else if (a.lse) {
      a.lse[out_row(a, tl, kv, G, row)] = Z == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(Z)) * LN2;
    }
  }
  if (whole) return;
  __syncthreads();
  fold_parts<T>(c, a, p, tl, pa, column, kv, G, reinterpret_cast<float*>(lds));
}

constexpr int ATT_PART_STEP = 256;         // rows of a part: a multiple of what the four waves take in a turn
constexpr long long ATT_WORKGROUPS = 1024;

struct AttLaunch {
  AttPlan plan;
  int row_tiles, key_tiles;              // RT, KT
  int n_tiles;
  size_t rows;                           // of all parts, in the workspace
};

AttLaunch plan_attention(const Fp4View& c, int Hq, int dtype, int n, int64_t n_tokens, int max_rows, bool one_each) {
  const int G = Hq / c.Hkv;
  const long long rows_each = one_each ? G : (n_tokens * G + n - 1) / n;        // score rows of a request, on average
  AttLaunch l;
  l.row_tiles = rows_each <= 16 || dtype == LAQ_F32 ? 1 : 2;
  l.key_tiles = l.row_tiles == 1 ? 4 : 2;
  if (c.d > 128) l.key_tiles = 2;
  const int TR = 16 * l.row_tiles;
  l.plan.tiles_per = (G + TR - 1) / TR;
  l.n_tiles = one_each ? n * l.plan.tiles_per : (int)(n_tokens * G / TR) + n;
  l.plan.ws_rows = one_each && G < TR ? G : TR;
  const long long busy = (one_each ? l.n_tiles : n_tokens * G / TR > n ? n_tokens * G / TR : n) * (long long)c.Hkv;
  long long parts = (ATT_WORKGROUPS + busy - 1) / busy;
  const long long most = (max_rows + ATT_PART_STEP - 1) / ATT_PART_STEP;
  if (parts > most) parts = most;
  // the folding workgroup has two words for every row and part in LDS: what the kernel's other use of it leaves room for
  const int fold_most = ATT_WAVES * 32 * ((c.d < 128 ? c.d : 128) * 2 + 32) / (8 * TR);
  if (parts > fold_most) parts = fold_most;
  const long long steps = (most + parts - 1) / parts;
  l.plan.part_rows = (int)(steps * ATT_PART_STEP);
  l.plan.parts = (int)((most + steps - 1) / steps);
  const int per_block = c.block_rows / 16, turn = ATT_WAVES * l.key_tiles;
  l.plan.adv_blocks = turn / per_block;
  l.plan.adv_tiles = turn % per_block;
  l.rows = l.plan.parts == 1 ? 0 : (size_t)l.n_tiles * c.Hkv * l.plan.parts * l.plan.ws_rows;
  return l;
}

template <typename T, int D32, int RT, int KT>
hipError_t launch_att(const Fp4View& c, const Fp4Attention& a, const AttLaunch& l, const AttParts& pa, hipStream_t st) {
  hipLaunchKernelGGL((fp4_attention_kernel<T, D32, RT, KT>), dim3((unsigned)((long long)l.n_tiles * c.Hkv * l.plan.parts)), dim3(ATT_THREADS), 0, st, c, a,
                     l.plan, pa);
  return hipGetLastError();
}

template <typename T, int D32>
hipError_t launch_d(const Fp4View& c, const Fp4Attention& a, const AttLaunch& l, const AttParts& pa, hipStream_t st) {
  if constexpr (is_f32(T())) {
    return launch_att<T, D32, 1, D32 <= 4 ? 4 : 2>(c, a, l, pa, st);
  } else {
    if (l.row_tiles == 1) return launch_att<T, D32, 1, D32 <= 4 ? 4 : 2>(c, a, l, pa, st);
    return launch_att<T, D32, 2, 2>(c, a, l, pa, st);
  }
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
  const size_t some = plan_attention(c, Hq, dtype, n, n_tokens, max_rows, false).rows;
  const size_t one = n_tokens == n ? plan_attention(c, Hq, dtype, n, n_tokens, max_rows, true).rows : 0;
  return (some > one ? some : one) * (2 * sizeof(unsigned long long) + c.d * sizeof(float));
}

bool fp4_attention_fits(const Fp4View& c, int Hq, int dtype, int n, int64_t n_tokens, int max_rows, bool one_each) {
  const AttLaunch l = plan_attention(c, Hq, dtype, n, n_tokens, max_rows, one_each);
  return (long long)l.n_tiles * c.Hkv * l.plan.parts < (1ll << 32) / ATT_THREADS;
}

hipError_t launch_fp4_attention(const Fp4View& c, int dtype, const Fp4Attention& a, void* ws, size_t, hipStream_t st) {
  AttLaunch l = plan_attention(c, a.Hq, dtype, a.n, a.n_tokens, a.max_rows, a.start == nullptr);
  if (!ws) l.plan.parts = 1;
  static std::atomic<uint32_t> launches{(uint32_t)(std::chrono::steady_clock::now().time_since_epoch().count() * 0x9E3779B97F4A7C15ull >> 32)};
  AttParts pa{static_cast<unsigned long long*>(ws), nullptr, 0};
  if (l.plan.parts > 1) {
    pa.sums = reinterpret_cast<float*>(pa.marks + 2 * l.rows);
    do pa.nonce = launches.fetch_add(1); while (pa.nonce == 0);        // 0 is the cleared mark
  }
  return dtype == LAQ_BF16 ? launch_t<uint16_t>(c, a, l, pa, st) : launch_t<float>(c, a, l, pa, st);
}

}  // namespace laq
