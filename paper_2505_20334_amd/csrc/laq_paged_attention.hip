// Attention over the paged cache of 32, 16 or 8 bits (include/laq_cache.h: laq_cache_attention).
//
// A column is a KV head of a request and a tile of 16 or 32 of its score rows (row r = query head r % G of the group of the request's token r / G).  The
// lengths, which the host does not know, are as unequal as requests are, so the keys of all columns are shared out evenly (laq_paged_columns.h): as many
// workgroups as the device holds, each with one range of a line of turns, which it finds from the lengths and which may end in one column and go on in the next.
// (A workgroup for a fixed number of rows and a second launch to join them: 128 requests of 1000 to 8192 rows 542 us, 373 so; a second launch takes 4 to 40.)
// Of a turn the four waves take 16 * KT keys each, every wave for all rows of the tile, with its own reference m, sum z and sums O (one pass, exponentials of s - m;
// m moves only when a score is more than 8 above it, so that the usual step has no maximum over lanes).  The waves are folded at the end through LDS, the
// ranges of a column by the workgroup that finds all of them finished, in a fixed order.
//
// Bound: memory.  128 requests x 8 heads x 1000 to 8192 rows of d = 128: bf16 2.43 GB in 371 us, 6.6 TB/s; 8 bits 1.22 GB in 208 us, 5.9 TB/s; 96 x 6144 rows of bf16 6.7 TB/s; the
// vector units are busy 16 % of the time, the matrix cores 6 % (four requests of 32768 to 131071 rows in 8 bits: 32 and 11 %).  Small calls: dependent trips to memory, about 11 us for 520 rows: lengths (2.4), table and asking for keys (2.6),
// keys and products (1.9), fold (0.9), sums, marks and join (3).  fp32 caches with more than 16 score rows: the matrix cores' fp32 rate, an eighth of bf16's for these products.
//
// No LDS on the way of K and V, and registers for one step: K's are read again as soon as the scores are made, V's as soon as the sums are, so that about a step of a
// wave is on its way at any time and its code is there once (two steps in turn, twice the registers and the code: four long requests in 8 bits 191 us, so 172).  Products have the keys as the first operand's rows, so that a lane has four keys of one score row (column n =
// lane % 16, keys 4g .. 4g + 3 of a tile for lane group g = lane / 16), and all that belongs to a score row lies in lanes n, n + 16, n + 32, n + 48:
//   S^T = K Q^T   a lane reads pieces of one key row, in the order of the operand (the sum over channels may take them in any order, Q the same)
//   O^T = V^T P^T P^T is where S^T left it: a lane group's keys are, by definition, its part of the keys summed over.  bf16 (16 x 16 x 32): a lane needs
//                 eight keys of one channel; it reads eight channels of its eight keys, and a permutation of 8 x 8 numbers in registers, two a
//                 instruction, makes the operands of eight products.  fp32 (16 x 16 x 4): one key a lane, so the pieces are operands as they are
// A lane's pieces of V are VN channels: its product row m of product e of piece h is channel (16 h + m) VN + e.
#include "laq_marks.h"
#include "laq_paged_columns.h"

namespace laq {

namespace {

constexpr int ATT_WAVES = 4, ATT_THREADS = 64 * ATT_WAVES;
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 acc) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, acc, 0, 0, 0); }

// Eight floats as sums of N bf16 each, each the nearest of what is left: of three nothing is (down to 2^-126).  ODD, for queries: the first part of a number beyond bf16's largest
// is that one, an infinity or a NaN is its first part, and nothing is left of it (weights are at most 2^8, or NaN, whose parts may all be).
template <int N, bool ODD>
__device__ __forceinline__ void split(f32x4 a, f32x4 b, u32x4* parts) {
  constexpr float MOST = 0x1.fep127f;
  float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}, first[8];
  bool is[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    is[i] = !ODD || __builtin_fabsf(x[i]) < __builtin_inff();
    first[i] = ODD && is[i] ? __builtin_amdgcn_fmed3f(x[i], -MOST, MOST) : x[i];
  }
#pragma unroll
  for (int p = 0; p < N; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t both = p == 0 ? pack2(first[2 * i], first[2 * i + 1]) : pack2(x[2 * i], x[2 * i + 1]);
      parts[p][i] = both;
      x[2 * i] -= __uint_as_float(both << 16);
      x[2 * i + 1] -= __uint_as_float(both & 0xffff0000u);
      if (ODD && p == 0) {
        x[2 * i] = is[2 * i] ? x[2 * i] : 0.f;
        x[2 * i + 1] = is[2 * i + 1] ? x[2 * i + 1] : 0.f;
      }
    }
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Workgroups that a compute unit holds of a kernel: what their registers leave (the compiler is told to keep to it), measured with one more or less: bf16, d = 128, 16 score rows, three
// 383 us against 371 (128 requests); fp32 over fp32, 32 score rows, one 299 against 253 (4 x 256 tokens over 2048); 8 bits, 32 score rows, two 54.7 against 53.7; in parts, two 92 and 121 against 68.
constexpr int resident(bool f32, int type, int d, int nt) {
  const bool parts = f32 && type != LAQ_F32;
  if (d <= 64) return nt == 1 && !parts ? 3 : 2;
  if (d <= 128) return nt == 1 ? 2 : parts || type == LAQ_E4M3 ? 1 : 2;
  return 1;
}

// Q: the queries' numbers (and what the products are made in), E: the cache's, D: head sizes up to D, NT: 16 score rows NT times.
template <typename Q, typename E, int D, int NT, bool W>
struct Kinds {
  static constexpr bool F32 = std::is_same<Q, float>::value, SCALED = std::is_same<E, E4m3>::value;
  // fp32: products of fp32 where the cache is, otherwise of bf16, in which the cache's numbers are exact, with queries and weights as sums of three
  static constexpr bool FLOATS = std::is_same<E, float>::value;
  static constexpr int PARTS = F32 && !FLOATS ? 3 : 1;
  // Parts of a weight for the product with V.  Of bf16 queries two, which leave 2^-16 of it: results are away from exact ones by no more than their own rounding, 0.0017 of themselves
  // (one part: 0.0018 to 0.0023).  Memory's time hides the second products: 128 requests 371 us, in 8 bits 207, 520 rows 12, 32 x 8 tokens 61, each +-1 % (two of 8192 rows, 256
  // tokens 166 -> 173); but not where 8 bits are converted for two tiles of score rows (32 x 8 tokens 50 -> 53): one there
  static constexpr int WEIGHTS = FLOATS ? 1 : F32 ? 3 : SCALED && NT == 2 ? 1 : 2;
  // the cache has infinities, which the later parts would make NaN of: they meet the first part alone
  static constexpr bool LATER_K = PARTS > 1 && !SCALED, LATER_V = WEIGHTS > 1 && !SCALED;
  static constexpr int KT = FLOATS ? 1 : SCALED ? 4 : 2;        // tiles of 16 keys a step
  static constexpr int KN = FLOATS ? 4 : 8, KP = D / (4 * KN);  // numbers of a piece of K; pieces of a lane's key row
  // A read of K is 16 bytes, KW pieces side by side: piece i of lane group g has the numbers from here on (8 bits read 8 bytes a lane: 128 requests 293 us, so 214)
  static constexpr int KW = 16 / (KN * (int)sizeof(E));
  static constexpr __host__ __device__ int k_channel(int i, int g) { return i / KW * (4 * KW * KN) + g * (KW * KN) + i % KW * KN; }
  // blocks of a multiple of a step's keys, so that a step lies in one: one descriptor for its tiles
  // (8 bits, whose steps have four tiles: 128 requests of 1000 to 8192 rows 214 -> 209 us, 12 tokens of fp32 with d = 256 244 -> 199; others +-1 %, and where registers
  // are short already it costs more: fp32 with d = 128 70 -> 83)
  static constexpr bool WIDE = W, MAY_BE_WIDE = SCALED && !(F32 && D <= 128 && NT == 1);
  static constexpr int SPANS = WIDE ? 1 : KT, SPAN = 16 * KT / SPANS;        // descriptors of a step; keys of each
  static constexpr int RESIDENT = resident(F32, FLOATS ? LAQ_F32 : SCALED ? LAQ_E4M3 : LAQ_BF16, D, NT);      // workgroups of a compute unit (a wave of each on every SIMD)
  static constexpr bool ONCE = NT == 1;                      // one workgroup reads a row: past the caches
  static constexpr int VN = FLOATS || D == 64 ? 4 : 8, VP = D / (16 * VN);
  static constexpr int OT = D / 16;                          // output tiles
  static constexpr int PAD = D + 4;
};

// The keys of a step as they came from memory.
template <typename K, typename E>
struct StepKeys {
  Raw<E, K::KN> k[K::KT][K::KP];
  Raw<E, K::VN> v[K::KT][4][K::VP];
  uint32_t ks[K::KT], vs[K::KT];                             // SCALED: of this lane's key row; of its four keys of V
  // of the step that is read next: where its spans begin (numbers; scales), and how many bytes of each there are (0: not there)
  int64_t base[K::SPANS], scales[K::SPANS];
  uint32_t bytes[K::SPANS];
};
// W pieces side by side, 16 bytes together.
template <bool ONCE, int W, typename R>
__device__ __forceinline__ void fetch_wide(R* r, __amdgpu_buffer_rsrc_t tile, int at) {
  struct Wide { u32x4 x; } w;
  fetch<ONCE>(w, tile, at);
  if constexpr (W == 1) {
    r[0].x = w.x;
  } else if constexpr (W == 2) {
    r[0].x = u32x2{w.x[0], w.x[1]};
    r[1].x = u32x2{w.x[2], w.x[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i].x = w.x[i];
  }
}

template <typename Q, typename E, int D, int NT, bool WIDE>
__global__ __launch_bounds__(ATT_THREADS, (Kinds<Q, E, D, NT, WIDE>::RESIDENT)) void paged_attention_kernel(PagedView c, PagedAttention a, AttPlan p, Partials part) {
  using K = Kinds<Q, E, D, NT, WIDE>;
  constexpr int STEP = 16 * K::KT, TURN = STEP * ATT_WAVES;
  __shared__ float sums[ATT_WAVES][16][K::PAD];
  __shared__ float2 marks[ATT_WAVES][16];
  __shared__ bool odds[ATT_WAVES];
  const int H = c.Hkv, G = a.Hq / H;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;

  __shared__ ShareScan<ATT_WAVES> scan;
  Share sh;
  if (!first_range<ATT_THREADS, TURN>(c, a, G, p, scan, sh)) return;

  for (;;) {
  const Column col = column_of(sh.req, G, p.tile, sh.tile);
  const int turns = p.shares ? turns_of<TURN>(sh.req) : 1, turns_here = (int)min((int64_t)(turns - sh.turn), sh.left), head = sh.head;
  if (col.rows == 0 && !p.shares) return;
  const bool cut = p.shares && turns_here < turns;
  const int keys = col.keys(G), from = (int)min((int64_t)keys, (int64_t)sh.turn * TURN);
  const int to = p.shares ? (int)min((int64_t)keys, (int64_t)(sh.turn + turns_here) * TURN) : keys;

  // the score rows of this lane's columns
  int last[NT];
  u32x4 q[NT][K::KP][K::PARTS];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = 16 * t + n;
    const bool on = r < col.rows;
    last[t] = on ? col.last(r, G) : 0x7fffffff;
    const int rr = col.row0 + (on ? r : 0);
    const Q* src = static_cast<const Q*>(a.q.x) + (int64_t)(col.token0 + rr / G) * a.q.token + (int64_t)(head * G + rr % G) * a.q.head;
#pragma unroll
    for (int i = 0; i < K::KP; ++i) {
      const int at = K::k_channel(i, g);
      const bool in = on && at < c.d;
      if constexpr (K::PARTS == 1) {
        q[t][i][0] = in ? *reinterpret_cast<const u32x4*>(src + at) : u32x4{};
      } else {
        const f32x4 a4 = in ? *reinterpret_cast<const f32x4*>(src + at) : f32x4{}, b4 = in ? *reinterpret_cast<const f32x4*>(src + at + 4) : f32x4{};
        split<K::PARTS, true>(a4, b4, q[t][i]);
      }
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

  // where the lane's pieces lie behind a tile's first row, in bytes (channels beyond d: the next row's or nothing, for nobody)
  const int row_bytes = (int)(c.row * sizeof(E));
  const int k_at = n * row_bytes + g * 16;
  int v_at[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v_at[j] = (4 * g + j) * row_bytes + n * (K::VN * (int)sizeof(E));
  const int tile_bytes = 16 * row_bytes;
  const E *kx = static_cast<const E*>(c.k.x) + head * c.head, *vx = static_cast<const E*>(c.v.x) + head * c.head;
  typedef __attribute__((address_space(4))) const int32_t* ConstTable;
  const ConstTable table = (ConstTable)(unsigned long long)(a.table + (int64_t)sh.request * a.blocks_per_inst);

  // this wave's steps: keys from + (wave + 4 i) * STEP on.  Its place in the blocks moves with it, and the blocks' numbers are asked for a step ahead
  struct Place { int page, off; } at{0, 0};
  const int turn_pages = TURN / c.block_rows, turn_rows = TURN - turn_pages * c.block_rows;
  const auto forward = [&](Place& w, int pages, int rows) {
    w.page += pages;
    w.off += rows;
    if (w.off >= c.block_rows) {
      w.off -= c.block_rows;
      ++w.page;
    }
  };
  int blocks[K::SPANS];                                      // of the step that is loaded next
  const auto ask = [&](int left) {
    Place w = at;
#pragma unroll
    for (int i = 0; i < K::SPANS; ++i) {
      blocks[i] = K::SPAN * i < left ? table[w.page] : -1;
      forward(w, 0, K::SPAN);
    }
  };
  // The step at `at`, with `left` keys from its beginning on (none: nothing is read).  Rows behind them are not read: zeros.  K first, which moves what is
  // there and where it lies to s; then V, which goes on to the next step.
  const auto load_k = [&](int left, StepKeys<K, E>& s) {
    Place w = at;
#pragma unroll
    for (int i = 0; i < K::SPANS; ++i) {
      const bool there = (uint32_t)blocks[i] < (uint32_t)c.n_blocks;         // (-1 is not)
      const int block = there ? blocks[i] : 0;
      const int rows = min(K::SPAN, left - K::SPAN * i);
      s.bytes[i] = there ? (uint32_t)(rows - 1) * (uint32_t)row_bytes + (uint32_t)(c.d * (int)sizeof(E)) : 0u;
      s.base[i] = block * c.block + (int64_t)w.off * c.row;
      if constexpr (K::SCALED) s.scales[i] = ((int64_t)block * H + head) * c.block_rows + w.off;
      forward(w, 0, K::SPAN);
    }
#pragma unroll
    for (int kt = 0; kt < K::KT; ++kt) {
      const int i = WIDE ? 0 : kt, more = WIDE ? kt * tile_bytes : 0;
      const __amdgpu_buffer_rsrc_t kb = tile_of(kx + s.base[i], s.bytes[i]);
#pragma unroll
      for (int x = 0; x < K::KP; x += K::KW) fetch_wide<K::ONCE, K::KW>(&s.k[kt][x], kb, k_at + more + x / K::KW * 64);
      if constexpr (K::SCALED)
        s.ks[kt] = __builtin_amdgcn_raw_buffer_load_b8(tile_of(c.k.scales + s.scales[i], s.bytes[i] ? (uint32_t)K::SPAN : 0u), n + (WIDE ? 16 * kt : 0), 0, 0);
    }
    forward(at, turn_pages, turn_rows);
    ask(left - TURN);
  };
  const auto load_v = [&](StepKeys<K, E>& s) {
#pragma unroll
    for (int kt = 0; kt < K::KT; ++kt) {
      const int i = WIDE ? 0 : kt, more = WIDE ? kt * tile_bytes : 0;
      const __amdgpu_buffer_rsrc_t vb = tile_of(vx + s.base[i], s.bytes[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int x = 0; x < K::VP; ++x) fetch<K::ONCE>(s.v[kt][j][x], vb, v_at[j] + more + x * (16 * K::VN * (int)sizeof(E)));
      if constexpr (K::SCALED)
        s.vs[kt] = __builtin_amdgcn_raw_buffer_load_b32(tile_of(c.v.scales + s.scales[i], s.bytes[i] ? (uint32_t)K::SPAN : 0u), 4 * g + (WIDE ? 16 * kt : 0), 0, 0);
    }
  };

  const auto scale_of_v = [&](const StepKeys<K, E>& s, int kt, int j) { return e4m3_scale_value(s.vs[kt] >> (8 * j) & 255u); };
  // one step, and the reads of the next one: its K as soon as this one's is used, its V likewise, so that about a step is on its way at any time
  const auto compute = [&](int key, StepKeys<K, E>& s) {
    f32x4 x[NT][K::KT];
#pragma unroll
    for (int kt = 0; kt < K::KT; ++kt) {
#pragma unroll
      for (int t = 0; t < NT; ++t) x[t][kt] = f32x4{};
      const float ks = K::SCALED ? e4m3_scale_value(s.ks[kt]) : 1.f;
#pragma unroll
      for (int i = 0; i < K::KP; ++i) {
        if constexpr (K::FLOATS) {
          f32x4 k = floats(s.k[kt][i]);
          if (c.d != D && K::k_channel(i, g) >= c.d) k = f32x4{};
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[t][kt] = mfma(k[e], __uint_as_float(q[t][i][0][e]), x[t][kt]);
        } else {
          u32x4 k = pairs(s.k[kt][i], ks);
          if (c.d != D && K::k_channel(i, g) >= c.d) k = u32x4{};
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int part = K::PARTS - 1; part >= 0; --part) x[t][kt] = mfma(k, q[t][i][part], x[t][kt]);
        }
      }
    }
    if constexpr (K::LATER_K) {
      // (the later parts of a query are 0 or of either sign, and make a NaN of an infinity of K: what the first part leaves is multiplied with the finite numbers
      // alone.  Every score that an infinity spoils so is a NaN)
      bool bad = false;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int kt = 0; kt < K::KT; ++kt)
#pragma unroll
          for (int j = 0; j < 4; ++j) bad |= x[t][kt][j] != x[t][kt][j];
      if (__any(bad)) {
#pragma unroll
        for (int kt = 0; kt < K::KT; ++kt) {
#pragma unroll
          for (int t = 0; t < NT; ++t) x[t][kt] = f32x4{};
#pragma unroll
          for (int i = 0; i < K::KP; ++i) {
            if (c.d != D && K::k_channel(i, g) >= c.d) clear(s.k[kt][i]);
            const u32x4 k = pairs(s.k[kt][i], 1.f);
            drop_odd(s.k[kt][i]);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int part = K::PARTS - 1; part >= 0; --part) x[t][kt] = mfma(part ? pairs(s.k[kt][i], 1.f) : k, q[t][i][part], x[t][kt]);
          }
        }
      }
    }
    const int left = to - key;                                       // (keys of the step as far as `left`; sums with key could pass 2^31)
    bool there[K::KT], edge = min(left, first_last - key + 1) < STEP;   // a key that not every row sees
#pragma unroll
    for (int kt = 0; kt < K::KT; ++kt) {
      there[kt] = s.bytes[WIDE ? 0 : kt] != 0;
      edge |= !there[kt];
    }
    load_k(left - TURN, s);
    if (edge) {
#pragma unroll
      for (int kt = 0; kt < K::KT; ++kt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int at = 16 * kt + 4 * g + j;
          // (keys behind this range belong to nobody here)
#pragma unroll
          for (int t = 0; t < NT; ++t)
            if (!there[kt] || at >= left || at > last[t] - key) x[t][kt][j] = MINUS_INF;
          if constexpr (K::SCALED) s.vs[kt] = at >= left ? s.vs[kt] & ~(255u << (8 * j)) : s.vs[kt];      // (255 makes a NaN of the zeros)
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
    // added at the end.  (Of keys that nobody sees here nothing was read.)
    if (key > first_last - STEP + 1 && first_last < to - 1) {
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
            const bool none = vs == 255u;
#pragma unroll
            for (int i = 0; i < K::VP; ++i) {
              if (none) clear(s.v[kt][j][i]);
              else drop_odd(s.v[kt][j][i]);
            }
            if constexpr (K::SCALED) s.vs[kt] = none ? s.vs[kt] & ~(255u << (8 * j)) : s.vs[kt];
          }
        }
    }
    bool odd_v = false;                                              // an infinity or a NaN in V of the step
    if constexpr (K::LATER_V) {
      u16x2 most{};
#pragma unroll
      for (int kt = 0; kt < K::KT; ++kt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < K::VP; ++i)
#pragma unroll
            for (int w = 0; w < K::VN / 2; ++w) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, s.v[kt][j][i].x[w] & 0x7fff7fffu));
      odd_v = __any(most[0] >= 0x7f80 || most[1] >= 0x7f80);
    }
    if constexpr (K::FLOATS) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < K::VP; ++i) {
          const f32x4 v = floats(s.v[0][j][i]);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int t = 0; t < NT; ++t) o[t][i * K::VN + e] = mfma(v[e], x[t][0][j], o[t][i * K::VN + e]);
        }
    } else {
#pragma unroll
      for (int h = 0; h < K::KT; h += 2) {
        u32x4 w[NT][K::WEIGHTS];
#pragma unroll
        for (int t = 0; t < NT; ++t)
          split<K::WEIGHTS, false>(x[t][h], x[t][h + 1], w[t]);
        // [key][channel pair] to [channel][key pair], and the weights times them.  ODD: V's infinities and NaN alone, the weights' first part
        const auto products = [&](int i, auto odd_only) {
          constexpr bool ODD = decltype(odd_only)::value;
          using P = decltype(pairs(s.v[0][0][0], 1.f));
          P v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = pairs(s.v[h + j / 4][j % 4][i], K::SCALED ? scale_of_v(s, h + j / 4, j % 4) : 1.f);
#pragma unroll
          for (int e = 0; e < K::VN; ++e) {
            const auto word = [&](int j) { return ODD ? v[j][e / 2] ^ without_odd(v[j][e / 2], E{}) : v[j][e / 2]; };
            u32x4 f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = __builtin_amdgcn_perm(word(2 * j + 1), word(2 * j), e & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int part = ODD ? 0 : K::WEIGHTS - 1; part >= 0; --part) o[t][i * K::VN + e] = mfma(f, w[t][part], o[t][i * K::VN + e]);
          }
        };
        if constexpr (K::LATER_V) {
          // (the later parts of a weight are 0 or negative, and make a NaN of an infinity: V's odd numbers are multiplied with the first part alone, then V without them)
          if (odd_v) {
#pragma unroll
            for (int i = 0; i < K::VP; ++i) {
              products(i, std::true_type{});
#pragma unroll
              for (int j = 0; j < 8; ++j) drop_odd(s.v[h + j / 4][j % 4][i]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < K::VP; ++i) products(i, std::false_type{});
      }
    }
    load_v(s);
  };

  if (to - from > wave * STEP) {
    StepKeys<K, E> s;
    int key = from + wave * STEP;
    at.page = (int)((uint32_t)key / (uint32_t)c.block_rows);
    at.off = (int)((uint32_t)key - (uint32_t)at.page * c.block_rows);
    ask(to - key);
    load_k(to - key, s);
    load_v(s);
    for (;;) {
      compute(key, s);
      if (to - key <= TURN) break;
      key += TURN;
    }
  }

  // the waves' sums, score rows of 16 at a time
  const bool wave_odd = __any(odd);
  if (lane == 0) odds[wave] = wave_odd;
  const int64_t place = (int64_t)sh.place() * p.tile;
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
    constexpr int PER = D / 4;
    for (int i = threadIdx.x; i < 16 * PER; i += ATT_THREADS) {
      const int rr = i / PER, at = i % PER * 4, r = 16 * t + rr;
      if (r >= col.rows || at >= c.d) continue;
      float top = marks[0][rr].x, Z = marks[0][rr].y;
      f32x4 y = *reinterpret_cast<const f32x4*>(&sums[0][rr][at]);
      bool any_odd = odds[0];
#pragma unroll
      for (int v = 1; v < ATT_WAVES; ++v) {
        join(top, Z, y, marks[v][rr].x, marks[v][rr].y, *reinterpret_cast<const f32x4*>(&sums[v][rr][at]), a.scale2);
        any_odd |= odds[v];
      }
      if (any_odd) {
        const int upto = min(to - 1, col.last(r, G));
        for (int key = max(from, first_last + 1); key <= upto; ++key) {
          const int page = (int)((uint32_t)key / (uint32_t)c.block_rows), off = key - page * c.block_rows, block = table[page];
          if (block < 0 || block >= c.n_blocks) continue;
          const E* v = vx + block * c.block + (int64_t)off * c.row;
          const uint32_t vs = K::SCALED ? c.v.scales[((int64_t)block * H + head) * c.block_rows + off] : 0u;
          for (int e = 0; e < 4; ++e) {
            const float f = number(v, at + e, vs);
            if (f - f != 0.f) y[e] += f;
          }
        }
      }
      if (!cut) {
        put_out<Q>(c, a, col, head, G, r, at, top, Z, y);
      } else {
        if (at == 0) store_pair(part.mz + place + r, top, Z);
        store_pair(part.sums + (place + r) * c.d + at, y[0], y[1]);
        store_pair(part.sums + (place + r) * c.d + at + 2, y[2], y[3]);
      }
    }
  }
  if (!p.shares) return;
  if (cut) join_ranges<Q, ATT_THREADS, NT == 1 ? 8 : 4>(c, a, part, sh, col, G, p.tile, turns, &sums[0][0][0]);
  if (!next_column<TURN>(c, a, G, p.tile, turns, turns_here, sh)) return;
  __syncthreads();                                           // (the LDS is free)
  }
}

// ---- the host's part -------------------------------------------------------------------------

int tiles_of_rows(int d, int n, int64_t n_tokens, int G) {
  const int64_t rows = (n_tokens + n - 1) / n * G;                   // of a request, on average
  return rows <= 16 || d > 128 ? 1 : 2;
}

// max_rows 0: the most shares that a call of any bound has.
AttPlan plan_of(const PagedView& c, int Hq, int dtype, int n, int64_t n_tokens, bool has_start, int max_rows, bool may_share) {
  const int G = Hq / c.Hkv;
  AttPlan p;
  p.tile = 16 * tiles_of_rows(c.d, n, n_tokens, G);
  const int64_t columns = has_start ? n_tokens * G / p.tile + n : (int64_t)n * ((G + p.tile - 1) / p.tile);
  p.columns = (int32_t)(columns < 0x7fffffff ? columns : 0x7fffffff);
  p.shares = !may_share ? 0 : COMPUTE_UNITS * resident(dtype == LAQ_F32, c.type, c.d, p.tile / 16);
  if (may_share && max_rows > 0) {
    const int turn = ATT_WAVES * 16 * (c.type == LAQ_F32 ? 1 : c.type == LAQ_E4M3 ? 4 : 2);
    const int64_t turns = columns * c.Hkv * (((int64_t)max_rows + turn - 1) / turn);
    if (turns < p.shares) p.shares = (int32_t)turns;
  }
  return p;
}

struct Bytes {
  size_t marks, mz, sums;
  size_t all() const { return marks + mz + sums; }
};
Bytes bytes_of(const PagedView& c, const AttPlan& p) {
  const size_t rows = (size_t)p.shares * 2 * p.tile;
  return Bytes{((size_t)p.shares * 16 + 255) / 256 * 256, rows * sizeof(float2), rows * c.d * sizeof(float)};
}

template <typename Q, typename E, int D>
hipError_t start_attention(const PagedView& c, const PagedAttention& a, const AttPlan& p, const Partials& part, hipStream_t st) {
  const dim3 grid((unsigned)(p.shares ? p.shares : (int64_t)p.columns * c.Hkv));
  const auto start = [&](auto nt, auto wide) {
    hipLaunchKernelGGL((paged_attention_kernel<Q, E, D, nt(), wide()>), grid, dim3(ATT_THREADS), 0, st, c, a, p, part);
  };
  const auto by_blocks = [&](auto nt) {
    using K = Kinds<Q, E, D, nt(), true>;
    if constexpr (K::MAY_BE_WIDE) {
      if (c.block_rows % (16 * K::KT) == 0) return start(nt, std::true_type{});
    }
    start(nt, std::false_type{});
  };
  if constexpr (D <= 128) {
    if (p.tile == 32) {
      by_blocks(std::integral_constant<int, 2>{});
      return hipGetLastError();
    }
  }
  by_blocks(std::integral_constant<int, 1>{});
  return hipGetLastError();
}

template <typename Q, typename E>
hipError_t by_size(const PagedView& c, const PagedAttention& a, const AttPlan& p, const Partials& part, hipStream_t st) {
  if (c.d <= 64) return start_attention<Q, E, 64>(c, a, p, part, st);
  if (c.d <= 128) return start_attention<Q, E, 128>(c, a, p, part, st);
  return start_attention<Q, E, 256>(c, a, p, part, st);
}

}  // namespace

size_t paged_attention_bytes(const PagedView& c, int Hq, int dtype, int n, int64_t n_tokens, int) {
  if (paged_prompt_call(c, Hq, dtype, n, n_tokens)) return 0;
  return bytes_of(c, plan_of(c, Hq, dtype, n, n_tokens, true, 0, true)).all();
}

bool paged_attention_fits(const PagedView& c, int dtype, const PagedAttention& a, bool cut) {
  const AttPlan p = plan_of(c, a.Hq, dtype, a.n, a.n_tokens, a.start != nullptr, a.max_rows, cut);
  return paged_prompt_call(c, a.Hq, dtype, a.n, a.n_tokens) || p.shares || (int64_t)p.columns * c.Hkv < (1 << 24);
}

hipError_t launch_paged_attention(const PagedView& c, int dtype, const PagedAttention& a, void* ws, hipStream_t st) {
  if (paged_prompt_call(c, a.Hq, dtype, a.n, a.n_tokens)) return launch_paged_prompt(c, a, st);
  static MarkNumbers numbers;
  const AttPlan p = plan_of(c, a.Hq, dtype, a.n, a.n_tokens, a.start != nullptr, a.max_rows, ws != nullptr);
  const Bytes b = bytes_of(c, p);
  char* const at = static_cast<char*>(ws);
  Partials part{reinterpret_cast<unsigned long long*>(at), reinterpret_cast<float2*>(at + b.marks), reinterpret_cast<float*>(at + b.marks + b.mz), 0};
  if (ws) part.nonce = numbers.next();
  if (dtype == LAQ_BF16)
    return c.type == LAQ_BF16 ? by_size<uint16_t, uint16_t>(c, a, p, part, st) : by_size<uint16_t, E4m3>(c, a, p, part, st);
  switch (c.type) {
    case LAQ_F32: return by_size<float, float>(c, a, p, part, st);
    case LAQ_BF16: return by_size<float, uint16_t>(c, a, p, part, st);
    default: return by_size<float, E4m3>(c, a, p, part, st);
  }
}

}  // namespace laq
