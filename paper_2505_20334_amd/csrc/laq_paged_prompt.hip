// Attention of many tokens of a request over the paged cache, bf16 (laq_cache_attention for chunks of a prompt).
//
// A workgroup has a column of 128 score rows, a wave 32 of them, and goes through all keys that they see, 64 at a time, which lie in LDS for the four waves
// (two stages in turn: the next one is read while one is used; 8 bits become bf16 on the way).  Products are 32 x 32 x 16 with the keys (S^T = K Q^T), then the
// channels (O^T = V^T P^T), as the first operand's rows: a lane has 16 keys of one score row of each 32, and they are, as they are, its part of P^T.  V^T is read
// from LDS by its transposing read.  The 16-byte pieces of a row change places with the row's number so that reads meet in no bank.
// One pass, exponentials of s - m with a reference m that moves only when a score is more than 8 above it.
// Weights are rounded to bf16 for the product with V: results are 0.0023 of themselves away from exact ones, of which their own rounding is 0.0017.  In two parts it would be that alone,
// but the products are what takes the time here: 4 x 512 tokens 227 -> 286 us, 8 bits 253 -> 297, a prompt of 4096 tokens 161 -> 204.
//
// 4 x 512 tokens x 32 heads over 2100 to 8704 rows 229 us, 814 TFLOP/s; a prompt of 4096 tokens 161 us, 855 TFLOP/s; 8 bits 249 us.  Bound: the instructions beside the products (for 32 products of a stage and wave 190 vector instructions, 32 of them exponentials, 90
// scalar ones and 56 of LDS; vector units and matrix cores are each busy 35 % of the time), with two waves a SIMD to fill each other's waits, and, in a call like the first, columns of the longest request that run on alone when those beside them have ended.
// Sharing the keys out evenly as the other kernel does was slower: sums of 128 rows of every cut column go through memory, and tokens early in a prompt see few keys (331 and 365 us against 297 and 236 then).
#include "laq_paged_columns.h"

namespace laq {

namespace {

constexpr int WAVES = 4, THREADS = 64 * WAVES, WAVE_ROWS = 32, TILE = WAVES * WAVE_ROWS, STAGE = 64;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* LdsQuad;

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 acc) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}

// LDS and memory operations and products stay on their side; other instructions may pass.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0x406); }

// Where piece `piece` (eight numbers) of row `row` lies in LDS, in numbers.
template <int D> __device__ __forceinline__ int k_place(int row, int piece) { return row * D + (piece ^ (row & (D / 8 - 1))) * 8; }
// (the transposing read takes half pieces of four rows at a time)
template <int D> __device__ __forceinline__ int v_place(int row, int piece) { return row * D + (piece ^ ((D == 64 ? row >> 1 & 1 : row & 3) << 2)) * 8; }

// Column number `rank` in the order in which the workgroups of up to 64 requests take them: requests with the most rows first, of each the last tiles first.
// The first 256 workgroups go to a compute unit each, the second 256 beside them, these in the opposite order, so that long columns lie beside short ones.
__device__ __forceinline__ bool ranked_column(const PagedView& c, const PagedAttention& a, int G, int H, int rank, int* request, int64_t* tile, Request* req) {
  const int lane = threadIdx.x & 63;
  Request r{0, 0, 0};
  if (lane < a.n) r = request_of(a, c.block_rows, lane);
  const int tiles = lane < a.n ? tiles_of(r, G, TILE) : 0;
  int before = 0, all = 0;                                             // tiles of requests that come first; of all
  for (int i = 0; i < a.n; ++i) {
    const int held = __builtin_amdgcn_readlane(r.held, i), t = __builtin_amdgcn_readlane(tiles, i);
    if (held > r.held || (held == r.held && i < lane)) before += t;
    all += t;
  }
  if (rank >= all) return false;
  const int round = COMPUTE_UNITS / H;
  if (rank >= round && rank < 2 * round) rank = round + min(2 * round, all) - 1 - rank;
  const uint64_t mine = __ballot(rank >= before && rank < before + tiles);
  if (mine == 0) return false;
  const int l = __builtin_ctzll(mine);
  *request = l;
  *tile = __builtin_amdgcn_readlane(tiles, l) - 1 - (rank - __builtin_amdgcn_readlane(before, l));
  *req = Request{__builtin_amdgcn_readlane(r.token0, l), __builtin_amdgcn_readlane(r.tokens, l), __builtin_amdgcn_readlane(r.held, l)};
  return true;
}

// WIDE: blocks of a multiple of 64 rows, so that a stage lies in one (of a stage's 257 scalar instructions 87 are left: 4 x 512 tokens 259 -> 229 us).
template <typename E, int D, bool WIDE>
__global__ __launch_bounds__(THREADS, 2) void paged_prompt_kernel(PagedView c, PagedAttention a) {
  constexpr bool SCALED = std::is_same<E, E4m3>::value;
  constexpr int PIECES = D / 8, ROWS = THREADS / PIECES, PASSES = STAGE / ROWS;     // of a row; rows that the workgroup reads at once
  constexpr int KS = D / 16, DT = D / 32;
  __shared__ alignas(16) uint16_t k_lds[2][STAGE * D], v_lds[2][STAGE * D];
  const int H = c.Hkv, G = a.Hq / H;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
  const int head = blockIdx.x % H;
  int request;
  int64_t tile;
  Request req;
  if (a.n <= 64) {
    if (!ranked_column(c, a, G, H, blockIdx.x / H, &request, &tile, &req)) return;
  } else {
    const int slot = blockIdx.x / H;
    request = find_request(a, G, TILE, slot);
    tile = slot - first_column(a, G, TILE, request);
    req = request_of(a, c.block_rows, request);
  }
  const Column col = column_of(req, G, TILE, tile);
  if (col.rows == 0) return;
  const int to = col.keys(G), first_last = col.last(0, G);             // all rows see the keys up to first_last

  // this wave's score rows
  const int r = wave * WAVE_ROWS + n;
  const bool on = r < col.rows;
  const int last = on ? col.last(r, G) : 0x7fffffff;
  const int wave_first = col.last(wave * WAVE_ROWS, G);                // (of rows that are not there: more than all keys)
  const int wave_to = wave * WAVE_ROWS < col.rows ? min(to, col.last(min(wave * WAVE_ROWS + WAVE_ROWS, col.rows) - 1, G) + 1) : 0;
  const int row = col.row0 + (on ? r : 0);
  u32x4 q[KS];
  {
    const uint16_t* src = static_cast<const uint16_t*>(a.q.x) + (int64_t)(col.token0 + row / G) * a.q.token + (int64_t)(head * G + row % G) * a.q.head;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int at = (2 * i + h) * 8;
      q[i] = on && at < c.d ? *reinterpret_cast<const u32x4*>(src + at) : u32x4{};
    }
  }
  f32x16 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x16{};
  float m = MINUS_INF, above = MINUS_INF, less = 0.f, z = 0.f;
  const float margin = 8.f / a.scale2;
  bool odd = false;                                                    // an infinity or a NaN in V that not every row of the column sees

  // stages: this thread's pieces of 64 rows
  const int piece = threadIdx.x % PIECES, my_row = threadIdx.x / PIECES, wave_row = wave * (64 / PIECES);
  const int row_bytes = (int)(c.row * sizeof(E));
  // (channels beyond d: behind the end, where nothing is read; zeros)
  const int pass_bytes = piece * 8 < c.d ? ROWS * row_bytes : 0;
  const int my_at = piece * 8 < c.d ? (WIDE ? my_row : my_row & 15) * row_bytes + piece * (8 * (int)sizeof(E)) : 0x7fffffff - 16;
  const E *kx = static_cast<const E*>(c.k.x) + head * c.head, *vx = static_cast<const E*>(c.v.x) + head * c.head;
  typedef __attribute__((address_space(4))) const int32_t* ConstTable;
  const ConstTable table = (ConstTable)(unsigned long long)(a.table + (int64_t)request * a.blocks_per_inst);
  Raw<E, 8> k[PASSES], v[PASSES];
  uint32_t ks[PASSES], vs[PASSES];
  int page = 0, off = 0, blocks[STAGE / 16];                           // of the stage that is read next
  uint32_t there_next = 0, there = 0;                                  // a bit for each tile of 16 rows: of the stage on its way; of the one in use
  const auto ask = [&](int left) {
    if constexpr (WIDE) {
      blocks[0] = left > 0 ? table[page] : -1;
      return;
    }
    int pg = page, of = off;
#pragma unroll
    for (int i = 0; i < STAGE / 16; ++i) {
      blocks[i] = 16 * i < left ? table[pg] : -1;
      of += 16;
      if (of >= c.block_rows) {
        of = 0;
        ++pg;
      }
    }
  };
  const auto load = [&](int left) {
    if constexpr (WIDE) {
      const bool is = (uint32_t)blocks[0] < (uint32_t)c.n_blocks;      // (-1 is not)
      const int block = is ? blocks[0] : 0;
      const int64_t base = block * c.block + (int64_t)off * c.row;
      const uint32_t bytes = is ? (uint32_t)(min(STAGE, left) - 1) * (uint32_t)row_bytes + (uint32_t)(c.d * (int)sizeof(E)) : 0u;
      const __amdgpu_buffer_rsrc_t kb = tile_of(kx + base, bytes), vb = tile_of(vx + base, bytes);
      there_next = is ? 15u : 0u;
#pragma unroll
      for (int u = 0; u < PASSES; ++u) {
        fetch<false>(k[u], kb, my_at + u * pass_bytes);
        fetch<false>(v[u], vb, my_at + u * pass_bytes);
      }
      if constexpr (SCALED) {
        const int64_t sc = ((int64_t)block * H + head) * c.block_rows + off;
        const __amdgpu_buffer_rsrc_t ksb = tile_of(c.k.scales + sc, is ? (uint32_t)STAGE : 0u), vsb = tile_of(c.v.scales + sc, is ? (uint32_t)STAGE : 0u);
#pragma unroll
        for (int u = 0; u < PASSES; ++u) {
          ks[u] = __builtin_amdgcn_raw_buffer_load_b8(ksb, my_row + u * ROWS, 0, 0);
          vs[u] = __builtin_amdgcn_raw_buffer_load_b8(vsb, my_row + u * ROWS, 0, 0);
        }
      }
      off += STAGE;
      if (off >= c.block_rows) {
        off = 0;
        ++page;
      }
      ask(left - STAGE);
      return;
    }
    int64_t base[STAGE / 16], scales[STAGE / 16];
    uint32_t bytes[STAGE / 16];
    there_next = 0;
#pragma unroll
    for (int i = 0; i < STAGE / 16; ++i) {
      const bool is = (uint32_t)blocks[i] < (uint32_t)c.n_blocks;      // (-1 is not)
      const int block = is ? blocks[i] : 0;
      there_next |= (uint32_t)is << i;
      base[i] = block * c.block + (int64_t)off * c.row;
      if constexpr (SCALED) scales[i] = ((int64_t)block * H + head) * c.block_rows + off;
      bytes[i] = is ? (uint32_t)(min(16, left - 16 * i) - 1) * (uint32_t)row_bytes + (uint32_t)(c.d * (int)sizeof(E)) : 0u;
      off += 16;
      if (off >= c.block_rows) {
        off = 0;
        ++page;
      }
    }
#pragma unroll
    for (int u = 0; u < PASSES; ++u) {
      int t = 0;                                                       // the tile of this wave's rows
      if constexpr (ROWS == 16) t = u;
      else t = u * (ROWS / 16) + wave_row / 16;
      int64_t b = base[0], sc = scales[0];
      uint32_t by = bytes[0];
#pragma unroll
      for (int i = 1; i < STAGE / 16; ++i) {
        b = t == i ? base[i] : b;
        sc = t == i ? scales[i] : sc;
        by = t == i ? bytes[i] : by;
      }
      fetch<false>(k[u], tile_of(kx + b, by), my_at);
      fetch<false>(v[u], tile_of(vx + b, by), my_at);
      if constexpr (SCALED) {
        ks[u] = __builtin_amdgcn_raw_buffer_load_b8(tile_of(c.k.scales + sc, by ? 16u : 0u), my_row & 15, 0, 0);
        vs[u] = __builtin_amdgcn_raw_buffer_load_b8(tile_of(c.v.scales + sc, by ? 16u : 0u), my_row & 15, 0, 0);
      }
    }
    ask(left - STAGE);
  };
  // the pieces to LDS; `key`, `left`: of the stage
  const auto put = [&](int buf, int key, int left) {
    const bool edge = left <= STAGE || key > first_last - STAGE;       // rows behind the end, or that not every row sees
#pragma unroll
    for (int u = 0; u < PASSES; ++u) {
      const int rr = u * ROWS + my_row;
      if (edge) {
        if (SCALED && rr >= left) ks[u] = vs[u] = 0;                   // (255 makes a NaN of the zeros)
        if (rr > first_last - key) {
          odd |= has_odd(v[u], SCALED ? vs[u] : 0u);
          drop_odd(v[u]);
          if (SCALED && vs[u] == 255u) {
            clear(v[u]);
            vs[u] = 0;
          }
        }
      }
      const u32x4 kk = pairs(k[u], SCALED ? e4m3_scale_value(ks[u]) : 1.f), vv = pairs(v[u], SCALED ? e4m3_scale_value(vs[u]) : 1.f);
      *reinterpret_cast<u32x4*>(&k_lds[buf][k_place<D>(rr, piece)]) = kk;
      *reinterpret_cast<u32x4*>(&v_lds[buf][v_place<D>(rr, piece)]) = vv;
    }
  };

  const int v_row = 4 * h + (lane & 15) / 4, v_channel = (lane >> 4 & 1) * 16 + (lane & 3) * 4;
  const auto compute = [&](int buf, int key) {
    // LDS reads are asked for a group of products ahead, and kept there: left to itself the compiler puts each in front of its product and waits for it
    constexpr int GROUP = 4, K_GROUPS = 2 * KS / GROUP, PER = KS / GROUP;
    f32x16 x[2] = {};
    u32x4 kf[2][GROUP];
    const auto read_k = [&](int gr, u32x4* f) {
#pragma unroll
      for (int j = 0; j < GROUP; ++j) f[j] = *reinterpret_cast<const u32x4*>(&k_lds[buf][k_place<D>(32 * (gr / PER) + n, 2 * (gr % PER * GROUP + j) + h)]);
    };
    read_k(0, kf[0]);
#pragma unroll
    for (int gr = 0; gr < K_GROUPS; ++gr) {
      if (gr + 1 < K_GROUPS) read_k(gr + 1, kf[(gr + 1) & 1]);
      keep_order();
#pragma unroll
      for (int j = 0; j < GROUP; ++j) x[gr / PER] = mfma(kf[gr & 1][j], q[gr % PER * GROUP + j], x[gr / PER]);
      keep_order();
    }
    u32x4 vf[2][DT];
    const auto read_v = [&](int gr, u32x4* f) {                        // 16 keys
      const int row0 = 16 * gr + v_row;
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const int ch = 32 * i + v_channel;
        const uint2 l = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)&v_lds[buf][v_place<D>(row0, ch / 8) + (ch & 4)]));
        const uint2 u = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad)&v_lds[buf][v_place<D>(row0 + 8, ch / 8) + (ch & 4)]));
        f[i] = u32x4{l.x, l.y, u.x, u.y};
      }
    };
    read_v(0, vf[0]);
    keep_order();
    if (key > wave_first - STAGE || there != 15u) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int at = 32 * s + 8 * (e / 4) + 4 * h + e % 4;
          if (!(there >> (2 * s + e / 8) & 1u) || at >= to - key || at > last - key) x[s][e] = MINUS_INF;
        }
    }
    float most = x[0][0];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int e = 0; e < 16; ++e) most = fmaxf(most, x[s][e]);
    if (__any(most > above)) {
      most = fmaxf(most, m);
      most = fmaxf(most, __shfl_xor(most, 32));
      if (most > m) {
        const float by = m == MINUS_INF ? 0.f : __builtin_amdgcn_exp2f((m - most) * a.scale2);
        m = most;
        above = most + margin;
        less = most * a.scale2;
        z *= by;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] *= by;
      }
    }
#pragma unroll
    for (int gr = 0; gr < 4; ++gr) {                                   // 16 keys
      const int s = gr / 2, e0 = gr % 2 * 8;
      if (gr < 3) read_v(gr + 1, vf[(gr + 1) & 1]);
      keep_order();
#pragma unroll
      for (int e = e0; e < e0 + 8; ++e) {
        x[s][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[s][e], a.scale2, -less));
        z += x[s][e];
      }
      const u32x4 w{pack2(x[s][e0], x[s][e0 + 1]), pack2(x[s][e0 + 2], x[s][e0 + 3]), pack2(x[s][e0 + 4], x[s][e0 + 5]), pack2(x[s][e0 + 6], x[s][e0 + 7])};
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] = mfma(vf[gr & 1][i], w, o[i]);
      keep_order();
    }
  };

  if (to > 0) {
    ask(to);
    load(to);
    put(0, 0, to);
    there = there_next;
    load(to - STAGE);                                                  // (behind the end nothing is read)
    __syncthreads();
    int key = 0, buf = 0;
    for (;;) {
      if (key < wave_to) compute(buf, key);
      if (to - key <= STAGE) break;
      key += STAGE;
      buf ^= 1;
      put(buf, key, to - key);
      there = there_next;
      load(to - key - STAGE);
      __syncthreads();
    }
  }

  z += __shfl_xor(z, 32);
  // (whether any wave met one)
  if (__syncthreads_or(odd) && on) {
    const int upto = min(to - 1, last);
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int at = 32 * i + 8 * b + 4 * h;
        if (at >= c.d) continue;
        for (int key = max(0, first_last + 1); key <= upto; ++key) {
          const int pg = (int)((uint32_t)key / (uint32_t)c.block_rows), of = key - pg * c.block_rows, block = table[pg];
          if (block < 0 || block >= c.n_blocks) continue;
          const E* src = vx + block * c.block + (int64_t)of * c.row;
          const uint32_t sc = SCALED ? c.v.scales[((int64_t)block * H + head) * c.block_rows + of] : 0u;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float f = number(src, at + e, sc);
            if (f - f != 0.f) o[i][4 * b + e] += f;
          }
        }
      }
  }
  if (!on) return;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int at = 32 * i + 8 * b + 4 * h;
      if (at < c.d) put_out<uint16_t>(c, a, col, head, G, r, at, m, z, f32x4{o[i][4 * b], o[i][4 * b + 1], o[i][4 * b + 2], o[i][4 * b + 3]});
    }
}

// Columns of a KV head, at most.
int64_t columns_of(int G, int n, int64_t n_tokens) { return n_tokens * G / TILE + n; }

}  // namespace

// With more score rows of a request than the other kernel's tile and enough columns to keep the device busy.  This kernel : the one that shares keys out, us, 32
// heads on 8, requests of equal numbers of tokens, blocks of 64 rows.
// bf16: 32 requests of 1000 to 2000 rows, 10 tokens 54 : 78, 16 tokens 56 : 85, 32 tokens 62 : 141; 16 of 1000 to 4096, 64 tokens 103 : 212.  128 workgroups: 16 of 2048 rows, 20 tokens
// 54 : 81, four of 8192, 128 tokens 189 : 186, but two, 256 tokens 189 : 176 and one of 16384, 512 tokens 365 : 320 (many tiles of a request read its keys from the caches
// there); 160: two of 8192 189 : 213, one of 16384 367 : 391.  d = 64: 128 workgroups, 16 of 2048, 9 tokens 35 : 33 (blocks of 16 rows 47 : 32), eight of 4096, 64 tokens 65 : 84, so from 64
// score rows on (of calls of fewer with more workgroups some lose by it: 256, 9 tokens 30 : 38, 512 59 : 92).
// 8 bits, which every wave of this one converts again: 128 workgroups, 16 of 2048, 9 tokens 59 : 33, eight of 4096, 33 tokens 124 : 71; 192: one of 16384 469 : 391, two of 8192 240 : 217,
// four 240 : 238, eight of 4096 125 : 137; 224: one of 16384 469 : 452, two of 8192 240 : 256; 256: 238 : 283 and 16 of 2048 69 : 112.  d = 64: 192, two of 8192 142 : 111, eight of 4096
// 76 : 73; 256, two 143 : 139, eight 76 : 89.
// The host knows no lengths, so it is the average number of tokens that chooses, padding counted, and for all requests: where decoding requests come with a chunk, none of their
// keys is shared out.  63 of 1000 to 8192 rows beside 512 tokens over 4096 247 us (in two calls 191 + 87), but with one of 131072 rows among them 2556 (264 + 87); 16 of 1000 to
// 8192 rows in a batch padded to 256 tokens 165 (not padded 62).
bool paged_prompt_call(const PagedView& c, int Hq, int dtype, int n, int64_t n_tokens) {
  if (dtype != LAQ_BF16 || c.d > 128) return false;
  const int G = Hq / c.Hkv;
  const int64_t rows = (n_tokens + n - 1) / n * G, tiles = (rows + TILE - 1) / TILE, columns = tiles * n * c.Hkv;
  return rows >= (c.d <= 64 ? 64 : 33) && columns >= (c.type == LAQ_E4M3 ? 200 : tiles <= 4 ? 128 : 160) && columns_of(G, n, n_tokens) * c.Hkv < (1 << 24);
}

hipError_t launch_paged_prompt(const PagedView& c, const PagedAttention& a, hipStream_t st) {
  const dim3 grid((unsigned)(columns_of(a.Hq / c.Hkv, a.n, a.n_tokens) * c.Hkv));
  const auto start = [&](auto numbers, auto d, auto wide) {
    hipLaunchKernelGGL((paged_prompt_kernel<std::remove_pointer_t<decltype(numbers)>, d(), wide()>), grid, dim3(THREADS), 0, st, c, a);
  };
  const auto by_size = [&](auto numbers, auto wide) {
    if (c.d <= 64) start(numbers, std::integral_constant<int, 64>{}, wide);
    else start(numbers, std::integral_constant<int, 128>{}, wide);
  };
  const auto by_type = [&](auto wide) {
    if (c.type == LAQ_BF16) by_size((uint16_t*)nullptr, wide);
    else by_size((E4m3*)nullptr, wide);
  };
  if (c.block_rows % STAGE == 0) by_type(std::true_type{});
  else by_type(std::false_type{});
  return hipGetLastError();
}

}  // namespace laq
