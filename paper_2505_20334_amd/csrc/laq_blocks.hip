// Block tables and slots of requests whose lengths change (include/laq_fp4.h: laq_block_map).
//
// Everything follows from three running sums over the requests: rows appended, blocks taken, blocks given back.  Every workgroup makes
// them for itself (8 bytes a request, from the caches), and all of them share the slots, the new table entries and the list's; no
// workgroup reads what another writes: a block that is given back and taken in the same call is read from the table of the request that
// gives it back (its entries stay), and the list is written only where more blocks come back than go, and then no block is taken from
// it.  The lengths and the list's size, which all workgroups read, are written by the one that finds the others done (state[2] counts them).
//
// What bounds it: a launch and four dependent trips to memory.
#include "laq_fp4_codes.h"

namespace laq {

namespace {

struct MapArgs {
  int32_t n, block_rows, n_blocks, width, per;         // per: requests of a thread
  int32_t shift;                                        // log2 of block_rows, or -1
  const int32_t* add;
  int32_t *rows, *table, *list, *state, *start, *slots;
  int64_t n_slots;
};

struct Request {
  int32_t old_rows, new_rows, have, want;
  int32_t more;                          // rows appended
  int32_t need, back;                    // blocks taken (if there are enough), given back
  bool wide;                             // more blocks than the table holds
};
__device__ __forceinline__ int blocks_of(const MapArgs& a, int rows) { return a.shift >= 0 ? rows >> a.shift : rows / a.block_rows; }
__device__ __forceinline__ Request request(const MapArgs& a, int rows, int add) {
  Request r;
  const int most = a.width * a.block_rows;
  r.old_rows = min(max(rows, 0), most);
  const long long now = max((long long)r.old_rows + add, 0ll);
  r.wide = now > most;
  r.new_rows = r.wide ? r.old_rows : (int)now;
  r.have = blocks_of(a, r.old_rows) + (r.old_rows != blocks_of(a, r.old_rows) * a.block_rows);
  r.want = blocks_of(a, r.new_rows) + (r.new_rows != blocks_of(a, r.new_rows) * a.block_rows);
  r.more = max(add, 0);
  r.need = max(r.want - r.have, 0);
  r.back = max(r.have - r.want, 0);
  return r;
}

// Sums that stay at the largest number.
__device__ __forceinline__ uint32_t add_most(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }
// Inclusive sum over the lanes of a wave: within 16 lanes by shifts of 1, 2, 4, 8, then from the last lane of 16 and of 32 to the lanes behind (by
// lane exchanges through the LDS three of these took 2 us).
__device__ __forceinline__ uint32_t wave_sums(uint32_t x) {
  x = add_most(x, __builtin_amdgcn_update_dpp(0u, x, 0x111, 0xf, 0xf, false));
  x = add_most(x, __builtin_amdgcn_update_dpp(0u, x, 0x112, 0xf, 0xf, false));
  x = add_most(x, __builtin_amdgcn_update_dpp(0u, x, 0x114, 0xf, 0xf, false));
  x = add_most(x, __builtin_amdgcn_update_dpp(0u, x, 0x118, 0xf, 0xf, false));
  x = add_most(x, __builtin_amdgcn_update_dpp(0u, x, 0x142, 0xa, 0xf, false));
  return add_most(x, __builtin_amdgcn_update_dpp(0u, x, 0x143, 0xc, 0xf, false));
}

// The thread whose requests hold number x of a running sum.
template <int THREADS>
__device__ __forceinline__ int holder(const uint32_t* before, uint32_t x) {
  int lo = 0;
#pragma unroll
  for (int step = THREADS / 2; step > 0; step /= 2)
    if (before[lo + step] <= x) lo += step;
  return lo;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void block_map_kernel(MapArgs a) {
  constexpr int WAVES = THREADS / 64;
  __shared__ uint32_t more_before[THREADS], need_before[THREADS], back_before[THREADS];
  __shared__ uint32_t wave_more[WAVES], wave_need[WAVES], wave_back[WAVES];
  __shared__ uint32_t taken_most;
  __shared__ int refused_all, last;
  __shared__ int2 given[THREADS];        // rows and add of all requests, where a thread has one
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int i0 = (int)min((long long)tid * a.per, (long long)a.n), i1 = (int)min((long long)i0 + a.per, (long long)a.n);

  const bool one = a.per == 1;
  const int held = a.state[0];
  int2 mine = {0, 0};
  if (i0 < i1) mine = int2{a.rows[i0], a.add[i0]};
  given[tid] = mine;
  // of this thread's requests; of any (after the first barrier)
  auto own = [&](int i) { return i == i0 ? request(a, mine.x, mine.y) : request(a, a.rows[i], a.add[i]); };
  auto any = [&](int i) {
    const int2 x = one ? given[i] : int2{a.rows[i], a.add[i]};
    return request(a, x.x, x.y);
  };
  // (blocks are entries of the table: their sums are ints; rows appended beyond 2^32 - 1 have no slots and no start of their own)
  uint32_t more = 0, need = 0, back = 0;
  for (int i = i0; i < i1; ++i) {
    const Request r = own(i);
    more = add_most(more, r.more);
    need += r.need;
    back += r.back;
  }
  uint32_t more0 = wave_sums(more), need0 = wave_sums(need), back0 = wave_sums(back);
  if (lane == 63) {
    wave_more[wave] = more0;
    wave_need[wave] = need0;
    wave_back[wave] = back0;
  }
  if (tid == 0) {
    taken_most = 0;
    refused_all = 0;
  }
  __syncthreads();
  // of the threads before this one
  more0 = __builtin_amdgcn_update_dpp(0u, more0, 0x138, 0xf, 0xf, false);     // (from the lane before: a sum that stays at its most has no difference)
  need0 -= need;
  back0 -= back;
  uint32_t all_back = 0, all_more = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) {
      more0 = add_most(more0, wave_more[w]);
      need0 += wave_need[w];
      back0 += wave_back[w];
    }
    all_back += wave_back[w];
    all_more = add_most(all_more, wave_more[w]);
  }
  more_before[tid] = more0;
  need_before[tid] = need0;
  back_before[tid] = back0;

  const uint32_t count = (uint32_t)min(max(held, 0), a.n_blocks);
  const long long there = (long long)count + all_back;
  // blocks taken: up to the last request that gets its own
  uint32_t upto = need0, taken = 0;
  int refused = 0;
  for (int i = i0; i < i1; ++i) {
    const Request r = own(i);
    upto += r.need;
    if (r.need > 0 && upto <= there) taken = upto;
    if (r.wide || (r.need > 0 && upto > there)) ++refused;
  }
  if (taken) atomicMax(&taken_most, taken);
  if (refused) atomicAdd(&refused_all, refused);
  __syncthreads();
  taken = taken_most;
  refused = refused_all;

  // the block that comes back as number r (the last request's last one is number 0)
  auto given_back = [&](uint32_t r) {
    const uint32_t x = all_back - 1 - r;
    const int t = holder<THREADS>(back_before, x);
    uint32_t at = back_before[t];
    for (int i = t * a.per;; ++i) {
      const Request q = any(i);
      if (x < at + q.back) return a.table[(size_t)i * a.width + q.want + (x - at)];
      at += q.back;
    }
  };
  // the block that is taken as number k
  auto block = [&](uint32_t k) {
    const long long p = there - 1 - k;
    return p < count ? a.list[p] : given_back((uint32_t)(p - count));
  };

  const long long first = (long long)blockIdx.x * THREADS + tid, step = (long long)gridDim.x * THREADS;
  // four slots in a row each: they are mostly of one block
  for (long long s0 = first * 4; s0 < a.n_slots; s0 += step * 4) {
    int slot[4] = {-1, -1, -1, -1};
    if (s0 < all_more) {
      const int t = holder<THREADS>(more_before, (uint32_t)s0);
      long long at = more_before[t];
      uint32_t k = need_before[t];
      int i = t * a.per, known = -1, number = -1;
      Request r = any(i);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const long long s = s0 + x;
        if (s >= all_more) break;
        while (s >= at + r.more) {
          at += r.more;
          k += r.need;
          r = any(++i);
          known = -1;
        }
        if (r.wide || (r.need > 0 && k + r.need > there)) continue;
        const int row = r.old_rows + (int)(s - at), b = blocks_of(a, row);
        if (b != known) {
          known = b;
          number = b < r.have ? a.table[(size_t)i * a.width + b] : block(k + (b - r.have));
        }
        if (number >= 0 && number < a.n_blocks) slot[x] = number * a.block_rows + (row - b * a.block_rows);
      }
    }
    if (s0 + 4 <= a.n_slots && (reinterpret_cast<uintptr_t>(a.slots) & 15) == 0) {
      *reinterpret_cast<int4*>(a.slots + s0) = int4{slot[0], slot[1], slot[2], slot[3]};
    } else {
      for (int x = 0; x < 4 && s0 + x < a.n_slots; ++x) a.slots[s0 + x] = slot[x];
    }
  }
  for (long long x = first; x < taken; x += step) {
    const uint32_t k = (uint32_t)x;
    const int t = holder<THREADS>(need_before, k);
    uint32_t at = need_before[t];
    for (int i = t * a.per;; ++i) {
      const Request r = any(i);
      if (k < at + r.need) {
        a.table[(size_t)i * a.width + r.have + (k - at)] = block(k);
        break;
      }
      at += r.need;
    }
  }
  for (long long r = first; r < (long long)all_back - taken && count + r < a.n_blocks; r += step) a.list[count + r] = given_back((uint32_t)r);
  if (a.start && blockIdx.x == 0) {
    uint32_t at = more0;
    for (int i = i0; i < i1; ++i) {
      a.start[i] = (int)min(at, 0x7fffffffu);
      at = add_most(at, own(i).more);
    }
    if (tid == 0) a.start[a.n] = (int)min(all_more, 0x7fffffffu);
  }

  if (gridDim.x > 1) {
    __syncthreads();                     // (what this workgroup reads has been read)
    if (tid == 0) last = __hip_atomic_fetch_add(&a.state[2], 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (gridDim.x > 1 && !last) return;
  upto = need0;
  for (int i = i0; i < i1; ++i) {
    const Request r = own(i);
    upto += r.need;
    if (!r.wide && (r.need == 0 || upto <= there)) a.rows[i] = r.new_rows;
  }
  if (tid == 0) {
    a.state[0] = (int)min(there - taken, (long long)a.n_blocks);
    a.state[1] = refused;
    a.state[2] = 0;
  }
}

// Workgroups of 1024 threads with four slots each, or, in small calls, of 256 with two times four; where there are no slots (rows are dropped) and
// the pool has more than 4096 blocks, two blocks a thread.  They cost a count in memory at the end, 0.7 us for two of them, 1.5 for 128.
// 294000 slots of 256 requests, 9200 blocks, appended and dropped: two times four a thread 18.2 us, four 16.5, two 16.5, workgroups of 256 19.2;
// 160000 of 1000 requests 22.2, 18.8, 18.7.  19000 slots of 64 requests in five workgroups of 1024 14.2, in ten of 256 15.4.
constexpr int MAP_MOST_WORKGROUPS = 128;

}  // namespace

hipError_t launch_block_map(int n, int block_rows, int n_blocks, int width, const int32_t* add, int32_t* rows, int32_t* table, int32_t* list,
                            int32_t* state, int32_t* start, int32_t* slots, int64_t n_slots, hipStream_t st) {
  const int64_t work = n_slots ? n_slots / 4 : n_blocks > 4096 ? n_blocks : 1, wanted = (work + 511) / 512;
  const int threads = n <= 256 && wanted < 4 ? 256 : 1024;
  const int shift = (block_rows & (block_rows - 1)) == 0 ? __builtin_ctz(block_rows) : -1;
  const MapArgs a{n, block_rows, n_blocks, width, (int)(((int64_t)n + threads - 1) / threads), shift, add, rows, table, list, state, start, slots, n_slots};
  const int64_t groups = threads == 256 ? wanted : (wanted + 1) / 2;
  const dim3 grid((unsigned)(groups < 1 ? 1 : groups > MAP_MOST_WORKGROUPS ? MAP_MOST_WORKGROUPS : groups));
  if (threads == 256) hipLaunchKernelGGL(block_map_kernel<256>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(block_map_kernel<1024>, grid, dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace laq
