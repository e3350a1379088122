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

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ long long wave_sums(long long x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const long long y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// The thread whose requests hold number x of a running sum.
template <int THREADS>
__device__ __forceinline__ int holder(const long long* before, long long x) {
  int lo = 0;
#pragma unroll
  for (int step = THREADS / 2; step > 0; step /= 2)
    if (before[lo + step] <= x) lo += step;
  return lo;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void block_map_kernel(MapArgs a) {
  constexpr int WAVES = THREADS / 64;
  __shared__ long long more_before[THREADS + 1], need_before[THREADS + 1], back_before[THREADS + 1];
  __shared__ long long wave_more[WAVES], wave_need[WAVES], wave_back[WAVES];
  __shared__ long long taken_of[WAVES];
  __shared__ int refused_of[WAVES], last;
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
  long long more = 0, need = 0, back = 0;
  for (int i = i0; i < i1; ++i) {
    const Request r = own(i);
    more += r.more;
    need += r.need;
    back += r.back;
  }
  const long long more_in = wave_sums(more, lane), need_in = wave_sums(need, lane), back_in = wave_sums(back, lane);
  if (lane == 63) {
    wave_more[wave] = more_in;
    wave_need[wave] = need_in;
    wave_back[wave] = back_in;
  }
  __syncthreads();
  long long more0 = 0, need0 = 0, back0 = 0, all_back = 0, all_more = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) {
      more0 += wave_more[w];
      need0 += wave_need[w];
      back0 += wave_back[w];
    }
    all_back += wave_back[w];
    all_more += wave_more[w];
  }
  more0 += more_in - more;               // of the threads before this one
  need0 += need_in - need;
  back0 += back_in - back;
  more_before[tid] = more0;
  need_before[tid] = need0;
  back_before[tid] = back0;

  const long long count = min(max(held, 0), a.n_blocks), there = count + all_back;
  // blocks taken: up to the last request that gets its own
  long long upto = need0, taken = 0;
  int refused = 0;
  for (int i = i0; i < i1; ++i) {
    const Request r = own(i);
    upto += r.need;
    if (r.need > 0 && upto <= there) taken = upto;
    if (r.wide || (r.need > 0 && upto > there)) ++refused;
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    taken = max(taken, __shfl_xor(taken, o));
    refused += __shfl_xor(refused, o);
  }
  if (lane == 0) {
    taken_of[wave] = taken;
    refused_of[wave] = refused;
  }
  __syncthreads();
  refused = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    taken = max(taken, taken_of[w]);
    refused += refused_of[w];
  }

  // the block that comes back as number r (the last request's last one is number 0)
  auto given_back = [&](long long r) {
    const long long x = all_back - 1 - r;
    const int t = holder<THREADS>(back_before, x);
    long long at = back_before[t];
    for (int i = t * a.per;; ++i) {
      const Request q = any(i);
      if (x < at + q.back) return a.table[(size_t)i * a.width + q.want + (x - at)];
      at += q.back;
    }
  };
  // the block that is taken as number k
  auto block = [&](long long k) {
    const long long p = there - 1 - k;
    return p < count ? a.list[p] : given_back(p - count);
  };

  const long long first = (long long)blockIdx.x * THREADS + tid, step = (long long)gridDim.x * THREADS;
  // four slots in a row each: they are mostly of one block
  for (long long s0 = first * 4; s0 < a.n_slots; s0 += step * 4) {
    int slot[4] = {-1, -1, -1, -1};
    if (s0 < all_more) {
      const int t = holder<THREADS>(more_before, s0);
      long long at = more_before[t], k = need_before[t];
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
  for (long long k = first; k < taken; k += step) {
    const int t = holder<THREADS>(need_before, k);
    long long at = need_before[t];
    for (int i = t * a.per;; ++i) {
      const Request r = any(i);
      if (k < at + r.need) {
        a.table[(size_t)i * a.width + r.have + (k - at)] = block(k);
        break;
      }
      at += r.need;
    }
  }
  for (long long r = first; r < all_back - taken && count + r < a.n_blocks; r += step) a.list[count + r] = given_back(r);
  if (a.start && blockIdx.x == 0) {
    long long at = more0;
    for (int i = i0; i < i1; ++i) {
      a.start[i] = (int)min(at, 0x7fffffffll);
      at += own(i).more;
    }
    if (tid == 0) a.start[a.n] = (int)min(all_more, 0x7fffffffll);
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

// A thread has four slots, or as many blocks of a batch that is admitted or released, up to a workgroup per compute unit.
constexpr int MAP_MOST_WORKGROUPS = 256;

}  // namespace

hipError_t launch_block_map(int n, int block_rows, int n_blocks, int width, const int32_t* add, int32_t* rows, int32_t* table, int32_t* list,
                            int32_t* state, int32_t* start, int32_t* slots, int64_t n_slots, hipStream_t st) {
  const int threads = n <= 1024 ? 256 : 1024;
  const int shift = (block_rows & (block_rows - 1)) == 0 ? __builtin_ctz(block_rows) : -1;
  const MapArgs a{n, block_rows, n_blocks, width, (n + threads - 1) / threads, shift, add, rows, table, list, state, start, slots, n_slots};
  const int64_t work = n_slots > n_blocks / 4 ? n_slots : n_blocks / 4, wanted = (work + 1023) / 1024;
  const dim3 grid((unsigned)(wanted < 1 ? 1 : wanted > MAP_MOST_WORKGROUPS ? MAP_MOST_WORKGROUPS : wanted));
  if (threads == 256) hipLaunchKernelGGL(block_map_kernel<256>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(block_map_kernel<1024>, grid, dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace laq
