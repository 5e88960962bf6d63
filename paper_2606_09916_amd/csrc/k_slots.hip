// Slots pushed onto, and taken from, the stack of free ones.
//
// Both calls lay the sessions' lists end to end: session b's part of the T entries in all starts
// at the sum of the parts before it. A workgroup scans the sessions' counts, a tile at a time, for
// T and (with more than one tile) again for the parts that its share of the entries lies in, and
// finds the session of an entry by bisection: no workgroup waits for another one's sums.
// What the calls change in place (count, n_all over n_live, n_taken over n_new) is written by the
// workgroup that arrives last, once all have read it: count[1] counts the arrivals.
// Bound by a launch and the chain of loads (counts, then the stack or list, then the stores): 64
// sessions' tokens take 2 us each call beside the launch; 2.1 million slots of 64 histories, 51 MB,
// 24 us for both calls (floor 11). There the arrivals count, 10 ns each: 256 workgroups of 512
// threads 24.2, 512 of 256 30.2, 1024 of 256 40.1; with one entry of a thread on its way at a time
// instead of eight, 54.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ikv_internal.hpp"

namespace ikv {

constexpr int ST = 512;                    // threads per workgroup
constexpr int SLOT_TILE = ST;              // sessions scanned at a time, one a thread
constexpr int SLOT_SHARE = 1024;           // entries of a workgroup, at least
constexpr int SLOT_UNROLL = 8;             // entries of a thread on their way at once
constexpr int SLOT_GRID = 256;             // workgroups, at most

struct SlotsLds {
  int32_t wave[ST / WAVE];
  int32_t start[SLOT_TILE + 1];            // of the tile's sessions, within the tile
  int64_t off[SLOT_TILE];                  // where their parts lie in the per-position arrays
  int32_t qs[SLOT_TILE], nl[SLOT_TILE];
  int32_t last;
};

// Inclusive sums over the workgroup; *total of all. Counts sum to at most SLOTS_MOST: entry numbers stay in
// 32 bits, a round of the workgroup's threads past the last one too.
__device__ __forceinline__ int block_scan(int x, SlotsLds &s, int *total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < WAVE; o <<= 1) {
    const int y = __shfl_up(x, o, WAVE);
    if (lane >= o) x += y;
  }
  __syncthreads();                         // the sums of the scan before have been read
  if (lane == WAVE - 1) s.wave[w] = x;
  __syncthreads();
  int sum = 0;
#pragma unroll
  for (int i = 0; i < ST / WAVE; ++i) {
    if (i == w) x += sum;
    sum += s.wave[i];
  }
  *total = sum;
  return x;
}

// The session whose part holds entry i of the tile: the last that starts at or before it.
__device__ __forceinline__ int find_session(const int32_t *start, int i) {
  int lo = 0;
#pragma unroll
  for (int step = SLOT_TILE / 2; step > 0; step >>= 1)
    if (start[lo + step] <= i) lo += step;
  return lo;
}

// Entries [from, to) of the lists laid end to end, of which the tile's sessions (s.start, s.off) hold
// `count` from `before` on: read(session, place in its part, entry) of SLOT_UNROLL entries a thread, then
// write(.., value) of each. A thread's entries lie ST apart, mostly in one session.
template <typename Read, typename Write>
__device__ __forceinline__ void slots_move(const SlotsLds &s, int before, int count, int from, int to, Read read, Write write) {
  const int lo = max(from - before, 0), hi = min(to - before, count);
  for (int i0 = lo + int(threadIdx.x); i0 < hi; i0 += ST * SLOT_UNROLL) {
    int b[SLOT_UNROLL], value[SLOT_UNROLL];
#pragma unroll
    for (int u = 0; u < SLOT_UNROLL; ++u) {
      const int i = min(i0 + u * ST, hi - 1);
      b[u] = u > 0 ? b[u - 1] : 0;
      if (u == 0 || s.start[b[u] + 1] <= i) b[u] = find_session(s.start, i);
      value[u] = read(b[u], i - s.start[b[u]], before + i);
    }
#pragma unroll
    for (int u = 0; u < SLOT_UNROLL; ++u) {
      const int i = i0 + u * ST;
      if (i < hi) write(b[u], i - s.start[b[u]], before + i, value[u]);
    }
  }
}

// Whether this workgroup is the last of `all` to arrive. All of its reads are done by then (their values
// have been used), which is all that the last one's writes have to wait for: the order needs no fence,
// and a release here would write each XCD's L2 back once per workgroup.
__device__ __forceinline__ bool last_to_arrive(int32_t *count, int all, SlotsLds &s) {
  __syncthreads();
  if (threadIdx.x == 0)
    s.last = all == 1 || __hip_atomic_fetch_add(&count[1], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == all - 1;
  __syncthreads();
  return s.last != 0;
}

__device__ __forceinline__ void leave(int32_t *count, int32_t n_free) {
  __hip_atomic_store(&count[0], n_free, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(&count[1], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The grid is sized for lists of N entries each; workgroups that the counts leave without a share
// end at once. (The counts are not changed by the call, so all workgroups agree on that.)
__global__ void __launch_bounds__(ST) k_return_slots(ikv_free_slots f, const ikv_session *__restrict__ sess, int B,
                                                     const int32_t *__restrict__ list,
                                                     const int32_t *__restrict__ n_list) {
  __shared__ SlotsLds s;
  const int tid = threadIdx.x;
  const int64_t n_free = max(0, int(min(int64_t(f.count[0]), f.num_slots)));
  const bool one = B <= SLOT_TILE;               // one tile: scanned once
  int n, end = 0, T = 0, tile_sum;
  auto scan = [&](int b0) __attribute__((always_inline)) {
    const int b = b0 + tid;
    n = b < B ? max(0, min(n_list[b], sess[b].N)) : 0;
    end = block_scan(n, s, &tile_sum);
  };
  for (int b0 = 0; b0 < B; b0 += SLOT_TILE) {
    scan(b0);
    T += tile_sum;
  }
  const int all = min(int(gridDim.x), max(1, (T + SLOT_SHARE - 1) / SLOT_SHARE));
  if (int(blockIdx.x) >= all) return;
  const int from = int(int64_t(T) * blockIdx.x / all), to = int(int64_t(T) * (blockIdx.x + 1) / all);
  int before = 0;
  for (int b0 = 0; b0 < B && before < to; b0 += SLOT_TILE) {
    if (!one) scan(b0);
    s.start[tid] = end - n;
    s.off[tid] = b0 + tid < B ? sess[b0 + tid].slot_off : 0;
    if (tid == 0) s.start[SLOT_TILE] = tile_sum;
    __syncthreads();
    slots_move(s, before, tile_sum, from, to, [&](int b, int k, int) { return list[s.off[b] + k]; },
               [&](int, int, int i, int slot) {
                 if (n_free + i < f.num_slots) f.slots[n_free + i] = slot;
               });
    before += tile_sum;
    __syncthreads();
  }
  if (last_to_arrive(f.count, all, s) && tid == 0) leave(f.count, int32_t(min(n_free + T, f.num_slots)));
}

struct TakeArgs {
  ikv_free_slots f;
  const ikv_session *sess;
  int B;
  const int32_t *n_new;                    // may be n_taken
  int32_t *slot_maps, *live;
  const int32_t *n_live;                   // may be n_all
  int32_t *n_all, *dst, *n_taken;
};

__global__ void __launch_bounds__(ST) k_take_slots(TakeArgs a) {
  __shared__ SlotsLds s;
  const int tid = threadIdx.x;
  const int n_free = max(0, int(min(int64_t(a.f.count[0]), a.f.num_slots)));
  const bool one = a.B <= SLOT_TILE;
  int n, nl, end = 0, tile_sum;
  // n: tokens that a session asks for, if its list has room; nl: its live entries
  auto scan = [&](int b0) __attribute__((always_inline)) {
    const int b = b0 + tid;
    n = nl = 0;
    if (b < a.B) {
      const ikv_session x = a.sess[b];
      n = a.n_new ? max(0, min(a.n_new[b], x.qe - x.qs)) : x.qe - x.qs;
      if (a.live) {
        nl = max(0, min(a.n_live[b], x.N));
        if (n > x.N - nl) n = 0;
      }
    }
    end = block_scan(n, s, &tile_sum);
  };
  int sum = 0, T = 0;
  for (int b0 = 0; b0 < a.B; b0 += SLOT_TILE) {
    scan(b0);
    // the largest sum that the stack holds is what is served
    int served = sum + end <= n_free ? sum + end : 0;
#pragma unroll
    for (int o = 1; o < WAVE; o <<= 1) served = max(served, __shfl_xor(served, o, WAVE));
    __syncthreads();
    if ((tid & 63) == 0) s.wave[tid >> 6] = served;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ST / WAVE; ++i) T = max(T, s.wave[i]);
    sum += tile_sum;
    if (sum > n_free) break;
  }
  const int32_t *top = a.f.slots + (n_free - T);
  const int from = int(int64_t(T) * blockIdx.x / gridDim.x), to = int(int64_t(T) * (blockIdx.x + 1) / gridDim.x);
  int before = 0;
  for (int b0 = 0; b0 < a.B && before < to; b0 += SLOT_TILE) {
    if (!one) scan(b0);
    s.start[tid] = end - n;
    s.off[tid] = b0 + tid < a.B ? a.sess[b0 + tid].slot_off : 0;
    s.qs[tid] = b0 + tid < a.B ? a.sess[b0 + tid].qs : 0;
    s.nl[tid] = nl;
    if (tid == 0) s.start[SLOT_TILE] = tile_sum;
    __syncthreads();
    slots_move(s, before, tile_sum, from, to, [&](int, int, int i) { return top[i]; },
               [&](int b, int t, int, int slot) {
                 const int64_t at = s.off[b] + t;
                 if (a.slot_maps) a.slot_maps[at + s.qs[b]] = slot;
                 if (a.live) a.live[at + s.nl[b]] = slot;
                 if (a.dst) a.dst[at] = slot;
               });
    before += tile_sum;
    __syncthreads();
  }
  if (!last_to_arrive(a.f.count, gridDim.x, s)) return;
  sum = 0;
  for (int b0 = 0; b0 < a.B; b0 += SLOT_TILE) {
    if (!one) scan(b0);
    const int b = b0 + tid, got = sum + end <= T ? n : 0;
    if (b < a.B) {
      a.n_taken[b] = got;
      if (a.live) a.n_all[b] = nl + got;
    }
    sum += tile_sum;
  }
  if (tid == 0) leave(a.f.count, n_free - T);
}

static unsigned slots_grid(int64_t entries) {
  return unsigned(std::max<int64_t>(1, std::min<int64_t>(SLOT_GRID, entries / SLOT_SHARE)));
}

hipError_t launch_return_slots(const ikv_free_slots &f, const ikv_session *sess_dev, int B, int64_t entries,
                               const int32_t *list, const int32_t *n_list, hipStream_t st) {
  KTimer kt_("k_return_slots", st);
  k_return_slots<<<slots_grid(entries), ST, 0, st>>>(f, sess_dev, B, list, n_list);
  return hipGetLastError();
}

hipError_t launch_take_slots(const ikv_free_slots &f, const ikv_session *sess_dev, int B, int64_t tokens,
                             const int32_t *n_new, int32_t *slot_maps, int32_t *live, const int32_t *n_live,
                             int32_t *n_all, int32_t *dst, int32_t *n_taken, hipStream_t st) {
  KTimer kt_("k_take_slots", st);
  k_take_slots<<<slots_grid(tokens), ST, 0, st>>>(TakeArgs{f, sess_dev, B, n_new, slot_maps, live, n_live, n_all, dst, n_taken});
  return hipGetLastError();
}

}  // namespace ikv
