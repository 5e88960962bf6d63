// Slots pushed onto, and taken from, the stack of free ones.
//
// Both calls lay the sessions' lists end to end: session b's part of the T entries in all starts
// at the sum of the parts before it. A workgroup scans the sessions' counts, TILE at a time, for
// T and again for the parts that its share of the entries lies in, and finds the session of an
// entry by bisection. Bound by a launch and by the chain of loads (sessions and counts, then the
// stack or list, then the stores): every workgroup repeats the scan rather than wait for one.
// What the calls change in place (count, n_all over n_live, n_taken over n_new) is written by
// the workgroup that arrives last, once all have read it: count[1] counts the arrivals.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ikv_internal.hpp"

namespace ikv {

constexpr int ST = 256;                    // threads per workgroup
constexpr int SLOT_TILE = ST;              // sessions scanned at a time, one a thread
constexpr int SLOT_SHARE = 1024;           // entries of a workgroup, at least

struct SlotsLds {
  int32_t wave[ST / WAVE];
  int32_t start[SLOT_TILE + 1];            // of the tile's sessions, within the tile
  int64_t off[SLOT_TILE];                  // where their parts lie in the per-position arrays
  int32_t qs[SLOT_TILE], nl[SLOT_TILE];
  int32_t last;
};

// Inclusive sums over the workgroup; *total of all. Counts sum to less than 2^31.
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

// Whether this workgroup is the last to arrive; all of its reads come before.
__device__ __forceinline__ bool last_to_arrive(int32_t *count, SlotsLds &s) {
  __syncthreads();
  if (threadIdx.x == 0)
    s.last = gridDim.x == 1 || __hip_atomic_fetch_add(&count[1], 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == int(gridDim.x) - 1;
  __syncthreads();
  return s.last != 0;
}

__device__ __forceinline__ void leave(int32_t *count, int32_t n_free) {
  __hip_atomic_store(&count[0], n_free, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(&count[1], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__global__ void __launch_bounds__(ST) k_return_slots(ikv_free_slots f, const ikv_session *__restrict__ sess, int B,
                                                     const int32_t *__restrict__ list,
                                                     const int32_t *__restrict__ n_list) {
  __shared__ SlotsLds s;
  const int tid = threadIdx.x;
  auto part = [&](int b) { return b < B ? max(0, min(n_list[b], sess[b].N)) : 0; };
  int T = 0, tile_sum;
  for (int b0 = 0; b0 < B; b0 += SLOT_TILE) {
    block_scan(part(b0 + tid), s, &tile_sum);
    T += tile_sum;
  }
  const int64_t n_free = max(0, int(min(int64_t(f.count[0]), f.num_slots)));
  const int from = int(int64_t(T) * blockIdx.x / gridDim.x), to = int(int64_t(T) * (blockIdx.x + 1) / gridDim.x);
  int before = 0;
  for (int b0 = 0; b0 < B && before < to; b0 += SLOT_TILE) {
    const int n = part(b0 + tid), end = block_scan(n, s, &tile_sum);
    s.start[tid] = end - n;
    s.off[tid] = b0 + tid < B ? sess[b0 + tid].slot_off : 0;
    __syncthreads();
    for (int i = max(from - before, 0) + tid; i < min(to - before, tile_sum); i += ST) {
      const int b = find_session(s.start, i);
      const int64_t at = n_free + before + i;
      if (at < f.num_slots) f.slots[at] = list[s.off[b] + (i - s.start[b])];
    }
    before += tile_sum;
    __syncthreads();
  }
  if (last_to_arrive(f.count, s) && tid == 0) leave(f.count, int32_t(min(n_free + T, f.num_slots)));
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
  // tokens that session b asks for, if its list has room; its live entries
  auto wanted = [&](int b, int *nl) {
    *nl = 0;
    if (b >= a.B) return 0;
    const ikv_session x = a.sess[b];
    const int n = a.n_new ? max(0, min(a.n_new[b], x.qe - x.qs)) : x.qe - x.qs;
    if (!a.live) return n;
    *nl = max(0, min(a.n_live[b], x.N));
    return n <= x.N - *nl ? n : 0;
  };
  int sum = 0, tile_sum, T = 0, nl;
  for (int b0 = 0; b0 < a.B; b0 += SLOT_TILE) {
    const int n = wanted(b0 + tid, &nl), end = sum + block_scan(n, s, &tile_sum);
    // the largest sum that the stack holds is what is served
    int served = end <= n_free ? end : 0;
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
    const int n = wanted(b0 + tid, &nl), end = block_scan(n, s, &tile_sum);
    s.start[tid] = end - n;
    s.off[tid] = b0 + tid < a.B ? a.sess[b0 + tid].slot_off : 0;
    s.qs[tid] = b0 + tid < a.B ? a.sess[b0 + tid].qs : 0;
    s.nl[tid] = nl;
    __syncthreads();
    for (int i = max(from - before, 0) + tid; i < min(to - before, tile_sum); i += ST) {
      const int b = find_session(s.start, i), t = i - s.start[b];
      const int32_t slot = top[before + i];
      const int64_t off = s.off[b] + t;
      if (a.slot_maps) a.slot_maps[off + s.qs[b]] = slot;
      if (a.live) a.live[off + s.nl[b]] = slot;
      if (a.dst) a.dst[off] = slot;
    }
    before += tile_sum;
    __syncthreads();
  }
  if (!last_to_arrive(a.f.count, s)) return;
  sum = 0;
  for (int b0 = 0; b0 < a.B; b0 += SLOT_TILE) {
    const int b = b0 + tid, n = wanted(b, &nl), end = sum + block_scan(n, s, &tile_sum), got = end <= T ? n : 0;
    if (b < a.B) {
      a.n_taken[b] = got;
      if (a.live) a.n_all[b] = nl + got;
    }
    sum += tile_sum;
  }
  if (tid == 0) leave(a.f.count, n_free - T);
}

static unsigned slots_grid(int64_t entries) {
  return unsigned(std::max<int64_t>(1, std::min<int64_t>(2 * 256, entries / SLOT_SHARE)));
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
