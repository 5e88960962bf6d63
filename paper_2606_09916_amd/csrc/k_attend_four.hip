// Attention of few query rows over the 4-bit cache, D = 128, bf16 queries and outputs: as
// k_attend_few.hip (waves own KV heads and a share of the list, 16-row blocks of queries, blocks of 32
// entries), with operands fed in the way that suits rows of half a cache line.
//
// A lane loads 32 adjacent codes of a key row and of a value row, a block that one scale covers:
//   S^T = K Q^T   codes become bf16 with their scale, exactly, and are the first product's operand as
//                 they are
//   O^T += V^T P^T  value rows become bf16 in the same way and go through the wave's own part of LDS,
//                 back by the transposing loads (4 entries x 16 channels by 16 lanes).
// Bound by reading the rows once, 136 bytes per entry and head: 48 layers x 8 heads x 92,300 entries in
// 823 us (5.9 TB/s; the same loads alone take 815). What it took:
//   - rows of 64 bytes share a line with the next head's. A wave takes both heads (NH = 2): waves of
//     one head each drift apart and fetch the lines again, 16% more (1030 us; with a barrier in each
//     round of the loop 950). Loads past the caches fetch them twice (1134; load-only 953 against 821).
//   - a lane that loads its channels of 8 value rows, and pairs them by byte permutes, takes 246 vector
//     instructions per 32 entries of a head where this takes 171.
//   - up to 8 rows (a decode always) fill half a block: the weights' second bf16 parts take the other
//     half, and one product does for two (ROWS = 8; 878 -> 853 us in the shape of that time).
// The scaled products of 4-bit with 8-bit operands (K = 128), which would take the codes unchanged, sum
// with an error of 2^-13 to 2^-14 of the sum of magnitudes: too much for logits.
#include <math.h>

#include "attend.hpp"
#include "ikv_internal.hpp"
#include "kv_codes.hpp"

namespace ikv {

constexpr float FOUR_SLACK = 8.f;                // log2: as in k_attend_few.hip
constexpr int FOUR_BLOCK = 32;                   // entries per block
constexpr int FOUR_ROW = 136;                    // bf16 of a value row in LDS
// The place of an entry's value row among 16. Rows lie 17 pieces of 16 bytes apart: the same piece of
// 16 rows, as it is written, lies in 16 different ones of the LDS's 256 bytes of banks, and two adjacent
// pieces of entries 0 .. 7 or 8 .. 15, as half a wave reads them, do not overlap there.
__device__ __forceinline__ int four_place(int e) { return 2 * (e & 7) + (e >> 3); }

template <int NH, int ROWS, int NW, bool O32>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2)))
k_attend_four(AttendArgs a, int heads, int rows_max) {
  constexpr int D = 128, RB = D / 2, KS = D / 32, NT = D / 16;
  constexpr bool HALF = ROWS == 8;               // rows fill half a 16-row block: their weights' second parts take the other
  constexpr int NR = HALF ? 1 : ROWS / 16, PP = HALF ? 1 : 2;          // 16-row blocks; products of one with the weights' parts
  constexpr int NB = 2;                          // blocks of entries in registers
  constexpr int STATE = (4 * NT + 2) * WAVE;     // floats of a 16-row block's state
  constexpr int VALUES = FOUR_BLOCK * FOUR_ROW * 2;                      // bytes
  constexpr int STATES = (NW - 1) * NH * NR * STATE * 4, LDS = NW * NH * VALUES > STATES ? NW * NH * VALUES : STATES;
  __shared__ __align__(16) char lds[LDS];        // values, a part per wave; then the states of a head's other waves

  const int b = blockIdx.z;
  const ikv_session s = a.sess[b];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ngrp = a.Hkv / (NH * heads), parts_wg = NW / heads, part_wg = w / heads;
  const int l = blockIdx.y / ngrp, hkv = ((blockIdx.y - l * ngrp) * heads + w % heads) * NH;
  const int split = blockIdx.x, nsplit = gridDim.x;
  const int g = lane >> 4, c = lane & 15;
  const int G = a.Hq / a.Hkv;
  const int n = a.decode ? 1 : s.qe - s.qs, rows = n * G;
  if (rows <= 0) return;                         // the merge skips the session too
  int64_t before = 0;
  if (a.decode) before = b;
  else
    for (int i = 0; i < b; ++i) before += a.sess[i].qe - a.sess[i].qs;
  // row r = 16 k + c of this lane: token r / G, head r % G of the group; rows past the last repeat
  // it and are not written
  const int N = max(0, min(a.n_live[b], s.N));
  int own[NR];                                   // list entry of the row's token
  int64_t q_at[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    const int r = min(16 * k + (HALF ? c & 7 : c), rows - 1), t = r / G, h = r - t * G;
    own[k] = N - n + t;
    q_at[k] = before * a.L * a.Hq * D + ((int64_t(l) * a.Hq + hkv * G + h) * n + t) * D;
  }
  const int64_t next_head = int64_t(G) * n * D;  // from a KV head's queries to the next one's

  // entries seen by any token: up to the sinks, then [lo, N)
  const int lo = a.window ? max(0, N - n - a.window + 1) : 0;
  const int first = min(a.sinks, lo), gap = lo - first;        // index v stands for entry v, or v + gap from `first` on
  const int T = N - gap;
  const int pieces = nsplit * parts_wg, chunk = ((T + pieces - 1) / pieces + 15) & ~15;
  const int v0 = min(T, (split * parts_wg + part_wg) * chunk), v1 = min(T, v0 + chunk);

  float m[NH][NR], lsum[NH][NR];                 // reference of row 16 k + c; this lane's sum of its weights
  f32x4_k o[NH][NR][NT];                         // [..][t][i]: channel 16 t + 4 g + i of that row
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      m[h][k] = -INFINITY;
      lsum[h][k] = 0.f;
#pragma unroll
      for (int t = 0; t < NT; ++t) o[h][k][t] = f32x4_k{0.f, 0.f, 0.f, 0.f};
    }

  if (v0 < v1) {
    // queries as the B operand: step ks has channels 32 g + 8 ks .. of lane group g
    bf16x8_k qf[NH][NR][KS];
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int k = 0; k < NR; ++k)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          qf[h][k][ks] = *reinterpret_cast<const bf16x8_k *>(static_cast<const uint16_t *>(a.q) + q_at[k] + h * next_head +
                                                             32 * g + 8 * ks);
    const uint32_t row_bytes = uint32_t(a.Hkv) * RB;
    const int64_t layer = int64_t(l) * a.num_slots;
    // wave-uniform bases; a row is a per-lane byte offset, of 32 bits by a 24-bit product where
    // slots, rows and layers are small enough
    const char *kbase = static_cast<const char *>(a.k) + (layer * a.Hkv + hkv) * RB;
    const char *vbase = static_cast<const char *>(a.v) + (layer * a.Hkv + hkv) * RB;
    const char *sbase = reinterpret_cast<const char *>(a.scales) + (layer * a.Hkv + hkv) * (D / 16);
    auto row_at = [&](int sl) __attribute__((always_inline)) {
      if constexpr (O32) return uint32_t(__umul24(uint32_t(sl), row_bytes));
      else return uint64_t(uint32_t(sl)) * row_bytes;
    };
    const int32_t *list = a.live + s.slot_off;
    const float to_log2 = 1.4426950408889634f / sqrtf(float(D));
    uint16_t *vl = reinterpret_cast<uint16_t *>(lds + w * (NH * VALUES));
    uint16_t *vput = vl + four_place(c) * FOUR_ROW + 32 * g;
    const uint16_t *vget = vl + four_place(4 * g + (c >> 2)) * FOUR_ROW + 4 * (c & 3);

    struct Block {
      uint4 k[2][NH], v[2][NH];                    // of entry 16 kb + c, channels 32 g ..
      uint2 s[2][NH];                              // scale bytes of that entry's key and value
    };
    struct Slots { int s[2]; };
    auto slots = [&](int base) __attribute__((always_inline)) {
      Slots x;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int v = min(base + 16 * kb + c, v1 - 1);         // the last one again past the end
        x.s[kb] = list[v < first ? v : v + gap];
      }
      return x;
    };
    auto load = [&](Block &x, const Slots &sl) __attribute__((always_inline)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const auto at = row_at(sl.s[kb]);
#pragma unroll
        for (int h = 0; h < NH; ++h) x.s[kb][h] = *reinterpret_cast<const uint2 *>(sbase + (at / 8 + 8 * h));
#pragma unroll
        for (int h = 0; h < NH; ++h) x.k[kb][h] = *reinterpret_cast<const uint4 *>(kbase + (at + 16 * g + RB * h));
#pragma unroll
        for (int h = 0; h < NH; ++h) x.v[kb][h] = *reinterpret_cast<const uint4 *>(vbase + (at + 16 * g + RB * h));
      }
    };
    bool odd = false;                              // a value that is not finite was left out
    auto compute = [&](Block &x, int base) __attribute__((always_inline)) {
      // a block that every token sees whole needs no mask: its last entry is at or before the
      // oldest token's own, and its first inside the newest's window or all of it among the sinks
      const int last = base + FOUR_BLOCK - 1, oldest = N - n;
      const int jl = last < first ? last : last + gap, j0 = base < first ? base : base + gap;
      const bool whole = last < v1 && jl <= oldest && (a.window == 0 || jl < a.sinks || j0 > N - 1 - a.window);
      f32x4_k acc[NH][NR][2];
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int k = 0; k < NR; ++k) acc[h][k][0] = acc[h][k][1] = f32x4_k{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            const float scale = __uint_as_float((x.s[kb][h].x >> (8 * g) & 255u) << 23);
            const bf16x8_k kf = __builtin_bit_cast(bf16x8_k, e2m1_scaled8((&x.k[kb][h].x)[ks], scale));
#pragma unroll
            for (int k = 0; k < NR; ++k)
              acc[h][k][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[h][k][ks], acc[h][k][kb], 0, 0, 0);
          }
      uint32_t vb[NH][2], top = 0;
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          vb[h][kb] = x.s[kb][h].y >> (8 * g) & 255u;
          top = max(top, vb[h][kb]);
        }
      // values that are not finite are added after the loop to the rows that see them: in a block that some
      // row does not see, and everywhere the infinite ones, whose products with the weights' second parts
      // (zero, or of the other sign) would be NaN
      if (__builtin_amdgcn_ballot_w64(top >= 253u) != 0) {
        bool out = !whole;
#pragma unroll
        for (int h = 0; h < NH; ++h) out |= (vb[h][0] - 253u < 2u) | (vb[h][1] - 253u < 2u);
        if (__builtin_amdgcn_ballot_w64(out) != 0) {
#pragma unroll
          for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t z = e2m1_odd((&x.v[kb][h].x)[i], vb[h][kb]);
                odd |= z != 0;
                (&x.v[kb][h].x)[i] &= ~z;
              }
              if (vb[h][kb] == 255u) vb[h][kb] = 127u;
            }
        }
      }
      if (!whole) {
#pragma unroll
        for (int k = 0; k < NR; ++k)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int v = base + 16 * kb + 4 * g + i, j = v < first ? v : v + gap;
              const bool see = (v < v1) & (j <= own[k]) & ((a.window == 0) | (j < a.sinks) | (j > own[k] - a.window));
#pragma unroll
              for (int h = 0; h < NH; ++h) acc[h][k][kb][i] = see ? acc[h][k][kb][i] : -INFINITY;
            }
      }
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4 *>(vput + h * (VALUES / 2) + 16 * kb * FOUR_ROW + 8 * i) =
                e2m1_scaled8((&x.v[kb][h].x)[i], __uint_as_float(vb[h][kb] << 23));
      float tmax[NH][NR];
      bool moves = false;
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int k = 0; k < NR; ++k) {
          tmax[h][k] = -INFINITY;
#pragma unroll
          for (int e = 0; e < 8; ++e) tmax[h][k] = fmaxf(tmax[h][k], acc[h][k][e >> 2][e & 3]);
          tmax[h][k] *= to_log2;
          moves |= !(tmax[h][k] - m[h][k] <= FOUR_SLACK);
        }
      if (__builtin_amdgcn_ballot_w64(moves) != 0) {
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int k = 0; k < NR; ++k) {
            float z = tmax[h][k];
            z = fmaxf(z, __shfl_xor(z, 16, WAVE));
            z = fmaxf(z, __shfl_xor(z, 32, WAVE));
            const float mn = !(z - m[h][k] <= FOUR_SLACK) ? fmaxf(m[h][k], z) : m[h][k];     // by this row alone
            const float corr = m[h][k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[h][k] - mn);
            m[h][k] = mn;
            lsum[h][k] *= corr;
#pragma unroll
            for (int t = 0; t < NT; ++t) o[h][k][t] *= corr;
          }
      }
      bf16x8_k pf[NH][NR][PP];
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int k = 0; k < NR; ++k) {
          const float ms = m[h][k] == -INFINITY ? 0.f : m[h][k];       // no logit above -inf yet: the weights are 2^-inf
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float p = __builtin_amdgcn_exp2f(fmaf(acc[h][k][e >> 2][e & 3], to_log2, -ms));
            lsum[h][k] += p;
            const __bf16 near = __bf16(p);
            if constexpr (HALF) pf[h][k][0][e] = __bf16(c < 8 ? p : p - float(near));
            else {
              pf[h][k][0][e] = near;
              pf[h][k][1][e] = __bf16(p - float(near));
            }
          }
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint16_t *from = vget + h * (VALUES / 2) + 16 * t;
          const uint2 x0 = read_tr16(from), x1 = read_tr16(from + 16 * FOUR_ROW);
          const bf16x8_k vf = __builtin_bit_cast(bf16x8_k, make_uint4(x0.x, x0.y, x1.x, x1.y));
#pragma unroll
          for (int p = PP - 1; p >= 0; --p)
#pragma unroll
            for (int k = 0; k < NR; ++k)
              o[h][k][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[h][k][p], o[h][k][t], 0, 0, 0);
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    };
    // NB blocks in registers: one computed, the others on their way
    Block x[NB];
    Slots sl[NB];
#pragma unroll
    for (int u = 0; u < NB - 1; ++u) sl[u] = slots(v0 + u * FOUR_BLOCK);
    Slots next = slots(v0 + (NB - 1) * FOUR_BLOCK);
#pragma unroll
    for (int u = 0; u < NB - 1; ++u) load(x[u], sl[u]);
    for (int base = v0; base < v1; base += NB * FOUR_BLOCK) {
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        const int at = base + u * FOUR_BLOCK;
        if (u > 0 && at >= v1) break;
        __builtin_amdgcn_sched_barrier(0);
        sl[(u + NB - 1) % NB] = next;
        next = slots(at + NB * FOUR_BLOCK);
        load(x[(u + NB - 1) % NB], sl[(u + NB - 1) % NB]);
        __builtin_amdgcn_sched_barrier(0);
        compute(x[u], at);
      }
    }
    if (__builtin_amdgcn_ballot_w64(odd) != 0)
      for (int v = v0; v < v1; ++v) {
        const int e = v < first ? v : v + gap;
        const auto at = row_at(list[e]);
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          const uint8_t *sb = reinterpret_cast<const uint8_t *>(sbase + (at / 8 + 8 * h)) + D / 32;
#pragma unroll
          for (int k = 0; k < NR; ++k) {
            const bool see = (e <= own[k]) & ((a.window == 0) | (e < a.sinks) | (e > own[k] - a.window));
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              const uint32_t four = *reinterpret_cast<const uint16_t *>(vbase + (at + RB * h + 8 * t + 2 * g)), byte = sb[t / 2];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t code = four >> (4 * i) & 15u;
                if (see && e2m1_odd(code, byte) != 0)
                  o[h][k][t][i] += byte == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(0x7f800000u | code >> 3 << 31);
              }
            }
          }
        }
      }
  }
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      lsum[h][k] += __shfl_xor(lsum[h][k], 16, WAVE);
      lsum[h][k] += __shfl_xor(lsum[h][k], 32, WAVE);
      if constexpr (HALF) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[h][k][t][i] += __shfl_xor(o[h][k][t][i], 8, WAVE);
      }
    }
  if (parts_wg > 1) {
    // the other waves of a head leave their state in LDS, lane for lane; the first joins them
    float *joint = reinterpret_cast<float *>(lds);
    __syncthreads();                             // every wave is done with its values
    if (part_wg > 0) {
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int k = 0; k < NR; ++k) {
          float *mine = joint + (((w - heads) * NH + h) * NR + k) * STATE + lane;
          mine[0] = m[h][k];
          mine[WAVE] = lsum[h][k];
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(2 + 4 * t + i) * WAVE] = o[h][k][t][i];
        }
    }
    __syncthreads();
    if (part_wg > 0) return;
    for (int p = 1; p < parts_wg; ++p) {
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int k = 0; k < NR; ++k) {
          const float *x = joint + (((w + (p - 1) * heads) * NH + h) * NR + k) * STATE + lane;
          const float mp = x[0], mn = fmaxf(m[h][k], mp);
          const float f = m[h][k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[h][k] - mn);
          const float fp = mp == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mp - mn);
          m[h][k] = mn;
          lsum[h][k] = lsum[h][k] * f + x[WAVE] * fp;
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[h][k][t][i] = o[h][k][t][i] * f + x[(2 + 4 * t + i) * WAVE] * fp;
        }
    }
  }
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    const int r = 16 * k + c;
    if (r >= rows) continue;                     // (of HALF, rows are at most 8)
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      if (nsplit == 1) {
        const float inv = own[k] < 0 ? 0.f : 1.0f / lsum[h][k];        // nothing seen: zero
        uint16_t *out = static_cast<uint16_t *>(a.out) + q_at[k] + h * next_head + 4 * g;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          uint32_t u[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) u[i] = float_to_bf16_bits(o[h][k][t][i] * inv);
          *reinterpret_cast<uint2 *>(out + 16 * t) = make_uint2(u[0] | u[1] << 16, u[2] | u[3] << 16);
        }
        continue;
      }
      const int64_t part = (((int64_t(b) * a.L + l) * a.Hkv + hkv + h) * nsplit + split) * rows_max + r;
      const int64_t parts = int64_t(gridDim.z) * a.L * a.Hkv * nsplit * rows_max;
      float *po = a.ws + part * D + 4 * g;
#pragma unroll
      for (int t = 0; t < NT; ++t)
        *reinterpret_cast<float4 *>(po + 16 * t) = make_float4(o[h][k][t][0], o[h][k][t][1], o[h][k][t][2], o[h][k][t][3]);
      if (g == 0) *reinterpret_cast<float2 *>(a.ws + parts * D + part * 2) = make_float2(m[h][k], lsum[h][k]);
    }
  }
}

template <int NH, int ROWS, int NW>
static void go_four(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  const dim3 grid(unsigned(p.splits), unsigned(a.L * (a.Hkv / (NH * p.heads))), unsigned(a.B));
  const int64_t row = int64_t(a.Hkv) * 64;
  if (a.num_slots <= (1 << 24) && row < (1 << 24) && a.num_slots * row <= (int64_t(1) << 32))
    k_attend_four<NH, ROWS, NW, true><<<grid, WAVE * NW, 0, st>>>(a, p.heads, p.rows);
  else
    k_attend_four<NH, ROWS, NW, false><<<grid, WAVE * NW, 0, st>>>(a, p.heads, p.rows);
}

// Up to 16 rows.
template <int NW> static void go_four_w(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  if (p.rows > 8) p.pair ? go_four<2, 16, NW>(a, p, st) : go_four<1, 16, NW>(a, p, st);
  else p.pair ? go_four<2, 8, NW>(a, p, st) : go_four<1, 8, NW>(a, p, st);
}

hipError_t launch_attend_four(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  KTimer kt_("k_attend_four", st);
  const int waves = p.heads * p.parts;
  if (p.rows > 16 && waves == 4) go_four<1, 32, 4>(a, p, st);
  else if (p.rows <= 16 && waves == 8) go_four_w<8>(a, p, st);
  else if (p.rows <= 16 && waves == 4) go_four_w<4>(a, p, st);
  else return hipErrorInvalidConfiguration;
  return hipGetLastError();
}

}  // namespace ikv
