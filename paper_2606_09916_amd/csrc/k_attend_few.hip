// Attention of few query rows: the decode of one token, or a chunk of a few tokens whose
// rows (n tokens x Hq / Hkv heads) of a KV head fit one 16-row matrix block, or two (NR) over
// the 8-bit cache with bf16 outputs (the other types' registers hold one).
//
// Bound by reading the rows of the list once (2 D + 8 bytes per entry, head and layer in
// 8-bit form, 4 D in bf16): 36 layers x 8 heads x 8192 int8 entries in 105 us (5.9 TB/s), bf16
// 187 us (6.4), 48 x 8 x 92,300 int8 in 1.49 ms (6.3). A wave owns one KV head and a split of the list and keeps
// everything in registers; the waves of a workgroup own adjacent heads, so together they
// read whole pieces of 4 rows. It walks blocks of 32 entries, the next block's rows on
// their way while one is computed:
//   S^T = K Q^T  (16 entries x 16 rows per product); lane (g, c) then holds entries
//                16 kb + 4 g + i of row c, times their scales
//   softmax      a reference per row and the sum of this lane's own weights; the reference
//                moves only when a logit is FEW_SLACK above it (weights stay below 2^8)
//   O^T += V^T P^T over the 32 entries. The contraction may take the entries in any order,
//                so index 8 g + e stands for entry 4 g + e (e < 4) or 16 + 4 g + e - 4: the
//                weights a lane holds are its operand as they are. A lane loads its D / 16
//                channels of those 8 entries' value rows, and byte permutes make the
//                operand of channel D / 16 c + j from them: no transpose through LDS.
// Codes enter the products as bf16, exactly; scales multiply the logits and the weights in
// float32. The weights are split into bf16 parts (two for bf16 outputs: 2^-17; three for
// float32 ones, and three for float32 queries: 2^-25), which costs matrix work that the
// reads hide. Values that are not finite (bf16 ones, E4M3's NaN codes) are left out of blocks that
// some row does not see whole and added after the loop; scales reach weights, which are set to
// zero where an entry is not seen. Over bf16 rows of D = 128 the instance spills 28 to 39 scalar
// registers (20 bytes a lane).
#include <math.h>

#include "attend.hpp"
#include "ikv_internal.hpp"
#include "kv_codes.hpp"

namespace ikv {

constexpr float FEW_SLACK = 8.f;                 // log2
constexpr int FEW_BLOCK = 32;                    // entries per block
typedef uint32_t u32x2_few __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_few __attribute__((ext_vector_type(4)));

// x as bf16 parts, the first the nearest, each next one the nearest of what is left.
template <int PARTS>
__device__ __forceinline__ void split_parts(const float (&x)[8], bf16x8_k (&o)[PARTS]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float r = x[e];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      o[p][e] = __bf16(r);
      r -= float(o[p][e]);
    }
  }
}

template <int FMT, typename IO, int D, int NR, bool O32>
__global__ void __launch_bounds__(64 * FEW_WAVES) __attribute__((amdgpu_waves_per_eu(2)))
k_attend_few(AttendArgs a, int heads, int rows_max) {
  constexpr int ES = FMT == KV_BF16 ? 2 : 1;     // bytes per element
  constexpr int KS = D / 32;                     // 32-channel steps of the first product
  constexpr int NC = D / 16;                     // channels of a lane in the second
  constexpr int KW = D * ES / 64;                // 16-byte loads of a lane per 16 key rows
  constexpr int VW = NC * ES / 4;                // words of a lane per value row
  constexpr int QP = sizeof(IO) == 4 ? 3 : 1;    // bf16 parts of the queries
  constexpr int PP = sizeof(IO) == 4 ? 3 : 2;    // and of the weights
  constexpr int NB = 2;                          // blocks of entries in registers (three or four: no faster)
  __shared__ __align__(16) float sc[FEW_WAVES][2][FEW_BLOCK];
  extern __shared__ float joint[];               // the parts' states, where a head has several waves

  const int b = blockIdx.z;
  const ikv_session s = a.sess[b];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int ngrp = a.Hkv / heads, parts_wg = (blockDim.x >> 6) / heads, part_wg = w / heads;
  const int l = blockIdx.y / ngrp, hkv = (blockIdx.y - l * ngrp) * heads + w % heads;
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
    const int r = min(16 * k + c, rows - 1), t = r / G, h = r - t * G;
    own[k] = N - n + t;
    q_at[k] = before * a.L * a.Hq * D + ((int64_t(l) * a.Hq + hkv * G + h) * n + t) * D;
  }

  // entries seen by any token: up to the sinks, then [lo, N)
  const int lo = a.window ? max(0, N - n - a.window + 1) : 0;
  const int first = min(a.sinks, lo), gap = lo - first;        // index v stands for entry v, or v + gap from `first` on
  const int T = N - gap;
  const int pieces = nsplit * parts_wg, chunk = ((T + pieces - 1) / pieces + 15) & ~15;
  const int v0 = min(T, (split * parts_wg + part_wg) * chunk), v1 = min(T, v0 + chunk);

  float m[NR], lsum[NR];                         // reference of row 16 k + c; this lane's sum of its weights
  f32x4_k o[NR][NC];                             // o[k][j][i]: channel NC (4 g + i) + j of that row
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    m[k] = -INFINITY;
    lsum[k] = 0.f;
#pragma unroll
    for (int j = 0; j < NC; ++j) o[k][j] = f32x4_k{0.f, 0.f, 0.f, 0.f};
  }

  if (v0 < v1) {
    // queries as the B operand, channels in the order the key loads have them
    bf16x8_k qf[NR][KS][QP];
#pragma unroll
    for (int k = 0; k < NR; ++k)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int ch = FMT == KV_BF16 ? 32 * ks + 8 * g : 64 * (ks >> 1) + 16 * g + 8 * (ks & 1);
        float x[8];
        load8(static_cast<const IO *>(a.q) + q_at[k] + ch, x);
        split_parts<QP>(x, qf[k][ks]);
      }
    const uint32_t row_bytes = uint32_t(a.Hkv) * D * ES;
    const int64_t layer = int64_t(l) * a.num_slots;
    // wave-uniform bases; a row is a per-lane byte offset, 32 bits wide where a layer is below 4 GB
    const char *kbase = static_cast<const char *>(a.k) + (layer * a.Hkv + hkv) * D * ES;
    const char *vbase = static_cast<const char *>(a.v) + (layer * a.Hkv + hkv) * D * ES;
    auto row_at = [&](int sl, uint32_t within) {
      if constexpr (O32) return uint32_t(sl) * row_bytes + within;
      else return uint64_t(uint32_t(sl)) * row_bytes + within;
    };
    const float2 *sbase = reinterpret_cast<const float2 *>(a.scales) + layer * a.Hkv + hkv;
    const int32_t *list = a.live + s.slot_off;
    const float to_log2 = 1.4426950408889634f / sqrtf(float(D));

    struct Block {
      uint4 k[2][KW];
      uint32_t v[8][VW];
      float2 s;
    };
    // slot of index base + (lane & 31), the last index's past the end
    auto slots = [&](int base) __attribute__((always_inline)) {
      const int v = min(base + (lane & 31), v1 - 1);
      return list[v < first ? v : v + gap];
    };
    // Value rows go past the caches (nothing reads them again: 123 -> 113 us at 8192 entries); key
    // rows do not, since two loads of 64 bytes share each of their lines (so: 121).
    auto load = [&](Block &x, int sl) __attribute__((always_inline)) {
      if constexpr (FMT != KV_BF16)                // in the order of use
        x.s = *reinterpret_cast<const float2 *>(reinterpret_cast<const char *>(sbase) + row_at(sl, 0) / (D / 8));
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const char *p = kbase + row_at(__builtin_amdgcn_ds_bpermute(4 * (16 * kb + c), sl), 16 * g);
#pragma unroll
        for (int j = 0; j < KW; ++j) x.k[kb][j] = *reinterpret_cast<const uint4 *>(p + 64 * j);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = e < 4 ? 4 * g + e : 16 + 4 * g + e - 4;
        const char *p = vbase + row_at(__builtin_amdgcn_ds_bpermute(4 * at, sl), c * (NC * ES));
        if constexpr (VW == 1) x.v[e][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(p));
        else if constexpr (VW == 2) {
          const u32x2_few y = __builtin_nontemporal_load(reinterpret_cast<const u32x2_few *>(p));
          x.v[e][0] = y.x;
          x.v[e][1] = y.y;
        } else {
          const u32x4_few y = __builtin_nontemporal_load(reinterpret_cast<const u32x4_few *>(p));
          x.v[e][0] = y.x;
          x.v[e][1] = y.y;
          x.v[e][2] = y.z;
          x.v[e][3] = y.w;
        }
      }
    };
    bool odd = false;                              // a value that is not finite was left out
    auto compute = [&](Block &x, int base) __attribute__((always_inline)) {
      f32x4_k acc[NR][2];
#pragma unroll
      for (int k = 0; k < NR; ++k) acc[k][0] = acc[k][1] = f32x4_k{0.f, 0.f, 0.f, 0.f};
      if constexpr (FMT != KV_BF16) {
        if (lane < FEW_BLOCK) {
          sc[w][0][lane] = x.s.x * to_log2;
          sc[w][1][lane] = x.s.y;
        }
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          uint4 u;
          if constexpr (FMT == KV_BF16) u = x.k[kb][ks];
          else {
            const uint4 y = x.k[kb][ks >> 1];
            const uint2 p = codes4<FMT>(ks & 1 ? y.z : y.x), q = codes4<FMT>(ks & 1 ? y.w : y.y);
            u = make_uint4(p.x, p.y, q.x, q.y);
          }
          const bf16x8_k kf = __builtin_bit_cast(bf16x8_k, u);
#pragma unroll
          for (int k = 0; k < NR; ++k)
#pragma unroll
            for (int p = QP - 1; p >= 0; --p)
              acc[k][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[k][ks][p], acc[k][kb], 0, 0, 0);
        }
      float4 vs[2];
      if constexpr (FMT != KV_BF16) {
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const float4 ks = *reinterpret_cast<const float4 *>(&sc[w][0][16 * kb + 4 * g]);
          vs[kb] = *reinterpret_cast<const float4 *>(&sc[w][1][16 * kb + 4 * g]);
#pragma unroll
          for (int k = 0; k < NR; ++k) acc[k][kb] *= f32x4_k{ks.x, ks.y, ks.z, ks.w};
        }
        __builtin_amdgcn_wave_barrier();
      } else {
#pragma unroll
        for (int k = 0; k < NR; ++k) acc[k][0] *= to_log2, acc[k][1] *= to_log2;
      }
      // a block that every token sees whole needs no mask: its last entry is at or before the
      // oldest token's own, and its first inside the newest's window or all of it among the sinks
      const int last = base + FEW_BLOCK - 1, oldest = N - n;
      const int jl = last < first ? last : last + gap, j0 = base < first ? base : base + gap;
      const bool whole = last < v1 && jl <= oldest && (a.window == 0 || jl < a.sinks || j0 > N - 1 - a.window);
      bf16x8_k pf[NR][PP];
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        uint32_t hidden = 0;                       // bit 4 kb + i: not seen by this row
        if (!whole) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int v = base + 16 * kb + 4 * g + i, j = v < first ? v : v + gap;
              const bool see = (v < v1) & (j <= own[k]) & ((a.window == 0) | (j < a.sinks) | (j > own[k] - a.window));
              hidden |= see ? 0u : 1u << (4 * kb + i);
              acc[k][kb][i] = see ? acc[k][kb][i] : -INFINITY;
            }
        }
        float tmax = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) tmax = fmaxf(tmax, acc[k][kb][i]);
        if (__builtin_amdgcn_ballot_w64(!(tmax - m[k] <= FEW_SLACK)) != 0) {
          tmax = fmaxf(tmax, __shfl_xor(tmax, 16, WAVE));
          tmax = fmaxf(tmax, __shfl_xor(tmax, 32, WAVE));
          const float mn = !(tmax - m[k] <= FEW_SLACK) ? fmaxf(m[k], tmax) : m[k];     // by this row alone
          const float corr = m[k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[k] - mn);
          m[k] = mn;
          lsum[k] *= corr;
#pragma unroll
          for (int j = 0; j < NC; ++j) o[k][j] *= corr;
        }
        const float ms = m[k] == -INFINITY ? 0.f : m[k];     // no logit above -inf yet: the weights are 2^-inf
        float pw[8];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float p = __builtin_amdgcn_exp2f(acc[k][kb][i] - ms);
            lsum[k] += p;
            if constexpr (FMT != KV_BF16) {
              p *= (&vs[kb].x)[i];
              if (hidden >> (4 * kb + i) & 1) p = 0.f;      // the scale of an unseen row may be anything
            }
            pw[4 * kb + i] = p;
          }
        split_parts<PP>(pw, pf[k]);
      }
      if constexpr (FMT != KV_INT8) {
        if (!whole) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int k = 0; k < VW; ++k) {
              if constexpr (FMT == KV_BF16) {
                odd |= odd_low(x.v[e][k]) | odd_high(x.v[e][k]);
                x.v[e][k] = bf16_finite(x.v[e][k]);
              } else {
                const uint32_t nans = e4m3_nans(x.v[e][k]);
                odd |= nans != 0;
                x.v[e][k] = e4m3_finite(x.v[e][k], nans);
              }
            }
        }
      }
      // the operand of channels NC c + STEP k .. at a time
      constexpr int STEP = FMT == KV_BF16 ? 2 : 4;
#pragma unroll
      for (int k = 0; k < VW; ++k) {
        uint32_t f[STEP][4];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          if constexpr (FMT == KV_BF16) {
            f[0][p] = __builtin_amdgcn_perm(x.v[2 * p + 1][k], x.v[2 * p][k], 0x05040100u);
            f[1][p] = __builtin_amdgcn_perm(x.v[2 * p + 1][k], x.v[2 * p][k], 0x07060302u);
          } else {
            uint32_t y[4];
            codes_across<FMT>(x.v[2 * p][k], x.v[2 * p + 1][k], y);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i][p] = y[i];
          }
        }
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
          const bf16x8_k vf = __builtin_bit_cast(bf16x8_k, make_uint4(f[i][0], f[i][1], f[i][2], f[i][3]));
#pragma unroll
          for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int p = PP - 1; p >= 0; --p)
              o[r][STEP * k + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[r][p], o[r][STEP * k + i], 0, 0, 0);
        }
      }
    };
    // NB blocks in registers: one computed, the others on their way
    Block x[NB];
    int sl[NB];
#pragma unroll
    for (int u = 0; u < NB - 1; ++u) sl[u] = slots(v0 + u * FEW_BLOCK);
    int next = slots(v0 + (NB - 1) * FEW_BLOCK);
#pragma unroll
    for (int u = 0; u < NB - 1; ++u) load(x[u], sl[u]);
    for (int base = v0; base < v1; base += NB * FEW_BLOCK) {
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        constexpr int B1 = NB - 1;
        const int at = base + u * FEW_BLOCK;
        if (u > 0 && at >= v1) break;
        __builtin_amdgcn_sched_barrier(0);
        sl[(u + B1) % NB] = next;
        next = slots(at + NB * FEW_BLOCK);
        load(x[(u + B1) % NB], sl[(u + B1) % NB]);
        __builtin_amdgcn_sched_barrier(0);
        compute(x[u], at);
      }
    }
    if constexpr (FMT != KV_INT8) {
      if (__builtin_amdgcn_ballot_w64(odd) != 0)
        for (int v = v0; v < v1; ++v) {
          const int e = v < first ? v : v + gap;
          const char *row = vbase + row_at(list[e], 0);
#pragma unroll
          for (int k = 0; k < NR; ++k) {
            const bool see = (e <= own[k]) & ((a.window == 0) | (e < a.sinks) | (e > own[k] - a.window));
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int j = 0; j < NC; ++j) {
                const int ch = NC * (4 * g + i) + j;
                if constexpr (FMT == KV_BF16) {
                  const uint16_t y = reinterpret_cast<const uint16_t *>(row)[ch];
                  o[k][j][i] += see && odd_low(y) ? Store<uint16_t>::ld(&y) : 0.f;
                } else {
                  o[k][j][i] += see && (row[ch] & 0x7f) == 0x7f ? __uint_as_float(0x7fc00000u) : 0.f;
                }
              }
          }
        }
    }
  }
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    lsum[k] += __shfl_xor(lsum[k], 16, WAVE);
    lsum[k] += __shfl_xor(lsum[k], 32, WAVE);
  }
  if (parts_wg > 1) {
    // the other waves of a head leave their state in LDS, lane for lane; the first joins them
    constexpr int STATE = (4 * NC + 2) * WAVE;
    if (part_wg > 0) {
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        float *mine = joint + ((w - heads) * NR + k) * STATE + lane;
        mine[0] = m[k];
        mine[WAVE] = lsum[k];
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) mine[(2 + 4 * j + i) * WAVE] = o[k][j][i];
      }
    }
    __syncthreads();
    if (part_wg > 0) return;
    for (int p = 1; p < parts_wg; ++p) {
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        const float *x = joint + ((w + (p - 1) * heads) * NR + k) * STATE + lane;
        const float mp = x[0], mn = fmaxf(m[k], mp);
        const float f = m[k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[k] - mn);
        const float fp = mp == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mp - mn);
        m[k] = mn;
        lsum[k] = lsum[k] * f + x[WAVE] * fp;
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[k][j][i] = o[k][j][i] * f + x[(2 + 4 * j + i) * WAVE] * fp;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    const int r = 16 * k + c;
    if (r >= rows) continue;
    if (nsplit == 1) {
      const float inv = own[k] < 0 ? 0.f : 1.0f / lsum[k];             // nothing seen: zero
      IO *out = static_cast<IO *>(a.out) + q_at[k];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < NC; ++j) out[NC * (4 * g + i) + j] = Store<IO>::from(o[k][j][i] * inv);
      continue;
    }
    const int64_t part = (((int64_t(b) * a.L + l) * a.Hkv + hkv) * nsplit + split) * rows_max + r;
    const int64_t parts = int64_t(gridDim.z) * a.L * a.Hkv * nsplit * rows_max;
    float *po = a.ws + part * D;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NC; j += 4)
        *reinterpret_cast<float4 *>(po + NC * (4 * g + i) + j) =
            make_float4(o[k][j][i], o[k][j + 1][i], o[k][j + 2][i], o[k][j + 3][i]);
    if (g == 0) *reinterpret_cast<float2 *>(a.ws + parts * D + part * 2) = make_float2(m[k], lsum[k]);
  }
}

template <int FMT, typename IO, int D, int NR>
static void go_few(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  KTimer kt_("k_attend_few", st);
  const dim3 grid(unsigned(p.splits), unsigned(a.L * (a.Hkv / p.heads)), unsigned(a.B));
  const size_t lds = size_t(p.parts - 1) * p.heads * NR * (D / 4 + 2) * WAVE * sizeof(float);
  if (a.num_slots * a.Hkv * D * (FMT == KV_BF16 ? 2 : 1) < (int64_t(1) << 32))
    k_attend_few<FMT, IO, D, NR, true><<<grid, WAVE * p.heads * p.parts, lds, st>>>(a, p.heads, p.rows);
  else
    k_attend_few<FMT, IO, D, NR, false><<<grid, WAVE * p.heads * p.parts, lds, st>>>(a, p.heads, p.rows);
}

template <int FMT, typename IO>
static void go_few_d(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  if constexpr (FMT != KV_BF16 && sizeof(IO) == 2) {
    if (p.rows > 16) return a.D == 128 ? go_few<FMT, IO, 128, 2>(a, p, st) : go_few<FMT, IO, 64, 2>(a, p, st);
  }
  a.D == 128 ? go_few<FMT, IO, 128, 1>(a, p, st) : go_few<FMT, IO, 64, 1>(a, p, st);
}

hipError_t launch_attend_few(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  if (a.format == KV_BF16) go_few_d<KV_BF16, uint16_t>(a, p, st);
  else if (a.format == KV_INT8) a.io_f32 ? go_few_d<KV_INT8, float>(a, p, st) : go_few_d<KV_INT8, uint16_t>(a, p, st);
  else a.io_f32 ? go_few_d<KV_E4M3, float>(a, p, st) : go_few_d<KV_E4M3, uint16_t>(a, p, st);
  return p.splits > 1 ? launch_attend_merge(a, p, st) : hipGetLastError();
}

}  // namespace ikv
