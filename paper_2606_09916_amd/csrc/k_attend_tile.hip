// Attention of a chunk of new tokens: blocks of query rows against tiles of 64 entries.
//
// Row R of a KV head is (token R / G, head R % G of the group): a workgroup takes NW x 32
// consecutive rows, so the G heads of a token share every key and value read, and a block's
// tokens are neighbours with nearly the same entries to see. Bound by the matrix cores and the
// vector unit's work per logit together (busy 0.41 to 0.48 of the cycles, at a clock that falls
// to 1.8 to 2.0 GHz under them): Qwen3-8B, 509 tokens over 8192 entries, 2.54 TFLOP: int8 2.70 ms,
// E4M3 2.38; 14B, 1024 tokens, bf16, window 4096, 4.13 TFLOP: 4.06 ms, on the fastest machine
// (2.8 to 3.1, 2.4 to 2.55 and 4.2 to 4.6 on others). 256 rows: of 128, four
// waves, two workgroups a CU stage every tile twice as often (3.06 ms against 2.82); of 64 rows a
// wave the registers spill (6.0 ms).
//   staging   rows or codes go from HBM through registers, are made bf16 (exactly:
//             int8 codes as they are, E4M3 ones with their scales where those are powers of two,
//             as the store writes them; with another scale the product is rounded to bf16; E2M1 ones
//             with their blocks' scales) and
//             written to one of two LDS buffers, the keys a tile before the values: rows of D + 8,
//             entry 16 i + 4 j + k in row 16 i + 4 k + j. Pieces of adjacent rows, as they are written,
//             then lie in different banks, and so do the 16 rows that a product reads of the keys and
//             the 4 entries, 4 rows apart, that it reads of the values (4 bits, whose 16 lanes write 4
//             rows: 4375 -> 4250 us in the case below; the others, bit for bit, as fast as before)
//   S^T = K Q^T with 32 x 32 x 16 products: lane (h, c) holds entries 8 i + 4 h + (0..3) of
//             row c, so a row's softmax is two lanes' business
//   softmax   a reference per row that moves only when a logit is TILE_SLACK above it (the
//             weights stay below 2^8; most tiles exchange nothing between lanes)
//   O^T += V^T P^T: the contraction's order is free, so the weights a lane holds are its
//             operand as they are; the transposing LDS reads (4 entries x 16 channels by 16
//             lanes) bring the value operand in that order from row-major tiles.
// Weights are rounded to bf16 for bf16 outputs (2^-8 each, no more than the output's own
// rounding, and averaged over the entries; their sum is of the unrounded ones): against float64
// the long chunks are off by 0.0018 to 0.0019 where the output's rounding alone is 0.0017. float32
// outputs take queries and weights as three bf16 parts, which at D = 128 do not fit the
// registers: 42 to 67 of a lane's are spilled (8 layers, 200 tokens over 4000: 340 to 377 us). Of the
// bf16 outputs' instances, int8 with eight waves, and bf16 rows and E4M3 with four, spill two.
// 4 bits, 14B, 1021 tokens, window 4096, 4.12 TFLOP: 4.20 ms, 0.98 PFLOP/s: as bf16 rows, since the
// reads do not bound it. Keys as codes in LDS, made bf16 before each product, take 1% longer (a third
// of the LDS reads less, a third of the vector work more), 64 rows a wave in 512 registers 9.0 ms.
#include <math.h>

#include <type_traits>

#include "attend.hpp"
#include "ikv_internal.hpp"
#include "kv_codes.hpp"

namespace ikv {

typedef float f32x16_k __attribute__((ext_vector_type(16)));

constexpr float TILE_SLACK = 8.f;                // log2

// 8 floats as PARTS bf16 operands (nearest, then the nearest of what is left).
template <int PARTS>
__device__ __forceinline__ void tile_parts(const float *x, bf16x8_k (&o)[PARTS]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float r = x[e];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      o[p][e] = __bf16(r);
      if (p + 1 < PARTS) r -= float(o[p][e]);
    }
  }
}

// The LDS row of a tile's entry, and the entry of a row.
__device__ __forceinline__ int tile_place(int e) { return (e & ~15) | (e & 3) << 2 | (e >> 2 & 3); }

template <int FMT, typename IO, int D, int NW, bool O32>
__global__ void __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2)))
k_attend_tile(AttendArgs a, int blocks, int nsplit, int units) {
  constexpr int RB = kv_row_bytes(FMT, D);
  constexpr int NT = 64 * NW, ROWS = 32 * NW;
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int ROW = D + 8;                      // bf16 of a row in LDS, 16 bytes past a multiple of the banks
  constexpr int PB = RB < 64 ? 8 : 16;           // bytes of a piece
  constexpr int PPR = RB / PB;                   // pieces of a row
  constexpr int PIECES = TILE_KEYS * PPR;        // of a tile's keys (as many of its values)
  constexpr int PP_ = PIECES > NT ? PIECES / NT : 1;       // pieces of keys, and of values, of a thread
  constexpr int QP = sizeof(IO) == 4 ? 3 : 1, PP = QP;
  static_assert(PIECES % NT == 0 || 2 * PIECES == NT, "whole pieces, or one of keys or values a thread");
  __shared__ __align__(16) uint16_t ks_[2][TILE_KEYS * ROW];
  __shared__ __align__(16) uint16_t vs_[2][TILE_KEYS * ROW];
  __shared__ __align__(16) float sc_[2][2][TILE_KEYS];               // scales: keys' (times log2 e / sqrt D), values'

  // units (session, layer, KV head) in steps of 8, so that a unit's blocks and splits run on
  // one XCD and share its rows in that L2; the blocks with the most entries first
  const int per = blocks * nsplit;
  const int id = blockIdx.x, in = (id >> 3) % per, unit = (id >> 3) / per * 8 + (id & 7);
  if (unit >= units) return;
  const int rb = blocks - 1 - in / nsplit, split = in % nsplit;
  const int hkv = unit % a.Hkv, l = unit / a.Hkv % a.L, b = unit / a.Hkv / a.L;
  const ikv_session s = a.sess[b];
  const int G = a.Hq / a.Hkv, n = s.qe - s.qs, rows = n * G;
  const int row0 = rb * ROWS;
  if (row0 >= rows) return;
  int64_t before = 0;
  for (int i = 0; i < b; ++i) before += a.sess[i].qe - a.sess[i].qs;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h2 = lane >> 5, c = lane & 31;
  const int row = row0 + 32 * w + c, rr = min(row, rows - 1);
  const int t = rr / G, h = rr - t * G;
  const int64_t q_at = before * a.L * a.Hq * D + ((int64_t(l) * a.Hq + hkv * G + h) * n + t) * D;

  // what the block sees: up to the sinks, then [lo, own of its newest token]
  const int N = max(0, min(a.n_live[b], s.N)), own = N - n + t;
  const int t0 = row0 / G, t1 = min(rows - 1, row0 + ROWS - 1) / G;
  const int own0 = N - n + t0, own1 = N - n + t1;
  const int lo = a.window ? max(0, own0 - a.window + 1) : 0;
  const int first = min(a.sinks, lo), gap = lo - first;        // index v stands for entry v, or v + gap from `first` on
  const int T = max(0, own1 + 1 - gap);
  const int ntile = (T + TILE_KEYS - 1) / TILE_KEYS;
  const int tb = int(int64_t(ntile) * split / nsplit), te = int(int64_t(ntile) * (split + 1) / nsplit);
  // this wave's tokens
  const int wrow0 = min(row0 + 32 * w, rows - 1), wrow1 = min(row0 + 32 * w + 31, rows - 1);
  const int wown0 = N - n + wrow0 / G, wown1 = N - n + wrow1 / G;
  const bool wave_on = row0 + 32 * w < rows;

  float m = -INFINITY, lsum = 0.f;
  f32x16_k o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.f;

  if (tb < te) {
    bf16x8_k qf[KS][QP];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      float x[8];
      load8(static_cast<const IO *>(a.q) + q_at + 16 * ks + 8 * h2, x);
      tile_parts<QP>(x, qf[ks]);
    }
    const uint32_t row_bytes = uint32_t(a.Hkv) * RB;
    // byte offset of a slot's row: 32 bits, by a 24-bit product, where slots, rows and layers are small enough
    auto row_at = [&](int sl) __attribute__((always_inline)) {
      if constexpr (O32) return uint32_t(__umul24(uint32_t(sl), row_bytes));
      else return uint64_t(uint32_t(sl)) * row_bytes;
    };
    const int64_t layer = int64_t(l) * a.num_slots;
    const char *kbase = static_cast<const char *>(a.k) + (layer * a.Hkv + hkv) * RB;
    const char *vbase = static_cast<const char *>(a.v) + (layer * a.Hkv + hkv) * RB;
    const char *sbase = reinterpret_cast<const char *>(a.scales) + (layer * a.Hkv + hkv) * (FMT == KV_E2M1 ? D / 16 : 8);
    const int32_t *list = a.live + s.slot_off;
    const float to_log2 = 1.4426950408889634f / sqrtf(float(D));

    // Staging: in the iteration of tile i, the keys of tile i + 2 and the values and scales of
    // tile i + 1 go from registers to LDS, and those of the tiles after them are loaded. A
    // thread's pieces of a tile's values lie in the rows of its pieces of the keys, an iteration
    // later: a row's byte offset is found once. Tiles wholly past the sinks and before the end
    // read their slots at a uniform address.
    const bool takes_k = PIECES >= NT || tid < PIECES, takes_v = PIECES >= NT || tid >= PIECES;
    typedef typename std::conditional<O32, uint32_t, uint64_t>::type Off;
    struct Regs {
      uint4 k[PP_], v[PP_];
      float2 sc;                                   // int8: of entry `lane`
      float ks[PP_], vs[PP_];                      // E4M3: of the pieces' rows; E2M1: of their blocks
    };
    struct Slots { int32_t s[PP_], sc; };
    struct Offs { Off o[PP_], sc; };
    auto entry = [&](int v) __attribute__((always_inline)) {
      v = max(0, min(v, T - 1));                   // past the end the last one again, masked
      return v < first ? v : v + gap;
    };
    const int key0 = tid % PIECES / PPR;           // LDS row of the thread's first piece; each next one NT / PPR on
    const int at0 = tile_place(key0);              // and its entry within the tile
    auto slots = [&](int tile) __attribute__((always_inline)) {
      Slots x;
      const int va = tile * TILE_KEYS;
      if (va >= first && va + TILE_KEYS <= T) {
        const int32_t *at = list + (va + gap);
#pragma unroll
        for (int i = 0; i < PP_; ++i) x.s[i] = at[at0 + i * (NT / PPR)];
        if constexpr (FMT == KV_INT8) x.sc = at[lane];
      } else {
#pragma unroll
        for (int i = 0; i < PP_; ++i) x.s[i] = list[entry(va + at0 + i * (NT / PPR))];
        if constexpr (FMT == KV_INT8) x.sc = list[entry(va + lane)];
      }
      return x;
    };
    auto offsets = [&](const Slots &x) __attribute__((always_inline)) {
      Offs y;
#pragma unroll
      for (int i = 0; i < PP_; ++i) y.o[i] = row_at(x.s[i]) + Off(tid % PPR * PB);
      if constexpr (FMT == KV_INT8) y.sc = row_at(x.sc);
      return y;
    };
    auto scale_at = [&](Off row) __attribute__((always_inline)) {           // of a row offset: 8 bytes for D
      return *reinterpret_cast<const float2 *>(sbase + (row / D) * 8);
    };
    // E2M1: of the block that holds a piece, by its byte offset; i: of keys (0), of values (1)
    auto block_scale = [&](Off piece, int i) __attribute__((always_inline)) {
      const uint8_t *p = reinterpret_cast<const uint8_t *>(sbase) + piece / RB * (D / 16) + piece % RB / 16;
      return __uint_as_float(uint32_t(p[i * (D / 32)]) << 23);
    };
    auto piece_at = [](const char *p) __attribute__((always_inline)) {
      if constexpr (PB == 16) return *reinterpret_cast<const uint4 *>(p);
      const uint2 x = *reinterpret_cast<const uint2 *>(p);
      return make_uint4(x.x, x.y, 0u, 0u);
    };
    // the keys of one tile (offsets k) and the values and scales of the one before (offsets v)
    auto load = [&](const Offs &k, const Offs &v, Regs &r) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < PP_; ++i) {
        if (takes_k) {
          r.k[i] = piece_at(kbase + k.o[i]);
          if constexpr (FMT == KV_E4M3) r.ks[i] = scale_at(k.o[i]).x;
          if constexpr (FMT == KV_E2M1) r.ks[i] = block_scale(k.o[i], 0);
        }
        if (takes_v) {
          r.v[i] = piece_at(vbase + v.o[i]);
          if constexpr (FMT == KV_E4M3) r.vs[i] = scale_at(v.o[i]).y;
          if constexpr (FMT == KV_E2M1) r.vs[i] = block_scale(v.o[i], 1);
        }
      }
      if constexpr (FMT == KV_INT8) r.sc = scale_at(v.sc);
    };
    // whether some token of [o0, o1] does not see all of the tile's entries
    auto edge = [&](int tile, int o0, int o1) __attribute__((always_inline)) {
      const int va = tile * TILE_KEYS, vb = va + TILE_KEYS - 1;
      const int ja = va < first ? va : va + gap, jb = vb < first ? vb : vb + gap;
      return !(vb < T && jb <= o0 && (a.window == 0 || jb < a.sinks || ja > o1 - a.window));
    };
    // the values and scales of `tile` (buffer tile & 1) and the keys of tile + 1. A value that is
    // not finite (a bf16 one, a NaN code, a scale, a product of both) would turn the zero weights
    // of rows that do not see it into NaN: in a tile that some row does not see whole it is left
    // out and added after the loop.
    bool odd = false;
    auto put = [&](uint16_t *dst, uint4 x, float scale, bool value, bool look) __attribute__((always_inline)) {
      if constexpr (FMT == KV_BF16) {
        if (look) {
          odd |= odd_low(x.x) | odd_high(x.x) | odd_low(x.y) | odd_high(x.y) | odd_low(x.z) | odd_high(x.z) |
                 odd_low(x.w) | odd_high(x.w);
          x = make_uint4(bf16_finite(x.x), bf16_finite(x.y), bf16_finite(x.z), bf16_finite(x.w));
        }
        *reinterpret_cast<uint4 *>(dst) = x;
      } else if constexpr (FMT == KV_E2M1) {
        // (infinite ones in any tile where the weights have several parts: k_attend_four.hip)
        bool out = look && !(scale < 0x1p126f);
        if constexpr (PP > 1) out |= value && scale >= 0x1p126f && scale < INFINITY;
        if (__builtin_amdgcn_ballot_w64(out) != 0) {
#pragma unroll
          for (int i = 0; i < PB / 4; ++i) {
            const uint32_t z = e2m1_odd((&x.x)[i], __float_as_uint(scale) >> 23);
            odd |= z != 0;
            (&x.x)[i] &= ~z;
          }
          if (!(fabsf(scale) < INFINITY)) scale = 1.0f;
        }
#pragma unroll
        for (int i = 0; i < PB / 4; ++i) reinterpret_cast<uint4 *>(dst)[i] = e2m1_scaled8((&x.x)[i], scale);
      } else {
        uint2 y[4];
        if constexpr (FMT == KV_E4M3) {
          y[0] = e4m3_scaled4(x.x, scale), y[1] = e4m3_scaled4(x.y, scale);
          y[2] = e4m3_scaled4(x.z, scale), y[3] = e4m3_scaled4(x.w, scale);
          if (__builtin_amdgcn_ballot_w64(no_power(scale)) != 0 && no_power(scale)) {
            y[0] = e4m3_times4(x.x, scale), y[1] = e4m3_times4(x.y, scale);
            y[2] = e4m3_times4(x.z, scale), y[3] = e4m3_times4(x.w, scale);
          }
          // NaN codes, products past the largest bf16 (448 * 2^119 is below it), scales that are not finite
          if (look && __builtin_amdgcn_ballot_w64((e4m3_nans(x.x) | e4m3_nans(x.y) | e4m3_nans(x.z) | e4m3_nans(x.w)) != 0 ||
                                                  !(fabsf(scale) < 0x1p119f)) != 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              odd |= odd_low(y[i].x) | odd_high(y[i].x) | odd_low(y[i].y) | odd_high(y[i].y);
              y[i] = make_uint2(bf16_finite(y[i].x), bf16_finite(y[i].y));
            }
          }
        } else {
          y[0] = codes4<FMT>(x.x), y[1] = codes4<FMT>(x.y), y[2] = codes4<FMT>(x.z), y[3] = codes4<FMT>(x.w);
        }
        reinterpret_cast<uint4 *>(dst)[0] = make_uint4(y[0].x, y[0].y, y[1].x, y[1].y);
        reinterpret_cast<uint4 *>(dst)[1] = make_uint4(y[2].x, y[2].y, y[3].x, y[3].y);
      }
    };
    auto store = [&](const Regs &r, int tile, int par) __attribute__((always_inline)) {
      const bool look = edge(tile, own0, own1);
      constexpr int EL = D / PPR;                  // elements of a piece
      const int at = tid % PPR * EL;
#pragma unroll
      for (int i = 0; i < PP_; ++i) {
        const int key = key0 + i * (NT / PPR);
        if (takes_k) put(&ks_[par ^ 1][key * ROW + at], r.k[i], r.ks[i], false, false);
        if (takes_v) put(&vs_[par][key * ROW + at], r.v[i], r.vs[i], true, look);
      }
      if constexpr (FMT == KV_INT8) {
        if (tid < TILE_KEYS) {
          const bool bad = look && !(fabsf(r.sc.y) < INFINITY);
          odd |= bad;
          sc_[par][0][tid] = r.sc.x * to_log2;
          sc_[par][1][tid] = bad ? 0.f : r.sc.y;
        }
      }
    };
    typedef f32x16_k Logits[2];
    // channels 16 ks of the logits of a tile whose keys are in buffer `par`, both 32-entry halves
    auto first_product = [&](Logits &x, int par, int ks) __attribute__((always_inline)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bf16x8_k kf = *reinterpret_cast<const bf16x8_k *>(&ks_[par][(32 * kb + tile_place(c)) * ROW + 8 * h2 + 16 * ks]);
#pragma unroll
        for (int p = QP - 1; p >= 0; --p) x[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks][p], x[kb], 0, 0, 0);
      }
    };
    // The iteration of `tile`, its logits in x (raw products): their scales, mask and reference,
    // then its weights and second product beside the first product of the next tile (into y).
    auto step = [&](Logits &x, Logits &y, int tile, int par, Regs &r, const Offs &ko, const Offs &vo)
        __attribute__((always_inline)) {
      if constexpr (FMT == KV_INT8) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            const float4 ks = *reinterpret_cast<const float4 *>(&sc_[par][0][32 * kb + 8 * i4 + 4 * h2]);
            x[kb][4 * i4] *= ks.x;
            x[kb][4 * i4 + 1] *= ks.y;
            x[kb][4 * i4 + 2] *= ks.z;
            x[kb][4 * i4 + 3] *= ks.w;
          }
      }
      if (edge(tile, wown0, wown1)) {
        const int va = tile * TILE_KEYS;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int v = va + 32 * kb + 8 * (i >> 2) + 4 * h2 + (i & 3), j = v < first ? v : v + gap;
            const bool see = (v < T) & (j <= own) & ((a.window == 0) | (j < a.sinks) | (j > own - a.window));
            x[kb][i] = see ? x[kb][i] : -INFINITY;
          }
      }
      float tmax = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) tmax = fmaxf(tmax, x[kb][i]);
      if constexpr (FMT != KV_INT8) tmax *= to_log2;
      if (__builtin_amdgcn_ballot_w64(!(tmax - m <= TILE_SLACK)) != 0) {
        tmax = fmaxf(tmax, __shfl_xor(tmax, 32, WAVE));
        const float mn = !(tmax - m <= TILE_SLACK) ? fmaxf(m, tmax) : m;     // by this row alone
        const float corr = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        lsum *= corr;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] *= corr;
      }
      const float ms = m == -INFINITY ? 0.f : m;   // no logit above -inf yet: the weights are 2^-inf
      store(r, tile + 1, par ^ 1);
      load(ko, vo, r);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) y[kb][i] = 0.f;
      // The products one at a time with the vector work of 16-entry step st between them, in an
      // order that the fences keep: NP products of the next tile's logits, then, by turns, one of
      // them and one of step st - 1's values, then the last step's values. Operands are read from
      // LDS AHEAD products before their own. (509 tokens over 8192 entries, int8: 2739 us; in the
      // compiler's own order 2824; 4 bits, four waves, 1021 tokens, window 4096: 4170, 4340.) Four waves
      // with twice the pieces each, and float32's three parts, have no registers for operands ahead:
      // there the compiler orders them.
      constexpr bool FENCES = (NW == 8 || FMT == KV_E2M1) && QP == 1;
      constexpr int NP = D / 32, OPS = 8 * NP, AHEAD = FENCES ? 2 : 0;
      auto is_first = [](int n) { return n < NP || (n < 7 * NP && (n - NP) % 2 == 0); };
      auto first_of = [](int n) { return n < NP ? n : NP + (n - NP) / 2; };
      auto second_of = [](int n) { return n < 7 * NP ? (n - NP) / 2 : n - 4 * NP; };
      const int lr = lane & 15;
      const uint16_t *kr = &ks_[par ^ 1][tile_place(c) * ROW + 8 * h2];
      const uint16_t *vr = &vs_[par][(4 * (lr >> 2) + h2) * ROW + 16 * (lane >> 4 & 1) + 4 * (lr & 3)];
      auto operand = [&](int n) __attribute__((always_inline)) {
        if (is_first(n)) {
          const int q = first_of(n);
          return *reinterpret_cast<const uint4 *>(kr + 32 * (q & 1) * ROW + 16 * (q >> 1));
        }
        const int q = second_of(n), st = q / NP, db = q % NP;
        const uint2 x0 = read_tr16(vr + 16 * st * ROW + 32 * db), x1 = read_tr16(vr + (16 * st + 2) * ROW + 32 * db);
        return make_uint4(x0.x, x0.y, x1.x, x1.y);
      };
      uint4 f[AHEAD + 1];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) f[n] = operand(n);
      bf16x8_k pf[2][PP];
      float w[8], sum = 0.f;
      float4 vs[2];
#pragma unroll
      for (int n = 0; n < OPS; ++n) {
        if constexpr (FENCES) __builtin_amdgcn_sched_barrier(0);
        if (n + AHEAD < OPS) f[(n + AHEAD) % (AHEAD + 1)] = operand(n + AHEAD);
        const bf16x8_k u = __builtin_bit_cast(bf16x8_k, f[n % (AHEAD + 1)]);
        if (is_first(n)) {
          const int q = first_of(n);
#pragma unroll
          for (int p = QP - 1; p >= 0; --p)
            y[q & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u, qf[q >> 1][p], y[q & 1], 0, 0, 0);
        } else {
          const int q = second_of(n);
#pragma unroll
          for (int p = PP - 1; p >= 0; --p)
            o[q % NP] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u, pf[q / NP & 1][p], o[q % NP], 0, 0, 0);
        }
        if (n < 7 * NP) {
          const int st = n < NP ? 0 : 1 + (n - NP) / (2 * NP);
          const int at = n < NP ? n : (n - NP) % (2 * NP), of = n < NP ? NP : 2 * NP;
          if constexpr (FMT == KV_INT8) {
            if (at == 0) {
#pragma unroll
              for (int i4 = 0; i4 < 2; ++i4)
                vs[i4] = *reinterpret_cast<const float4 *>(&sc_[par][1][16 * st + 8 * i4 + 4 * h2]);
            }
          }
#pragma unroll
          for (int e = 8 * at / of; e < 8 * (at + 1) / of; ++e) {
            const float z = x[st >> 1][8 * (st & 1) + e];
            w[e] = __builtin_amdgcn_exp2f(FMT == KV_INT8 ? z - ms : fmaf(z, to_log2, -ms));
            sum += w[e];
            if constexpr (FMT == KV_INT8) w[e] *= (&vs[e >> 2].x)[e & 3];
          }
          if (at == of - 1) tile_parts<PP>(w, pf[st & 1]);
        }
      }
      if constexpr (FENCES) __builtin_amdgcn_sched_barrier(0);
      lsum += sum;
    };
    auto iterate = [&](Logits &x, Logits &y, int tile, int par, Regs &r, const Offs &ko, const Offs &vo)
        __attribute__((always_inline)) {
      if (wave_on) step(x, y, tile, par, r, ko, vo);
      else {
        store(r, tile + 1, par ^ 1);
        load(ko, vo, r);
      }
    };
    Logits sA, sB;
    Regs r;
    Offs oa = offsets(slots(tb)), ob = offsets(slots(tb + 1));
    load(oa, oa, r);
    store(r, tb - 1, 1);                           // keys of the first tile (its values too, overwritten below)
    load(ob, oa, r);
    store(r, tb, 0);
    oa = offsets(slots(tb + 2));
    load(oa, ob, r);
    Slots next = slots(tb + 3);
    __syncthreads();
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) sA[kb][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) first_product(sA, 0, ks);
    __syncthreads();                               // before keys of tile tb + 2 take that buffer
    for (int tile = tb; tile < te; tile += 2) {
      ob = offsets(next);                          // of tile + 3; oa are those of tile + 2
      next = slots(tile + 4);
      iterate(sA, sB, tile, 0, r, ob, oa);
      __syncthreads();
      if (tile + 1 >= te) break;
      oa = offsets(next);
      next = slots(tile + 5);
      iterate(sB, sA, tile + 1, 1, r, oa, ob);
      __syncthreads();
    }
    // (the hint keeps E4M3's out of the loop's registers: 8 float32 layers, 20 tokens over 4000: 83 us, 87 without)
    const bool again = __syncthreads_or(odd);
    if (FMT == KV_E4M3 || FMT == KV_E2M1 ? __builtin_expect(again, false) : again)
      for (int v = tb * TILE_KEYS; v < min(T, te * TILE_KEYS); ++v) {
        const int j = v < first ? v : v + gap;
        const bool see = (j <= own) & ((a.window == 0) | (j < a.sinks) | (j > own - a.window));
        if constexpr (FMT == KV_BF16) {
          const uint16_t *vrow = reinterpret_cast<const uint16_t *>(vbase + row_at(list[j]));
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const uint16_t y = vrow[32 * db + 8 * (k >> 2) + 4 * h2 + (k & 3)];
              o[db][k] += see && odd_low(y) ? Store<uint16_t>::ld(&y) : 0.f;
            }
        } else if constexpr (FMT == KV_E2M1) {
          const Off at = row_at(list[j]);
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const uint32_t byte = __float_as_uint(block_scale(at + 16 * db, 1)) >> 23;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const int ch = 32 * db + 8 * (k >> 2) + 4 * h2 + (k & 3);
              const uint32_t w4 = uint32_t(reinterpret_cast<const uint8_t *>(vbase + at)[ch / 2]) >> (4 * (ch & 1)) & 15u;
              if (see && e2m1_odd(w4, byte) != 0)
                o[db][k] += byte == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(0x7f800000u | w4 >> 3 << 31);
            }
          }
        } else if constexpr (FMT == KV_E4M3) {
          const Off at = row_at(list[j]);
          const float scale = scale_at(at).y;
          const bool any = no_power(scale);
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
              const uint32_t w4 = *reinterpret_cast<const uint32_t *>(vbase + at + (32 * db + 8 * i4 + 4 * h2));
              const uint2 y = any ? e4m3_times4(w4, scale) : e4m3_scaled4(w4, scale);
              const uint32_t z[4] = {y.x << 16, y.x & 0xffff0000u, y.y << 16, y.y & 0xffff0000u};
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                o[db][4 * i4 + i] += see && odd_high(z[i]) ? __uint_as_float(z[i]) : 0.f;
              }
            }
        } else {
          const float add = see && !(fabsf(scale_at(row_at(list[j])).y) < INFINITY) ? __uint_as_float(0x7fc00000u) : 0.f;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[db] += add;
        }
      }
  }
  lsum += __shfl_xor(lsum, 32, WAVE);
  if (row >= rows) return;
  if (nsplit == 1) {
    const float inv = own < 0 ? 0.f : 1.0f / lsum;             // nothing seen: zero
    IO *out = static_cast<IO *>(a.out) + q_at;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const int ch = 32 * db + 8 * i4 + 4 * h2;
        if constexpr (sizeof(IO) == 4) {
          *reinterpret_cast<float4 *>(out + ch) = make_float4(o[db][4 * i4] * inv, o[db][4 * i4 + 1] * inv,
                                                              o[db][4 * i4 + 2] * inv, o[db][4 * i4 + 3] * inv);
        } else {
          uint32_t u[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) u[i] = float_to_bf16_bits(o[db][4 * i4 + i] * inv);
          *reinterpret_cast<uint2 *>(out + ch) = make_uint2(u[0] | u[1] << 16, u[2] | u[3] << 16);
        }
      }
    return;
  }
  // split state, as the merge reads it: blocks of ROWS rows per (unit, block, split)
  const int64_t at = ((int64_t(unit) * blocks + rb) * nsplit + split) * ROWS + 32 * w + c;
  const int64_t parts = int64_t(units) * blocks * nsplit * ROWS;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4)
      *reinterpret_cast<float4 *>(a.ws + at * D + 32 * db + 8 * i4 + 4 * h2) =
          make_float4(o[db][4 * i4], o[db][4 * i4 + 1], o[db][4 * i4 + 2], o[db][4 * i4 + 3]);
  if (h2 == 0) *reinterpret_cast<float2 *>(a.ws + parts * D + at * 2) = make_float2(m, lsum);
}

template <int FMT, typename IO, int D, int NW>
static void go_tile(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  const int units = a.B * a.L * a.Hkv;
  KTimer kt_("k_attend_tile", st);
  const dim3 grid(unsigned((units + 7) / 8 * 8 * p.blocks * p.splits));
  const int64_t row = int64_t(a.Hkv) * kv_row_bytes(FMT, D);
  if (a.num_slots <= (1 << 24) && row < (1 << 24) && a.num_slots * row <= (int64_t(1) << 32))
    k_attend_tile<FMT, IO, D, NW, true><<<grid, 64 * NW, 0, st>>>(a, p.blocks, p.splits, units);
  else
    k_attend_tile<FMT, IO, D, NW, false><<<grid, 64 * NW, 0, st>>>(a, p.blocks, p.splits, units);
}

template <int FMT, typename IO>
static hipError_t go_tile_d(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  if constexpr (FMT == KV_E2M1 && sizeof(IO) == 2) a.D == 128 ? go_tile<FMT, IO, 128, 4>(a, p, st) : go_tile<FMT, IO, 64, 4>(a, p, st);
  else if (a.D == 128) p.rows == 256 ? go_tile<FMT, IO, 128, 8>(a, p, st) : go_tile<FMT, IO, 128, 4>(a, p, st);
  else p.rows == 256 ? go_tile<FMT, IO, 64, 8>(a, p, st) : go_tile<FMT, IO, 64, 4>(a, p, st);
  return p.splits > 1 ? launch_attend_merge(a, p, st) : hipGetLastError();
}

hipError_t launch_attend_tile(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  if (a.format == KV_BF16) return go_tile_d<KV_BF16, uint16_t>(a, p, st);
  if (a.format == KV_INT8) return a.io_f32 ? go_tile_d<KV_INT8, float>(a, p, st) : go_tile_d<KV_INT8, uint16_t>(a, p, st);
  if (a.format == KV_E4M3) return a.io_f32 ? go_tile_d<KV_E4M3, float>(a, p, st) : go_tile_d<KV_E4M3, uint16_t>(a, p, st);
  return a.io_f32 ? go_tile_d<KV_E2M1, float>(a, p, st) : go_tile_d<KV_E2M1, uint16_t>(a, p, st);
}

}  // namespace ikv
