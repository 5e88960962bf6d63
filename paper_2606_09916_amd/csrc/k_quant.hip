// Rows between a pool (bf16 or float32) and the quantised cache, by slot lists.
//
// A row (one layer, slot and KV head; K or V) of D channels belongs to D / 8 adjacent
// lanes, 8 channels each.
// With a = max(max|x|, 2^-100):
//   int8  code = 127 x / a to the nearest whole number, ties to even, of the exact quotient.
//         bf16 rows often meet exact ties (x = a / 2 gives 63.5), where a product with a
//         rounded 127 / a would fall to either side. 127 / a is therefore held as a sum
//         hi + lo (error 2^-48 of it), so x hi + x lo, rounded once by the fused product, is
//         the nearest float32 to the quotient: exact at a tie (k + 1/2 has few bits), and
//         never moved onto one, because 254 x = (2k + 1) a cannot be missed by less than
//         2^-17 of itself with two 8-bit significands. float32 rows need the same in float64
//         (ties missed by no less than 2^-33).
//   e4m3  scale = 2^e with 448 2^e >= a > 224 2^e: x / scale is exact, and the conversion
//         rounds once.
//   e2m1  the same over the 32 channels of 4 lanes, with 7 2^e >= a > 7 2^(e - 1), e <= 125: the
//         conversion divides by 2^e, rounds once and holds what passes 6 there.
#include <type_traits>

#include "ikv_internal.hpp"
#include "kv_codes.hpp"
#include "quant_rows.hpp"

namespace ikv {

// PAST: a pool's rows, read or written, and the codes written pass the caches by, where there are more of
// them than the caches would keep for the call that comes next (quant_rows.hpp). Codes that are read never do:
// they may be there still, from the call that wrote them (so: 1021 rows read back in 30 us for 24).
typedef uint32_t u32x2_q __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_q __attribute__((ext_vector_type(4)));
template <bool PAST> __device__ __forceinline__ uint4 ld_row(const void *p) {
  if constexpr (!PAST) return *static_cast<const uint4 *>(p);
  const u32x4_q x = __builtin_nontemporal_load(static_cast<const u32x4_q *>(p));
  return make_uint4(x.x, x.y, x.z, x.w);
}
template <bool PAST> __device__ __forceinline__ void st_row(void *p, uint4 x) {
  if constexpr (PAST) __builtin_nontemporal_store(u32x4_q{x.x, x.y, x.z, x.w}, static_cast<u32x4_q *>(p));
  else *static_cast<uint4 *>(p) = x;
}
template <bool PAST> __device__ __forceinline__ void st_row(void *p, uint2 x) {
  if constexpr (PAST) __builtin_nontemporal_store(u32x2_q{x.x, x.y}, static_cast<u32x2_q *>(p));
  else *static_cast<uint2 *>(p) = x;
}
template <bool PAST> __device__ __forceinline__ void st_row(void *p, uint32_t x) {
  if constexpr (PAST) __builtin_nontemporal_store(x, static_cast<uint32_t *>(p));
  else *static_cast<uint32_t *>(p) = x;
}

template <typename T> struct Row8;               // 8 channels as loaded
template <> struct Row8<uint16_t> {
  uint4 w;
  template <bool PAST> __device__ __forceinline__ void ld(const uint16_t *p) { w = ld_row<PAST>(p); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
};
template <> struct Row8<float> {
  float4 a, b;
  template <bool PAST> __device__ __forceinline__ void ld(const float *p) {
    a = __builtin_bit_cast(float4, ld_row<PAST>(p));
    b = __builtin_bit_cast(float4, ld_row<PAST>(p + 4));
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
};

// The codes of this lane's 8 channels; amax the row's largest |x| as float bits.
template <typename T>
__device__ __forceinline__ uint2 quant8(const float (&x)[8], uint32_t amax_bits, int code, float *scale) {
  if (amax_bits >= 0x7f800000u) {                // an infinity or a NaN in the row
    *scale = __uint_as_float(0x7fc00000u);
    return make_uint2(0u, 0u);
  }
  const float a = fmaxf(__uint_as_float(amax_bits), 0x1p-100f);
  uint32_t w[2] = {0u, 0u};
  if (code == IKV_INT8) {
    *scale = a / 127.0f;
    if constexpr (sizeof(T) == 2) {
      const float hi = 127.0f / a, lo = fmaf(-hi, a, 127.0f) / a;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = int(rintf(fmaf(x[i], hi, x[i] * lo)));
        w[i >> 2] |= (uint32_t(c) & 255u) << (8 * (i & 3));
      }
    } else {
      const double ad = double(a), hi = 127.0 / ad, lo = fma(-hi, ad, 127.0) / ad;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double xd = double(x[i]);
        const int c = int(rint(fma(xd, hi, xd * lo)));
        w[i >> 2] |= (uint32_t(c) & 255u) << (8 * (i & 3));
      }
    }
  } else {
    // a = m 2^E, 1 <= m < 2, and 448 = 1.75 * 2^8: e = E - 8, one more where m > 1.75
    const uint32_t b = __float_as_uint(a);
    const int e = int(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    *scale = __uint_as_float(uint32_t(e + 127) << 23);
    const float inv = __uint_as_float(uint32_t(127 - e) << 23);        // e in [-108, 120]
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, 0, false);
      v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, v, true);
      w[i] = uint32_t(v);
    }
  }
  return make_uint2(w[0], w[1]);
}

// The same in 4 bits: 8 codes of a word; amax that of the block, *byte its scale.
__device__ __forceinline__ uint32_t quant8_e2m1(const float (&x)[8], uint32_t amax_bits, uint8_t *byte) {
  if (amax_bits >= 0x7f800000u) {
    *byte = 255;
    return 0u;
  }
  // a = m 2^E, 1 <= m < 2, and 7 = 1.75 * 2^2: e = E - 2, one more where m > 1.75
  const uint32_t b = __float_as_uint(fmaxf(__uint_as_float(amax_bits), 0x1p-100f));
  const int e = min(int(b >> 23) - 127 - 2 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0), 125);
  const float scale = __uint_as_float(uint32_t(e + 127) << 23);
  *byte = uint8_t(e + 127);
  uint32_t w = 0u;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

__device__ __forceinline__ int quant_rows(const ikv_session &s, const int32_t *n_rows, int b) {
  return n_rows ? max(0, min(n_rows[b], s.N)) : s.N;
}

// A workgroup takes `group` list entries of one layer at a time; an entry is `per` = Hkv D / 8 threads'
// work, a thread's 8 channels of its K and of its V row. A thread takes QU places at a time,
// all their slots loaded first, then all their rows: bound by memory, the kernels need that
// many bytes in flight per CU. 8192 rows of 36 layers x 8 heads, D = 128, bf16, E4M3: stored in
// 303 us (6.0 TB/s read and written), read back in 307 (6.0); 8189 in 4 bits 240 (6.4) and 258 (5.9).
// Both calls, 4 bits, with one place a thread 518, two 498, four 507, eight 589.

template <typename T, int D, bool FOUR, bool PAST>
__global__ void __launch_bounds__(QT) k_quant_store(const T *__restrict__ kpool, const T *__restrict__ vpool,
                                                    int64_t pool_slots, uint8_t *__restrict__ kc,
                                                    uint8_t *__restrict__ vc, void *__restrict__ scales,
                                                    int64_t num_slots, int Hkv, int code, int dead, int group,
                                                    const ikv_session *__restrict__ sess,
                                                    const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                                                    const int32_t *__restrict__ n_rows) {
  constexpr int LPR = D / 8;
  const int l = blockIdx.y, b = blockIdx.z, per = Hkv * LPR;
  const ikv_session s = sess[b];
  const int rows = quant_rows(s, n_rows, b);
  for (int k0 = blockIdx.x * group; k0 < rows; k0 += gridDim.x * group) {
    const int todo = quant_places(group, rows, k0, per);
    const int64_t e0 = s.slot_off + k0;
    for (int i0 = threadIdx.x; i0 < todo; i0 += QT * QU) {
      Row8<T> rk[QU], rv[QU];
      int64_t to[QU];
      int at[QU];                                    // place within the entry's row; -1: none
      int64_t from[QU];
#pragma unroll
      for (int u = 0; u < QU; ++u) {
        const int i = min(i0 + u * QT, todo - 1), k = i / per;
        const int64_t e = e0 + k;
        const int slot = dst[e];
        at[u] = i0 + u * QT < todo && slot != dead ? i - k * per : -1;
        to[u] = (int64_t(l) * num_slots + slot) * Hkv;
        from[u] = ((int64_t(l) * pool_slots + (src ? int64_t(src[e]) : e)) * Hkv) * D + (i - k * per) * 8;
      }
#pragma unroll
      for (int u = 0; u < QU; ++u)
        if (at[u] >= 0) {
          rk[u].template ld<PAST>(kpool + from[u]);
          rv[u].template ld<PAST>(vpool + from[u]);
        }
#pragma unroll
      for (int u = 0; u < QU; ++u) {
        if (at[u] < 0) continue;                     // the lanes of a row go together
        uint2 w[2];
        float sc[2];
        uint8_t byte[2];
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          float x[8];
          (kv ? rv[u] : rk[u]).get(x);
          uint32_t m = 0;                            // |x| as bits: ordered, a NaN above infinity
#pragma unroll
          for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
          for (int o = 1; o < (FOUR ? 4 : LPR); o <<= 1) m = max(m, uint32_t(__shfl_xor(int(m), o, WAVE)));
          if constexpr (FOUR) w[kv].x = quant8_e2m1(x, m, &byte[kv]);
          else w[kv] = quant8<T>(x, m, code, &sc[kv]);
        }
        const int64_t row = to[u] + at[u] / LPR;
        const int piece = at[u] % LPR;
        if constexpr (FOUR) {
          st_row<PAST>(kc + row * (D / 2) + piece * 4, w[0].x);
          st_row<PAST>(vc + row * (D / 2) + piece * 4, w[1].x);
          if (piece % 4 == 0) {
            uint8_t *p = static_cast<uint8_t *>(scales) + row * (D / 16) + piece / 4;
            p[0] = byte[0];
            p[D / 32] = byte[1];
          }
          continue;
        }
        st_row<PAST>(kc + row * D + piece * 8, w[0]);
        st_row<PAST>(vc + row * D + piece * 8, w[1]);
        if (piece == 0) reinterpret_cast<float2 *>(scales)[row] = make_float2(sc[0], sc[1]);
      }
    }
  }
}

// 8 codes of a word times their block's scale, exactly, to the pool's type.
template <bool PAST, typename T> __device__ __forceinline__ void put8_e2m1(T *o, uint32_t w, uint8_t byte) {
  const float scale = __uint_as_float(uint32_t(byte) << 23);           // 255: NaN
  if constexpr (sizeof(T) == 4) {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    st_row<PAST>(o, __builtin_bit_cast(uint4, make_float4(a[0], a[1], b[0], b[1])));
    st_row<PAST>(o + 4, __builtin_bit_cast(uint4, make_float4(c[0], c[1], d[0], d[1])));
  } else {
    st_row<PAST>(o, e2m1_scaled8(w, scale));
  }
}

// 8 codes times their scale, to the pool's type.
template <bool PAST, typename T> __device__ __forceinline__ void put8(T *o, uint2 w, float scale, int code) {
  const uint32_t u[2] = {w.x, w.y};
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int byte = int(u[i >> 2] >> (8 * (i & 3)));
    x[i] = (code == IKV_INT8 ? float(int8_t(byte)) : __builtin_amdgcn_cvt_f32_fp8(byte, 0)) * scale;
  }
  if constexpr (sizeof(T) == 4) {
    st_row<PAST>(o, __builtin_bit_cast(uint4, make_float4(x[0], x[1], x[2], x[3])));
    st_row<PAST>(o + 4, __builtin_bit_cast(uint4, make_float4(x[4], x[5], x[6], x[7])));
  } else {
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __bf16(x[i]);
    st_row<PAST>(o, __builtin_bit_cast(uint4, y));
  }
}

template <typename T, int D, bool FOUR, bool PAST>
__global__ void __launch_bounds__(QT) k_quant_load(const uint8_t *__restrict__ kc, const uint8_t *__restrict__ vc,
                                                   const void *__restrict__ scales, int64_t num_slots, int Hkv,
                                                   int code, int dead, int group, T *__restrict__ kpool,
                                                   T *__restrict__ vpool, int64_t pool_slots,
                                                   const ikv_session *__restrict__ sess,
                                                   const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                                                   const int32_t *__restrict__ n_rows) {
  constexpr int LPR = D / 8;
  const int l = blockIdx.y, b = blockIdx.z, per = Hkv * LPR;
  const ikv_session s = sess[b];
  const int rows = quant_rows(s, n_rows, b);
  for (int k0 = blockIdx.x * group; k0 < rows; k0 += gridDim.x * group) {
    const int todo = quant_places(group, rows, k0, per);
    const int64_t e0 = s.slot_off + k0;
    for (int i0 = threadIdx.x; i0 < todo; i0 += QT * QU) {
      uint2 wk[QU], wv[QU];
      float2 sc[QU];
      uint8_t bk[QU], bv[QU];
      int64_t to[QU], from[QU];
      bool on[QU];
#pragma unroll
      for (int u = 0; u < QU; ++u) {
        const int i = min(i0 + u * QT, todo - 1), k = i / per, at = i - k * per;
        const int64_t e = e0 + k;
        const int slot = src[e];
        on[u] = i0 + u * QT < todo && slot != dead;
        from[u] = (int64_t(l) * num_slots + slot) * per + at;                    // 8-code pieces
        to[u] = ((int64_t(l) * pool_slots + (dst ? int64_t(dst[e]) : e)) * per + at) * 8;
      }
#pragma unroll
      for (int u = 0; u < QU; ++u)
        if (on[u]) {
          if constexpr (FOUR) {
            wk[u].x = reinterpret_cast<const uint32_t *>(kc)[from[u]];
            wv[u].x = reinterpret_cast<const uint32_t *>(vc)[from[u]];
            const uint8_t *p = static_cast<const uint8_t *>(scales) + from[u] / LPR * (D / 16) + from[u] % LPR / 4;
            bk[u] = p[0];
            bv[u] = p[D / 32];
          } else {
            wk[u] = reinterpret_cast<const uint2 *>(kc)[from[u]];
            wv[u] = reinterpret_cast<const uint2 *>(vc)[from[u]];
            sc[u] = reinterpret_cast<const float2 *>(scales)[from[u] / LPR];
          }
        }
#pragma unroll
      for (int u = 0; u < QU; ++u)
        if (on[u] && FOUR) {
          put8_e2m1<PAST>(kpool + to[u], wk[u].x, bk[u]);
          put8_e2m1<PAST>(vpool + to[u], wv[u].x, bv[u]);
        } else if (on[u]) {
          put8<PAST>(kpool + to[u], wk[u], sc[u].x, code);
          put8<PAST>(vpool + to[u], wv[u], sc[u].y, code);
        }
    }
  }
}

static int quant_group(const ikv_quant_pool &c) { return quant_group(c.Hkv * (c.D / 8)); }
static dim3 quant_grid(const ikv_quant_pool &c, int B, int maxN, int most) {
  return dim3(unsigned(quant_groups(maxN, quant_group(c), int64_t(c.L) * B, most)), unsigned(c.L), unsigned(B));
}

static double quant_row_bytes(const ikv_quant_pool &c, const ikv_pool &p, int64_t rows) {
  return double(rows) * c.L * c.Hkv * c.D * (p.kv_dtype == IKV_BF16 ? 4 : 8);
}

// of(a channel, D, PAST) with these as types.
template <typename Of> static void quant_widths(bool bf16, bool d128, bool past, Of of) {
  auto with = [&](auto tag, auto d) { past ? of(tag, d, std::true_type()) : of(tag, d, std::false_type()); };
  auto wide = [&](auto tag) {
    d128 ? with(tag, std::integral_constant<int, 128>()) : with(tag, std::integral_constant<int, 64>());
  };
  bf16 ? wide(uint16_t()) : wide(float());
}

hipError_t launch_quant_store(const ikv_quant_pool &c, const ikv_pool &p, const ikv_session *sess_dev, int B, int maxN, int64_t rows,
                              const int32_t *src, const int32_t *dst, const int32_t *n_rows, hipStream_t st) {
  const dim3 grid = quant_grid(c, B, maxN, src ? QUANT_GRID : QUANT_GRID_NEW);
  const bool past = quant_row_bytes(c, p, rows) > QUANT_STORE_KEPT;
  KTimer kt_(past ? "k_quant_store<past>" : "k_quant_store", st);
  auto go = [&](auto tag, auto kernel) {
    using T = decltype(tag);
    kernel<<<grid, QT, 0, st>>>(static_cast<const T *>(p.k_pool), static_cast<const T *>(p.v_pool), p.num_slots,
                                static_cast<uint8_t *>(c.k_codes), static_cast<uint8_t *>(c.v_codes), c.scales,
                                c.num_slots, c.Hkv, c.code, c.dead_slot, quant_group(c), sess_dev, src, dst, n_rows);
  };
  auto of = [&](auto tag, auto d, auto by) {
    using T = decltype(tag);
    c.code == IKV_E2M1 ? go(tag, k_quant_store<T, d.value, true, by.value>) : go(tag, k_quant_store<T, d.value, false, by.value>);
  };
  quant_widths(p.kv_dtype == IKV_BF16, c.D == 128, past, of);
  return hipGetLastError();
}

hipError_t launch_quant_load(const ikv_quant_pool &c, const ikv_pool &p, const ikv_session *sess_dev, int B, int maxN, int64_t rows,
                             const int32_t *src, const int32_t *dst, const int32_t *n_rows, hipStream_t st) {
  const dim3 grid = quant_grid(c, B, maxN, QUANT_GRID);
  const bool past = quant_row_bytes(c, p, rows) > QUANT_LOAD_KEPT;
  KTimer kt_(past ? "k_quant_load<past>" : "k_quant_load", st);
  auto go = [&](auto tag, auto kernel) {
    using T = decltype(tag);
    kernel<<<grid, QT, 0, st>>>(static_cast<const uint8_t *>(c.k_codes), static_cast<const uint8_t *>(c.v_codes),
                                c.scales, c.num_slots, c.Hkv, c.code, c.dead_slot, quant_group(c), static_cast<T *>(p.k_pool),
                                static_cast<T *>(p.v_pool), p.num_slots, sess_dev, src, dst, n_rows);
  };
  auto of = [&](auto tag, auto d, auto by) {
    using T = decltype(tag);
    c.code == IKV_E2M1 ? go(tag, k_quant_load<T, d.value, true, by.value>) : go(tag, k_quant_load<T, d.value, false, by.value>);
  };
  quant_widths(p.kv_dtype == IKV_BF16, c.D == 128, past, of);
  return hipGetLastError();
}

}  // namespace ikv
