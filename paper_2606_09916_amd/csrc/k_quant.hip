// Rows between a pool (bf16 or float32) and the 8-bit cache, by slot lists.
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
#include "ikv_internal.hpp"
#include "quant_rows.hpp"

namespace ikv {

template <typename T> struct Row8;               // 8 channels as loaded
template <> struct Row8<uint16_t> {
  uint4 w;
  __device__ __forceinline__ void ld(const uint16_t *p) { w = *reinterpret_cast<const uint4 *>(p); }
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
  __device__ __forceinline__ void ld(const float *p) {
    a = reinterpret_cast<const float4 *>(p)[0];
    b = reinterpret_cast<const float4 *>(p)[1];
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

__device__ __forceinline__ int quant_rows(const ikv_session &s, const int32_t *n_rows, int b) {
  return n_rows ? max(0, min(n_rows[b], s.N)) : s.N;
}

// A workgroup takes `group` list entries of one layer; an entry is `per` = Hkv D / 8 threads'
// work, a thread's 8 channels of its K and of its V row. A thread takes QU places at a time,
// all their slots loaded first, then all their rows: bound by memory, the kernels need that
// many bytes in flight per CU. 8192 rows of 36 layers x 8 heads, D = 128, bf16, E4M3: stored in
// 350 us (5.2 TB/s read and written), read back in 311 (5.9); with one place a thread both took
// 1331, with eight 666.

template <typename T, int D>
__global__ void __launch_bounds__(QT) k_quant_store(const T *__restrict__ kpool, const T *__restrict__ vpool,
                                                    int64_t pool_slots, uint8_t *__restrict__ kc,
                                                    uint8_t *__restrict__ vc, float *__restrict__ scales,
                                                    int64_t num_slots, int Hkv, int code, int dead, int group,
                                                    const ikv_session *__restrict__ sess,
                                                    const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                                                    const int32_t *__restrict__ n_rows) {
  constexpr int LPR = D / 8;
  const int l = blockIdx.y, b = blockIdx.z, per = Hkv * LPR;
  const ikv_session s = sess[b];
  const int k0 = blockIdx.x * group;
  const int todo = quant_places(group, quant_rows(s, n_rows, b), k0, per);
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
        rk[u].ld(kpool + from[u]);
        rv[u].ld(vpool + from[u]);
      }
#pragma unroll
    for (int u = 0; u < QU; ++u) {
      if (at[u] < 0) continue;                     // the lanes of a row go together
      uint2 w[2];
      float sc[2];
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        float x[8];
        (kv ? rv[u] : rk[u]).get(x);
        uint32_t m = 0;                            // |x| as bits: ordered, a NaN above infinity
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) m = max(m, uint32_t(__shfl_xor(int(m), o, WAVE)));
        w[kv] = quant8<T>(x, m, code, &sc[kv]);
      }
      const int64_t row = to[u] + at[u] / LPR;
      const int piece = at[u] % LPR;
      *reinterpret_cast<uint2 *>(kc + row * D + piece * 8) = w[0];
      *reinterpret_cast<uint2 *>(vc + row * D + piece * 8) = w[1];
      if (piece == 0) reinterpret_cast<float2 *>(scales)[row] = make_float2(sc[0], sc[1]);
    }
  }
}

// 8 codes times their scale, to the pool's type.
template <typename T> __device__ __forceinline__ void put8(T *o, uint2 w, float scale, int code) {
  const uint32_t u[2] = {w.x, w.y};
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int byte = int(u[i >> 2] >> (8 * (i & 3)));
    x[i] = (code == IKV_INT8 ? float(int8_t(byte)) : __builtin_amdgcn_cvt_f32_fp8(byte, 0)) * scale;
  }
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4 *>(o)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(o)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    bf16x8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __bf16(x[i]);
    *reinterpret_cast<bf16x8 *>(o) = y;
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(QT) k_quant_load(const uint8_t *__restrict__ kc, const uint8_t *__restrict__ vc,
                                                   const float *__restrict__ scales, int64_t num_slots, int Hkv,
                                                   int code, int dead, int group, T *__restrict__ kpool,
                                                   T *__restrict__ vpool, int64_t pool_slots,
                                                   const ikv_session *__restrict__ sess,
                                                   const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                                                   const int32_t *__restrict__ n_rows) {
  constexpr int LPR = D / 8;
  const int l = blockIdx.y, b = blockIdx.z, per = Hkv * LPR;
  const ikv_session s = sess[b];
  const int k0 = blockIdx.x * group;
  const int todo = quant_places(group, quant_rows(s, n_rows, b), k0, per);
  const int64_t e0 = s.slot_off + k0;
  for (int i0 = threadIdx.x; i0 < todo; i0 += QT * QU) {
    uint2 wk[QU], wv[QU];
    float2 sc[QU];
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
        wk[u] = reinterpret_cast<const uint2 *>(kc)[from[u]];
        wv[u] = reinterpret_cast<const uint2 *>(vc)[from[u]];
        sc[u] = reinterpret_cast<const float2 *>(scales)[from[u] / LPR];
      }
#pragma unroll
    for (int u = 0; u < QU; ++u)
      if (on[u]) {
        put8(kpool + to[u], wk[u], sc[u].x, code);
        put8(vpool + to[u], wv[u], sc[u].y, code);
      }
  }
}

static int quant_group(const ikv_quant_pool &c) { return quant_group(c.Hkv * (c.D / 8)); }
static dim3 quant_grid(const ikv_quant_pool &c, int B, int maxN) {
  return dim3(unsigned(cdiv(maxN, quant_group(c))), unsigned(c.L), unsigned(B));
}

hipError_t launch_quant_store(const ikv_quant_pool &c, const ikv_pool &p, const ikv_session *sess_dev, int B, int maxN,
                              const int32_t *src, const int32_t *dst, const int32_t *n_rows, hipStream_t st) {
  const dim3 grid = quant_grid(c, B, maxN);
  KTimer kt_("k_quant_store<T, D>", st);
  auto go = [&](auto tag, auto kernel) {
    using T = decltype(tag);
    kernel<<<grid, QT, 0, st>>>(static_cast<const T *>(p.k_pool), static_cast<const T *>(p.v_pool), p.num_slots,
                                static_cast<uint8_t *>(c.k_codes), static_cast<uint8_t *>(c.v_codes), c.scales,
                                c.num_slots, c.Hkv, c.code, c.dead_slot, quant_group(c), sess_dev, src, dst, n_rows);
  };
  if (p.kv_dtype == IKV_BF16) c.D == 128 ? go(uint16_t(), k_quant_store<uint16_t, 128>) : go(uint16_t(), k_quant_store<uint16_t, 64>);
  else c.D == 128 ? go(float(), k_quant_store<float, 128>) : go(float(), k_quant_store<float, 64>);
  return hipGetLastError();
}

hipError_t launch_quant_load(const ikv_quant_pool &c, const ikv_pool &p, const ikv_session *sess_dev, int B, int maxN,
                             const int32_t *src, const int32_t *dst, const int32_t *n_rows, hipStream_t st) {
  const dim3 grid = quant_grid(c, B, maxN);
  KTimer kt_("k_quant_load<T, D>", st);
  auto go = [&](auto tag, auto kernel) {
    using T = decltype(tag);
    kernel<<<grid, QT, 0, st>>>(static_cast<const uint8_t *>(c.k_codes), static_cast<const uint8_t *>(c.v_codes),
                                c.scales, c.num_slots, c.Hkv, c.code, c.dead_slot, quant_group(c), static_cast<T *>(p.k_pool),
                                static_cast<T *>(p.v_pool), p.num_slots, sess_dev, src, dst, n_rows);
  };
  if (p.kv_dtype == IKV_BF16) c.D == 128 ? go(uint16_t(), k_quant_load<uint16_t, 128>) : go(uint16_t(), k_quant_load<uint16_t, 64>);
  else c.D == 128 ? go(float(), k_quant_load<float, 128>) : go(float(), k_quant_load<float, 64>);
  return hipGetLastError();
}

}  // namespace ikv
