// Attention of a session's newest tokens over its list of live slots, rows in bf16 or as
// 8-bit codes with scales, with an optional window and sinks.
#include <math.h>

#include "attend.hpp"
#include "ikv_internal.hpp"

namespace ikv {

// One workgroup per (token, layer and query head, session): blocks of 256 entries, a
// thread's entry's logit each, then the weighted values with a thread per channel.
template <int FMT, typename IO, int D>
__global__ void __launch_bounds__(256) k_attend_row(AttendArgs a) {
  __shared__ float qs[D], pw[256], red[4];
  __shared__ int64_t rows[256];
  const int b = blockIdx.z, l = blockIdx.y / a.Hq, h = blockIdx.y - l * a.Hq, g = h / (a.Hq / a.Hkv);
  const ikv_session s = a.sess[b];
  const int n = a.decode ? 1 : s.qe - s.qs, t = blockIdx.x;
  if (t >= n) return;
  int64_t before = 0;
  for (int i = 0; i < b; ++i) before += a.decode ? 1 : a.sess[i].qe - a.sess[i].qs;
  const int64_t at = before * a.L * a.Hq * D + ((int64_t(l) * a.Hq + h) * n + t) * D;
  const int tid = threadIdx.x;
  if (tid < D) qs[tid] = Store<IO>::ld(static_cast<const IO *>(a.q) + at + tid);
  __syncthreads();
  const int N = max(0, min(a.n_live[b], s.N)), own = N - n + t;
  const float scale = 1.0f / sqrtf(float(D));
  float m = -INFINITY, sum = 0.f, acc = 0.f;
  for (int j0 = 0; j0 <= own; j0 += 256) {
    const int j = j0 + tid;
    const bool seen = j <= own && (a.window == 0 || j < a.sinks || j > own - a.window);
    float x = -INFINITY, vs = 0.f;
    int64_t row = 0;
    if (seen) {
      row = (int64_t(l) * a.num_slots + a.live[s.slot_off + j]) * a.Hkv + g;
      float dot = 0.f;
      for (int d = 0; d < D; ++d) {
        float kd;
        if constexpr (FMT == KV_BF16) kd = Store<uint16_t>::ld(static_cast<const uint16_t *>(a.k) + row * D + d);
        else if constexpr (FMT == KV_INT8) kd = float(static_cast<const int8_t *>(a.k)[row * D + d]);
        else kd = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t *>(a.k)[row * D + d], 0);
        dot = fmaf(qs[d], kd, dot);
      }
      if constexpr (FMT != KV_BF16) {
        dot *= a.scales[row * 2];
        vs = a.scales[row * 2 + 1];
      } else vs = 1.f;
      x = dot * scale;
    }
    const float w = wave_max(x);
    if ((tid & 63) == 0) red[tid >> 6] = w;
    __syncthreads();
    const float mn = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), m);
    const float p = seen ? expf(x - mn) : 0.f;
    const float corr = m == -INFINITY ? 0.f : expf(m - mn);
    m = mn;
    pw[tid] = seen ? p * vs : 0.f;
    rows[tid] = seen ? row : -1;
    const float ws = wave_sum(p);
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = ws;
    __syncthreads();
    sum = sum * corr + (red[0] + red[1]) + (red[2] + red[3]);
    acc *= corr;
    if (tid < D)
      for (int i = 0; i < 256; ++i) {
        const int64_t r = rows[i];
        if (r < 0) continue;
        float vd;
        if constexpr (FMT == KV_BF16) vd = Store<uint16_t>::ld(static_cast<const uint16_t *>(a.v) + r * D + tid);
        else if constexpr (FMT == KV_INT8) vd = float(static_cast<const int8_t *>(a.v)[r * D + tid]);
        else vd = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t *>(a.v)[r * D + tid], 0);
        acc = fmaf(pw[i], vd, acc);
      }
    __syncthreads();
  }
  if (tid < D) static_cast<IO *>(a.out)[at + tid] = Store<IO>::from(own < 0 ? 0.f : acc / sum);
}

template <int FMT, typename IO>
static void launch_attend_d(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  const dim3 grid(unsigned(p.max_n), unsigned(a.L * a.Hq), unsigned(a.B));
  KTimer kt_("k_attend_row", st);
  if (a.D == 128) k_attend_row<FMT, IO, 128><<<grid, 256, 0, st>>>(a);
  else k_attend_row<FMT, IO, 64><<<grid, 256, 0, st>>>(a);
}

hipError_t launch_attend(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  if (p.few) return launch_attend_few(a, p, st);
  if (a.format == KV_BF16) launch_attend_d<KV_BF16, uint16_t>(a, p, st);
  else if (a.format == KV_INT8) a.io_f32 ? launch_attend_d<KV_INT8, float>(a, p, st) : launch_attend_d<KV_INT8, uint16_t>(a, p, st);
  else a.io_f32 ? launch_attend_d<KV_E4M3, float>(a, p, st) : launch_attend_d<KV_E4M3, uint16_t>(a, p, st);
  return hipGetLastError();
}

}  // namespace ikv
