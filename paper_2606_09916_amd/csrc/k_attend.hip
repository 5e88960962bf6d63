// The merge of splits, shared by the attention kernels of one row block and of many.
#include "attend.hpp"
#include "ikv_internal.hpp"

namespace ikv {

// Row blocks of `rows` rows per (unit = session, layer, KV head; block; split). The splits of
// a row: with M their largest reference, sum_z o_z 2^(m_z - M) over sum_z l_z 2^(m_z - M); a
// split that saw nothing has m = -inf and weighs zero.
template <typename IO, int D>
__global__ void __launch_bounds__(D) k_attend_merge(AttendArgs a, int nsplit, int rows) {
  __shared__ float sm[DEC_MAX_SPLITS], sl[DEC_MAX_SPLITS];
  const int u = blockIdx.x, blk = blockIdx.z, r = blockIdx.y;
  const int hkv = u % a.Hkv, l = u / a.Hkv % a.L, b = u / a.Hkv / a.L;
  const ikv_session s = a.sess[b];
  const int n = a.decode ? 1 : s.qe - s.qs, G = a.Hq / a.Hkv, R = blk * rows + r;
  if (R >= n * G) return;
  int64_t before = 0;
  if (a.decode) before = b;
  else
    for (int i = 0; i < b; ++i) before += a.sess[i].qe - a.sess[i].qs;
  const int d = threadIdx.x;
  const int64_t part = (int64_t(u) * gridDim.z + blk) * nsplit * rows + r;
  const int64_t parts = int64_t(gridDim.x) * gridDim.z * nsplit * rows;
  if (d < nsplit) {
    const float2 x = *reinterpret_cast<const float2 *>(a.ws + parts * D + (part + int64_t(d) * rows) * 2);
    sm[d] = x.x;
    sl[d] = x.y;
  }
  __syncthreads();
  float M = -INFINITY;
  for (int z = 0; z < nsplit; ++z) M = fmaxf(M, sm[z]);
  float acc = 0.f, sum = 0.f;
  if (M != -INFINITY)
#pragma unroll 8
    for (int z = 0; z < nsplit; ++z) {
      const float x = a.ws[(part + int64_t(z) * rows) * D + d];
      const float f = sm[z] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[z] - M);
      acc = fmaf(x, f, acc);
      sum = fmaf(sl[z], f, sum);
    }
  const int t = R / G, h = R - t * G;
  const int64_t at = before * a.L * a.Hq * D + ((int64_t(l) * a.Hq + hkv * G + h) * n + t) * D + d;
  static_cast<IO *>(a.out)[at] = Store<IO>::from(M == -INFINITY ? 0.f : acc / sum);
}

hipError_t launch_attend_merge(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  KTimer kt_("k_attend_merge", st);
  const dim3 grid(unsigned(a.B * a.L * a.Hkv), unsigned(p.rows), unsigned(p.blocks));
  if (a.D == 128)
    a.io_f32 ? k_attend_merge<float, 128><<<grid, 128, 0, st>>>(a, p.splits, p.rows)
             : k_attend_merge<uint16_t, 128><<<grid, 128, 0, st>>>(a, p.splits, p.rows);
  else
    a.io_f32 ? k_attend_merge<float, 64><<<grid, 64, 0, st>>>(a, p.splits, p.rows)
             : k_attend_merge<uint16_t, 64><<<grid, 64, 0, st>>>(a, p.splits, p.rows);
  return hipGetLastError();
}

hipError_t launch_attend(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  return p.few ? launch_attend_few(a, p, st) : launch_attend_tile(a, p, st);
}

}  // namespace ikv
