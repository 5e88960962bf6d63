// The merge of splits, shared by the attention kernels of one row block and of many.
#include "attend.hpp"
#include "ikv_internal.hpp"

namespace ikv {

// Row blocks of `rows` rows per (unit = session, layer, KV head; block; split). The splits of
// a row: with M their largest reference, sum_z o_z 2^(m_z - M) over sum_z l_z 2^(m_z - M); a
// split that saw nothing has m = -inf and weighs zero. A thread takes 4 channels of a row, a
// workgroup 1024 / D rows: bound by reading the state once.
constexpr int MERGE_THREADS = 256;

template <typename IO, int D>
__global__ void __launch_bounds__(MERGE_THREADS) k_attend_merge(AttendArgs a, int nsplit, int rows) {
  constexpr int TPR = D / 4;
  const int u = blockIdx.x, blk = blockIdx.z;
  const int r = blockIdx.y * (MERGE_THREADS / TPR) + threadIdx.x / TPR, d = threadIdx.x % TPR * 4;
  const int hkv = u % a.Hkv, l = u / a.Hkv % a.L, b = u / a.Hkv / a.L;
  const ikv_session s = a.sess[b];
  const int n = a.decode ? 1 : s.qe - s.qs, G = a.Hq / a.Hkv, R = blk * rows + r;
  if (r >= rows || R >= n * G) return;
  int64_t before = 0;
  if (a.decode) before = b;
  else
    for (int i = 0; i < b; ++i) before += a.sess[i].qe - a.sess[i].qs;
  const int64_t part = (int64_t(u) * gridDim.z + blk) * nsplit * rows + r;
  const int64_t parts = int64_t(gridDim.x) * gridDim.z * nsplit * rows;
  const float2 *ml = reinterpret_cast<const float2 *>(a.ws + parts * D) + part;
  float M = -INFINITY;
  for (int z = 0; z < nsplit; ++z) M = fmaxf(M, ml[int64_t(z) * rows].x);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
#pragma unroll 4
  for (int z = 0; z < nsplit; ++z) {
    const float4 x = *reinterpret_cast<const float4 *>(a.ws + (part + int64_t(z) * rows) * D + d);
    const float2 y = ml[int64_t(z) * rows];
    const float f = y.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(y.x - M);
    acc.x = fmaf(x.x, f, acc.x);
    acc.y = fmaf(x.y, f, acc.y);
    acc.z = fmaf(x.z, f, acc.z);
    acc.w = fmaf(x.w, f, acc.w);
    sum = fmaf(y.y, f, sum);
  }
  const int t = R / G, h = R - t * G;
  const bool sees = max(0, min(a.n_live[b], s.N)) - n + t >= 0;
  const float inv = sees ? 1.0f / sum : 0.f;                 // nothing seen: zero
  IO *o = static_cast<IO *>(a.out) + before * a.L * a.Hq * D + ((int64_t(l) * a.Hq + hkv * G + h) * n + t) * D + d;
  if constexpr (sizeof(IO) == 4) *reinterpret_cast<float4 *>(o) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  else {
    const uint32_t lo = float_to_bf16_bits(acc.x * inv) | uint32_t(float_to_bf16_bits(acc.y * inv)) << 16;
    const uint32_t hi = float_to_bf16_bits(acc.z * inv) | uint32_t(float_to_bf16_bits(acc.w * inv)) << 16;
    *reinterpret_cast<uint2 *>(o) = make_uint2(lo, hi);
  }
}

template <typename IO, int D>
static void go_merge(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  constexpr int per = MERGE_THREADS / (D / 4);
  const dim3 grid(unsigned(a.B * a.L * a.Hkv), unsigned((p.rows + per - 1) / per), unsigned(p.blocks));
  k_attend_merge<IO, D><<<grid, MERGE_THREADS, 0, st>>>(a, p.splits, p.rows);
}

hipError_t launch_attend_merge(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  KTimer kt_("k_attend_merge", st);
  if (a.D == 128) a.io_f32 ? go_merge<float, 128>(a, p, st) : go_merge<uint16_t, 128>(a, p, st);
  else a.io_f32 ? go_merge<float, 64>(a, p, st) : go_merge<uint16_t, 64>(a, p, st);
  return hipGetLastError();
}

hipError_t launch_attend(const AttendArgs &a, const AttendPlan &p, hipStream_t st) {
  return p.few ? launch_attend_few(a, p, st) : launch_attend_tile(a, p, st);
}

}  // namespace ikv
