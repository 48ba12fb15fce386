// Core attention with a sliding window and sinks, over the tasks of a windowed plan: the kernels of ca_fwd_body.h and ca_bwd_body.h with
// a second bound of the mask and the tiles of a window instead of those of a prefix.
//
// A row at document position p sees the keys j <= min(p, kv_len - 1) with j > p - window or j < sinks:
//   P = softmax over these of scale Q K^T,  O = P V,  dV = P^T dO,  dS = P (dO V^T - <dO, O>),  dQ = scale dS K,  dK = scale dS^T Q.
// A row that sees nothing has O = 0, LSE = -inf, and no gradient.
#include <algorithm>
#include <atomic>

#include "ca_bwd_body.h"
#include "ca_device.h"
#include "ca_fwd_body.h"
#include "ca_internal.h"
#include "ca_launch.h"

namespace ca {

// Workgroups are always halves of units (128 rows, 32 positions of 4 heads of a group where it has so many): the registers do not
// hold whole units' four row groups and a mask of two bounds (328 spilled at head_dim 128), and a half spans the fewer keys.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void ca_fwd_window_kernel(
    const FwdUnit *__restrict__ units, int n_units, const int32_t *__restrict__ slot_row, const int32_t *__restrict__ slot_pos,
    const int32_t *__restrict__ slot_lo, int sinks, int short_rows, const bf16_t *__restrict__ Q, const bf16_t *__restrict__ K,
    const bf16_t *__restrict__ V, bf16_t *__restrict__ O, float *__restrict__ LSE, int Hq, int Hkv, int64_t total_q, float c) {
  fwd_workgroup<D, true, true>(units, n_units, 0, slot_row, slot_pos, slot_lo, sinks, short_rows, Q, K, V, O, LSE, nullptr, nullptr, Hq, Hkv,
                               total_q, c);
}

template <int D>
__global__ __launch_bounds__(512, 2) void ca_dq_window_kernel(const FwdUnit *__restrict__ units, const int32_t *__restrict__ slot_row,
                                                              const int32_t *__restrict__ slot_pos, const int32_t *__restrict__ slot_lo,
                                                              int sinks, const bf16_t *__restrict__ Q, const bf16_t *__restrict__ K,
                                                              const bf16_t *__restrict__ V, const bf16_t *__restrict__ dO,
                                                              const float *__restrict__ l2_slot, const float *__restrict__ delta_slot,
                                                              bf16_t *__restrict__ dQ, int Hq, int Hkv, int64_t padded, float scale) {
  dq_workgroup<D, 8, true>(units[blockIdx.x], 0, slot_row, slot_pos, slot_lo, sinks, Q, K, V, dO, l2_slot, delta_slot, dQ, nullptr, Hq, Hkv,
                           padded, scale);
}

template <int D>
__global__ __launch_bounds__(256, 2) void ca_dkv_window_kernel(const WindowUnit *__restrict__ units, const int32_t *__restrict__ slot_pos,
                                                               const int32_t *__restrict__ slot_lo, int sinks,
                                                               const bf16_t *__restrict__ Qs, const bf16_t *__restrict__ K,
                                                               const bf16_t *__restrict__ V, const bf16_t *__restrict__ dOs,
                                                               const float *__restrict__ stats_kv, bf16_t *__restrict__ dK,
                                                               bf16_t *__restrict__ dV, float *__restrict__ parts, int Hq, int Hkv,
                                                               float scale) {
  dkv_workgroup<D, true>(int(blockIdx.x), units, slot_pos, slot_lo, sinks, Qs, K, V, dOs, stats_kv, dK, dV, parts, Hq, Hkv, scale);
}

template <int D>
static hipError_t launch_fwd_window_t(const ca_plan_t *p, const void *q, const void *k, const void *v, void *o, float *lse, hipStream_t st) {
  if (p->fwd_units.empty()) return hipSuccess;
  auto kern = ca_fwd_window_kernel<D>;
  constexpr int SMEM = FwdSmem<D, true>::TOTAL;
  static std::atomic<bool> done[16];
  const hipError_t e = set_smem(kern, SMEM, p->device, done);
  if (e != hipSuccess) return e;
  const int n = int(p->fwd_units.size());
  hipLaunchKernelGGL(kern, dim3(unsigned(2 * n)), dim3(256), SMEM, st, p->d_fwd_units, n, p->d_slot_row, p->d_slot_pos, p->d_slot_lo, p->sinks,
                     int(p->window < FWD_BN), static_cast<const bf16_t *>(q), static_cast<const bf16_t *>(k), static_cast<const bf16_t *>(v),
                     static_cast<bf16_t *>(o), lse, p->hq, p->hkv, p->total_q, p->scale * LOG2E);
  return hipGetLastError();
}

hipError_t launch_fwd_window(const ca_plan_t *p, const void *q, const void *k, const void *v, void *o, float *lse, hipStream_t st) {
  return p->d == 128 ? launch_fwd_window_t<128>(p, q, k, v, o, lse, st) : launch_fwd_window_t<64>(p, q, k, v, o, lse, st);
}

template <int D>
static hipError_t launch_bwd_window_t(const ca_plan_t *p, const void *q, const void *k, const void *v, const void *o, const void *d_o,
                                      const float *lse, void *dq, void *dk, void *dv, void *ws, hipStream_t st, hipEvent_t *ev) {
  char *const at = static_cast<char *>(ws);
  const float *const delta_slot = reinterpret_cast<float *>(at), *const l2_slot = reinterpret_cast<float *>(at + p->ws_off_l2);
  const float *const stats_kv = reinterpret_cast<float *>(at + p->ws_off_stats_kv);
  const bf16_t *const q_sorted = reinterpret_cast<bf16_t *>(at + p->ws_off_qs), *const do_sorted = reinterpret_cast<bf16_t *>(at + p->ws_off_dos);
  float *const parts = reinterpret_cast<float *>(at + p->ws_off_parts_kv);
  if (ev) (void)hipEventRecord(ev[0], st);
  prepare_bwd(p, q, o, d_o, lse, dq, dk, dv, ws, false, st);
  if (ev) (void)hipEventRecord(ev[1], st);
  if (p->bwd_workgroups > 0) {
    auto kern = ca_dkv_window_kernel<D>;
    static std::atomic<bool> done[16];
    const hipError_t e = set_smem(kern, DkvSmem<D>::TOTAL, p->device, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3(unsigned(p->bwd_workgroups)), dim3(256), DkvSmem<D>::TOTAL, st, p->d_window_units, p->d_pos_kv, p->d_slot_lo,
                       p->sinks, q_sorted, static_cast<const bf16_t *>(k), static_cast<const bf16_t *>(v), do_sorted, stats_kv,
                       static_cast<bf16_t *>(dk), static_cast<bf16_t *>(dv), parts, p->hq, p->hkv, p->scale);
  }
  if (!p->bwd_combine.empty()) combine_dkv(p, parts, dk, dv, st);
  if (ev) (void)hipEventRecord(ev[2], st);
  if (!p->fwd_units.empty()) {
    auto kern = ca_dq_window_kernel<D>;
    static std::atomic<bool> done[16];
    constexpr int SMEM = DqSmem<D, 8>::TOTAL;
    const hipError_t e = set_smem(kern, SMEM, p->device, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3(unsigned(p->fwd_units.size())), dim3(512), SMEM, st, p->d_fwd_units, p->d_slot_row,
                       p->d_slot_pos, p->d_slot_lo, p->sinks, static_cast<const bf16_t *>(q), static_cast<const bf16_t *>(k),
                       static_cast<const bf16_t *>(v), static_cast<const bf16_t *>(d_o), l2_slot, delta_slot, static_cast<bf16_t *>(dq), p->hq,
                       p->hkv, int64_t(p->slot_row.size()), p->scale);
  }
  if (ev) (void)hipEventRecord(ev[3], st);
  return hipGetLastError();
}

hipError_t launch_bwd_window(const ca_plan_t *p, const void *q, const void *k, const void *v, const void *o, const void *d_o,
                             const float *lse, void *dq, void *dk, void *dv, void *ws, hipStream_t st, hipEvent_t *ev) {
  return p->d == 128 ? launch_bwd_window_t<128>(p, q, k, v, o, d_o, lse, dq, dk, dv, ws, st, ev)
                     : launch_bwd_window_t<64>(p, q, k, v, o, d_o, lse, dq, dk, dv, ws, st, ev);
}

}  // namespace ca
