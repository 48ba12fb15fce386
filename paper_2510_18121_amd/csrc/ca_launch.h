// Launches and steps of launches that several sources share.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>

#include "ca_internal.h"

namespace ca {

// Zeros for gradients of rows that belong to no work unit (KV outside every scheduled document, Q rows outside every task).
void fill_uncovered(const ca_plan_t *p, void *dq, void *dk, void *dv, hipStream_t st);
// Adds up the pieces of dK/dV units.
void combine_dkv(const ca_plan_t *p, const float *parts, void *dk, void *dv, hipStream_t st);
hipError_t launch_fwd_window(const ca_plan_t *p, const void *q, const void *k, const void *v, void *o, float *lse, hipStream_t st);
hipError_t launch_bwd_window(const ca_plan_t *p, const void *q, const void *k, const void *v, const void *o, const void *d_o,
                             const float *lse, void *dq, void *dk, void *dv, void *ws, hipStream_t st, hipEvent_t *ev);

template <class F>
inline hipError_t set_smem(F kern, int bytes, int device, std::atomic<bool> *done) {
  // once per device; two threads that meet here both set the same value, which is harmless
  if (!done[device & 15].load(std::memory_order_acquire)) {
    hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    done[device & 15].store(true, std::memory_order_release);
  }
  return hipSuccess;
}

}  // namespace ca
