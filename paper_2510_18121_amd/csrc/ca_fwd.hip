// The forward kernel's launches, and the kernel that adds up the partial results of units cut into pieces.  What a workgroup does,
// and why so: ca_fwd_body.h.
#include <atomic>
#include <type_traits>

#include "ca_device.h"
#include "ca_fwd_body.h"
#include "ca_internal.h"

namespace ca {

template <int D, bool HALVES>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void ca_fwd_kernel(const FwdUnit *__restrict__ units, int n_units, int turns,
                                                                   const int32_t *__restrict__ slot_row,
                                                                   const int32_t *__restrict__ slot_pos,
                                                                   const bf16_t *__restrict__ Q,
                                                                   const bf16_t *__restrict__ K,
                                                                   const bf16_t *__restrict__ V, bf16_t *__restrict__ O,
                                                                   float *__restrict__ LSE, float *__restrict__ parts,
                                                                   float *__restrict__ stats, int Hq, int Hkv,
                                                                   int64_t total_q, float c /* scale * log2(e) */) {
  fwd_workgroup<D, HALVES, false>(units, n_units, turns, slot_row, slot_pos, nullptr, 0, 0, Q, K, V, O, LSE, parts, stats, Hq, Hkv,
                                  total_q, c);
}

// Adds up the pieces of the cut units: O = sum_i 2^(m_i - M) acc_i / sum_i 2^(m_i - M) l_i with M = max_i m_i, and LSE.
// One workgroup per (unit, group of 32 rows, 64 columns); see combine_parts.
template <int D>
__global__ __launch_bounds__(256) void ca_combine_fwd_kernel(const CombineUnit *__restrict__ units,
                                                             const int32_t *__restrict__ slot_row,
                                                             const float *__restrict__ parts,
                                                             const float *__restrict__ stats, bf16_t *__restrict__ O,
                                                             float *__restrict__ LSE, int Hq, int64_t total_q) {
  constexpr int NH = D / 64;  // 64-column halves
  __shared__ __attribute__((aligned(16))) float lds[COMBINE_LDS];
  __shared__ float ml[4][64][2];
  const CombineUnit u = units[blockIdx.x / (8 * NH)];
  const int h = blockIdx.x % NH, pair = (blockIdx.x / NH) % 8;
  const int head = u.b + (pair & (u.c - 1));
  const int32_t *const rows = slot_row + u.a + (pair >> __builtin_ctz(u.c)) * 32;
  const int row = rows[threadIdx.x & 31], orow = rows[threadIdx.x >> 3];  // of the lane's row, and of the row it stores
  float m = 0.f, l = 0.f;
  combine_parts<true>(parts + size_t(u.part0) * (FWD_BM * D) + pair * (32 * D) + h * (8 * 256), FWD_BM * D,
                      stats + (size_t(u.part0) * 8 + pair) * 128, 8 * 128, u.n_parts, 1.f, lds, ml, m, l,
                      [&](int) __attribute__((always_inline)) -> bf16_t * {
                        return orow >= 0 ? O + (size_t(orow) * Hq + head) * D + 64 * h : nullptr;
                      });
  if (h == 0 && threadIdx.x < 32 && row >= 0) LSE[size_t(head) * total_q + row] = 0.6931471805599453f * (m + fast_log2(l));
}

template <int D>
static hipError_t launch_fwd_t(const ca_plan_t *p, const void *q, const void *k, const void *v, void *o, float *lse,
                               void *parts, hipStream_t st) {
  if (p->fwd_units.empty()) return hipSuccess;
  const float c = p->scale * 1.4426950408889634f;
  float *const pp = static_cast<float *>(parts);
  float *const stats = pp ? pp + size_t(p->n_fwd_parts) * (FWD_BM * D) : nullptr;
  const size_t n = pp ? p->fwd_pieces.size() : p->fwd_units.size();
  const FwdForm form = pp ? p->fwd_piece_form : p->fwd_form;
  auto launch = [&](auto halves) {
    constexpr bool HALVES = decltype(halves)::value;
    auto kern = ca_fwd_kernel<D, HALVES>;
    constexpr int SMEM = FwdSmem<D>::TOTAL;
    static std::atomic<bool> attr_done[16];  // once per device; a second thread repeating the call is harmless
    if (!attr_done[p->device & 15].load(std::memory_order_acquire)) {
      hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, SMEM);
      if (e != hipSuccess) return e;
      attr_done[p->device & 15].store(true, std::memory_order_release);
    }
    hipLaunchKernelGGL(kern, dim3(unsigned(HALVES ? 2 * n : n)), dim3(256), SMEM, st, pp ? p->d_fwd_pieces : p->d_fwd_units, int(n),
                       int(form.turns), p->d_slot_row, p->d_slot_pos, static_cast<const bf16_t *>(q), static_cast<const bf16_t *>(k),
                       static_cast<const bf16_t *>(v), static_cast<bf16_t *>(o), lse, pp, stats, p->hq, p->hkv, p->total_q, c);
    return hipSuccess;
  };
  const hipError_t launched = form.halves ? launch(std::true_type{}) : launch(std::false_type{});
  if (launched != hipSuccess) return launched;
  if (pp) {
    hipLaunchKernelGGL(ca_combine_fwd_kernel<D>, dim3(unsigned(p->fwd_combine.size() * 8 * (D / 64))), dim3(256), 0, st,
                       p->d_fwd_combine, p->d_slot_row, pp, stats, static_cast<bf16_t *>(o), lse, p->hq, p->total_q);
  }
  return hipGetLastError();
}

hipError_t launch_fwd(const ca_plan_t *p, const void *q, const void *k, const void *v, void *o, float *lse, void *parts,
                      hipStream_t st) {
  return p->d == 128 ? launch_fwd_t<128>(p, q, k, v, o, lse, parts, st) : launch_fwd_t<64>(p, q, k, v, o, lse, parts, st);
}

}  // namespace ca
