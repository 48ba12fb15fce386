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
// 64K tokens, window 1024, 4 sinks, 32/8 heads of 128: 1.27 to 1.31 ms, 0.84 PFLOP/s of 4 D per (pair, head); 16K tokens, window 512, 16/16
// heads of 64: 75 us (80 with inputs that the last cache does not hold), 0.41.  Bound by vector instructions beside the MFMAs (at head_dim 128 the matrix pipe is busy 44 % of the time and vector
// instructions issue 50 %; 25 and 61 % at 64): 18 tiles per unit are few, and 2 to 4 of them are masked.
// At head_dim 64 four workgroups share a CU, with two stages of tiles and 128 registers a wave: 82 -> 75 us against three with three stages.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 4 : 2) void ca_fwd_window_kernel(
    const FwdUnit *__restrict__ units, int n_units, const int32_t *__restrict__ slot_row, const int32_t *__restrict__ slot_pos,
    const int32_t *__restrict__ slot_lo, int sinks, int short_rows, const bf16_t *__restrict__ Q, const bf16_t *__restrict__ K,
    const bf16_t *__restrict__ V, bf16_t *__restrict__ O, float *__restrict__ LSE, int Hq, int Hkv, int64_t total_q, float c) {
  fwd_workgroup<D, true, true>(units, n_units, 0, slot_row, slot_pos, slot_lo, sinks, short_rows, Q, K, V, O, LSE, nullptr, nullptr, Hq, Hkv,
                               total_q, c);
}

// -Delta = -<dO, O> and log2(e) * LSE of 64 slots and a head, by (head, slot) for dQ and in the order of dK/dV's tiles; rows of padding get
// probabilities of 0.  D / 8 lanes per row; the statistics leave through LDS as whole lines.  Bound by memory: 203 us, 5.4 TB/s, on the 64K tokens
// above (a workgroup per 64 slots and all heads, with the statistics stored as they came: 257 us).  O, which nothing else of the pass
// reads, passes the caches by (210 -> 200 us).
// O is the caller's, in bf16 (with shards of a merged row it is the whole row's), and Delta is what <dO, O> is with that: off by up to 2^-8 |dO| |O|.
// Where a row sees a few keys alone that is the largest of the roundings (relative error of dQ and dK: 0.0025 from windows of 16 keys
// on, 0.0027 with 6, 0.0036 with 2; 0.0017 is what rounding them to bf16 costs).
template <int D>
__global__ __launch_bounds__(256) void ca_window_prep_kernel(const int32_t *__restrict__ slot_row, const bf16_t *__restrict__ O,
                                                             const bf16_t *__restrict__ dO, const float *__restrict__ LSE,
                                                             float *__restrict__ delta_slot, float *__restrict__ l2_slot,
                                                             float *__restrict__ stats_kv, int64_t padded, int64_t total_q, int Hq) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES, N = BWD_BQ / ROWS;
  __shared__ float delta[BWD_BQ];
  const int64_t block = blockIdx.x / Hq;
  const int h = int(blockIdx.x - block * Hq), i0 = threadIdx.x / LANES, c = threadIdx.x % LANES;
  const int32_t *const rows = slot_row + block * BWD_BQ;
  bf16x8 a[N], b[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int row = max(0, rows[i0 + ROWS * n]);
    const size_t off = (size_t(row) * Hq + h) * D + 8 * c;
    a[n] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8 *>(O + off)), b[n] = *reinterpret_cast<const bf16x8 *>(dO + off);
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += float(a[n][i]) * float(b[n][i]);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (c == 0) delta[i0 + ROWS * n] = s;
  }
  __syncthreads();
  if (threadIdx.x >= BWD_BQ) return;
  const int i = threadIdx.x, row = rows[i];
  const float nd = row >= 0 ? -delta[i] : 0.f, l2 = row >= 0 ? LSE[int64_t(h) * total_q + row] * LOG2E : L2_PADDING;
  delta_slot[int64_t(h) * padded + block * BWD_BQ + i] = nd;
  l2_slot[int64_t(h) * padded + block * BWD_BQ + i] = l2;
  float *const st = stats_kv + ((block * Hq + h) * 2 + i / 32) * 64 + i % 32;
  st[0] = l2, st[32] = nd;
}

// dK/dV workgroups, then dQ workgroups (halves of units), in one launch: both are of four waves, two to a CU (three at head_dim 64), and
// the second kind fills the CUs that the first leaves idle.  64K tokens, window 1024, 4 sinks, 32/8 heads of 128: 3.78 ms, 0.72 PFLOP/s of
// 10 D per (pair, head), 1.0 of the 14 D that are executed (one after the other 3.86; 4K tokens of that kind 324 -> 232 us for the whole pass, with the
// cuts of ca_plan_window.h).  16K tokens, window 512, 16/16 heads of 64: 175 us, 0.43.  Bound by LDS latency, barriers and vector issue around the
// MFMAs, which are busy 54 % of the time (38 % at 64).
struct WindowArgs {
  const WindowUnit *units;
  const FwdUnit *dq_units;
  const int32_t *slot_row, *slot_pos, *slot_lo, *slot_src;
  const bf16_t *q, *k, *v, *d_o;
  const float *l2_slot, *delta_slot, *stats_kv;
  bf16_t *dq, *dk, *dv;
  float *parts;
  int n_dkv, n_dq, hq, hkv, sinks;
  int64_t padded;
  float scale;
};
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void ca_bwd_window_kernel(const WindowArgs a) {
  const int i = int(blockIdx.x);
  if (i < a.n_dkv) {
    dkv_workgroup<D, true>(i, a.units, a.slot_pos, a.slot_lo, a.slot_src, a.sinks, a.q, a.k, a.v, a.d_o, a.stats_kv, a.dk, a.dv, a.parts, a.hq,
                           a.hkv, a.scale);
  } else {
    int unit = i - a.n_dkv, half;
    half_of_unit(unit, a.n_dq, half);
    dq_workgroup<D, 4, true>(a.dq_units[unit], half, a.slot_row, a.slot_pos, a.slot_lo, a.sinks, a.q, a.k, a.v, a.d_o, a.l2_slot, a.delta_slot,
                             a.dq, nullptr, a.hq, a.hkv, a.padded, a.scale);
  }
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
  constexpr int SMEM = std::max(DkvSmem<D, true>::TOTAL, DqSmem<D, 4, true>::TOTAL);
  static_assert((D == 64 ? 3 : 2) * SMEM <= 160 * 1024, "as many workgroups to a CU as the registers allow");
  auto kern = ca_bwd_window_kernel<D>;
  static std::atomic<bool> done[16];
  const hipError_t e = set_smem(kern, SMEM, p->device, done);
  if (e != hipSuccess) return e;
  char *const at = static_cast<char *>(ws);
  auto in = [](const void *x) { return static_cast<const bf16_t *>(x); };
  auto out = [](void *x) { return static_cast<bf16_t *>(x); };
  WindowArgs a = {};
  a.units = p->d_window_units, a.dq_units = p->d_fwd_units, a.slot_row = p->d_slot_row, a.slot_pos = p->d_slot_pos, a.slot_lo = p->d_slot_lo, a.slot_src = p->d_slot_src;
  a.q = in(q), a.k = in(k), a.v = in(v), a.d_o = in(d_o);
  float *const delta_slot = reinterpret_cast<float *>(at), *const l2_slot = reinterpret_cast<float *>(at + p->ws_off_l2);
  float *const stats_kv = reinterpret_cast<float *>(at + p->ws_off_stats_kv);
  a.delta_slot = delta_slot, a.l2_slot = l2_slot, a.stats_kv = stats_kv;
  a.dq = out(dq), a.dk = out(dk), a.dv = out(dv), a.parts = reinterpret_cast<float *>(at + p->ws_off_parts_kv);
  a.hq = p->hq, a.hkv = p->hkv, a.sinks = p->sinks, a.padded = int64_t(p->slot_row.size()), a.scale = p->scale;
  auto launch = [&](int n_dkv, int n_dq) {
    a.n_dkv = n_dkv, a.n_dq = n_dq;
    if (n_dkv + n_dq > 0) hipLaunchKernelGGL(kern, dim3(unsigned(n_dkv + 2 * n_dq)), dim3(256), SMEM, st, a);
  };
  if (ev) (void)hipEventRecord(ev[0], st);
  fill_uncovered(p, dq, dk, dv, st);
  if (a.padded > 0) {
    hipLaunchKernelGGL(ca_window_prep_kernel<D>, dim3(unsigned(a.padded / BWD_BQ * a.hq)), dim3(256), 0, st, p->d_slot_row, in(o), in(d_o), lse, delta_slot,
                       l2_slot, stats_kv, a.padded, p->total_q, a.hq);
  }
  if (ev) (void)hipEventRecord(ev[1], st);
  const int n_dq = int(p->fwd_units.size());
  launch(p->bwd_workgroups, ev ? 0 : n_dq);  // (with timing enabled the same workgroups run as two launches, so that each kind has a time)
  if (!p->bwd_combine.empty()) combine_dkv(p, a.parts, dk, dv, st);
  if (ev) {
    (void)hipEventRecord(ev[2], st);
    launch(0, n_dq);
    (void)hipEventRecord(ev[3], st);
  }
  return hipGetLastError();
}

hipError_t launch_bwd_window(const ca_plan_t *p, const void *q, const void *k, const void *v, const void *o, const void *d_o,
                             const float *lse, void *dq, void *dk, void *dv, void *ws, hipStream_t st, hipEvent_t *ev) {
  return p->d == 128 ? launch_bwd_window_t<128>(p, q, k, v, o, d_o, lse, dq, dk, dv, ws, st, ev)
                     : launch_bwd_window_t<64>(p, q, k, v, o, d_o, lse, dq, dk, dv, ws, st, ev);
}

}  // namespace ca
