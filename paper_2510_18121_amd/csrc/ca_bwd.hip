// Backward kernels: dQ, dK, dV of L = sum(dO * O) with P recomputed from the saved log-sum-exp
// (Section 2.1: P is not stored in forward, it is recomputed during backward).
//
//   prep : per (slot, head): -Delta = -<dO, O> and L2 = log2(e) * LSE, stored in SLOT order (the order of the
//          planner's per-document sorted query rows), so that both main kernels read them contiguously.
//          Padding slots get L2 = +huge, which makes their recomputed probabilities exactly 0.
//   dq   : one workgroup = one of the forward's work units (256 query slots x one query head, or 256/hp slots x hp
//          heads of one KV group), walking over the document's keys like the forward does.  Lane <-> query row:
//            S^T = K Q^T, dP^T = V dO^T, P^T = exp2(c S^T - L2), dS^T = P^T (dP^T - Delta),
//            dQ^T += K^T dS^T   (K^T through transposing LDS reads of the same K tile)
//   dkv  : one workgroup = 128 keys of one document x one KV head, walking over every block of 64 query
//          slots that can see them, for each query head of the group.  Lane <-> key:
//            S = Q K^T, dP = dO V^T (K, V fragments of the wave's 32 keys stay in registers),
//            dV^T += dO^T P, dK^T += Q^T dS   (Q^T, dO^T through transposing LDS reads)
//          dK and dV are written once, already summed over the group's heads and all tasks of the document.
//   joint: both kinds of workgroup in one launch, for batches that fill the chip with neither.
//   combine: adds up the fp32 partial results of units that the planner cut into pieces, in order, and stores them.
// All products are v_mfma_f32_16x16x32_bf16.  On N(0,1) operands the chip's power limit, not the matrix pipe, sets the rate, and
// this shape costs less energy per flop than 32x32x16 (alone 1928 against 1741 TFLOP/s).  Its price is twice the MFMA
// instructions, each about 9 cycles of the vector issue port (probe; an exponential 9, other vector instructions 4): 870 port
// cycles per 1024 matrix cycles in the dK/dV kernel, 726 per 768 in the dQ kernel.  32x32x16 -> 16x16x32 with everything else
// alike, 128K tokens of long and short documents in shuffled shards (32/8 heads, head_dim 128): dK/dV kernel 108.0 -> 104.2 ms,
// dQ kernel 82.2 -> 77.4 ms.
// No atomics and no fp32 dQ accumulation: the price is that S and dP are computed in both kernels (7 contractions
// instead of the minimal 5).  Results are deterministic.  All but small batches take five, in ca_bwd_fused.hip, with the same
// results.
#include <algorithm>
#include <atomic>

#include "ca_bwd_body.h"
#include "ca_device.h"
#include "ca_fused.h"
#include "ca_internal.h"
#include "ca_launch.h"

namespace ca {


__global__ void ca_bwd_prep_kernel(const int32_t *__restrict__ slot_row, const int32_t *__restrict__ block_rpk,
                                   const bf16_t *__restrict__ Q, const bf16_t *__restrict__ O,
                                   const bf16_t *__restrict__ dO, const float *__restrict__ LSE,
                                   float *__restrict__ delta_slot, float *__restrict__ l2_slot,
                                   float *__restrict__ stats_kv,
                                   bf16_t *__restrict__ q_sorted, bf16_t *__restrict__ do_sorted,
                                   u32x4 *__restrict__ zero, int64_t zero16, int64_t padded, int64_t total_q, int Hq, int G,
                                   int D) {
  // D/8 lanes per (slot, head): -Delta = -<dO, O> and log2(e)*LSE in slot order (for the dQ kernel), and for the
  // dK/dV kernel the slot-ordered copies of Q and dO as [block of 64 slots][head][64][D] - the 64-row tile of a
  // (block, head) is one contiguous run, and the tiles of the heads of a block follow each other - with the same two
  // statistics in the row order of those tiles (padding rows: zeros, with an LSE that makes every probability 0).
  // In a packed block (a document of at most rpk = 16 or 32 rows) tile t of a KV group holds the rows of the group's
  // heads 64/rpk t .. 64/rpk (t + 1) - 1, rpk rows each; the group's remaining tiles are neither written nor read.
  const int lanes = D / 8;
  const int64_t idx = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (idx < zero16) zero[idx] = u32x4{0, 0, 0, 0};
  const int64_t pair = idx / lanes;
  const int c = int(idx % lanes);
  const bool ok = pair < padded * Hq;
  const int64_t slot = ok ? pair / Hq : 0;
  const int h = int(pair % Hq);
  const int row = ok ? slot_row[slot] : -1;
  float s = 0.f;
  u32x4 qv = {0, 0, 0, 0}, dv = {0, 0, 0, 0};
  if (row >= 0) {
    const size_t off = (size_t(row) * Hq + h) * D + 8 * c;
    const bf16x8 a = *reinterpret_cast<const bf16x8 *>(O + off);
    const bf16x8 b = *reinterpret_cast<const bf16x8 *>(dO + off);
    qv = *reinterpret_cast<const u32x4 *>(Q + off);
    dv = __builtin_bit_cast(u32x4, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) s += float(a[i]) * float(b[i]);
  }
  for (int o = lanes / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (ok) {
    const float nd = row >= 0 ? -s : 0.f;  // stored negated: both kernels add it
    const float l2 = row >= 0 && c == 0 ? LSE[int64_t(h) * total_q + row] * LOG2E : L2_PADDING;
    const int64_t blk = slot / BWD_BQ;
    const int rpk = block_rpk[blk];
    int th = h, tr = int(slot % BWD_BQ);  // tile (as a head index) and row of this (slot, head) in the dK/dV tiles
    bool in_tile = true;
    if (rpk != 0) {
      const int hpk = BWD_BQ / rpk, hg = h % G;
      in_tile = tr < rpk;  // the slots beyond are padding of the document
      th = h - hg + hg / hpk;
      tr += (hg % hpk) * rpk;
    }
    if (in_tile) {
      const size_t so = ((size_t(blk) * Hq + th) * BWD_BQ + tr) * D + 8 * c;
      *reinterpret_cast<u32x4 *>(q_sorted + so) = qv;
      *reinterpret_cast<u32x4 *>(do_sorted + so) = dv;
    }
    if (c == 0) {
      delta_slot[int64_t(h) * padded + slot] = nd;
      l2_slot[int64_t(h) * padded + slot] = l2;
      if (in_tile) {
        float *const st = stats_kv + ((blk * Hq + th) * 2 + tr / 32) * 64 + tr % 32;
        st[0] = l2, st[32] = nd;
      }
    }
  }
}

__global__ void ca_fill_zero_kernel(u32x4 *__restrict__ p, int64_t n16) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < n16; i += stride) p[i] = u32x4{0, 0, 0, 0};
}

template <int D>
__global__ __launch_bounds__(512, 2) void ca_bwd_dq_kernel(const FwdUnit *__restrict__ units,
                                                           const int32_t *__restrict__ slot_row,
                                                           const int32_t *__restrict__ slot_pos,
                                                           const bf16_t *__restrict__ Q, const bf16_t *__restrict__ K,
                                                           const bf16_t *__restrict__ V, const bf16_t *__restrict__ dO,
                                                           const float *__restrict__ l2_slot,
                                                           const float *__restrict__ delta_slot,
                                                           bf16_t *__restrict__ dQ, float *__restrict__ parts, int Hq,
                                                           int Hkv, int64_t padded, float scale) {
  dq_workgroup<D, 8>(units[blockIdx.x], 0, slot_row, slot_pos, nullptr, 0, Q, K, V, dO, l2_slot, delta_slot, dQ, parts, Hq, Hkv, padded,
                     scale);
}

template <int D>
__global__ __launch_bounds__(256, 2) void ca_bwd_dkv_kernel(const BwdUnit *__restrict__ units,
                                                            const int32_t *__restrict__ slot_pos,
                                                            const bf16_t *__restrict__ Qs, const bf16_t *__restrict__ K,
                                                            const bf16_t *__restrict__ V, const bf16_t *__restrict__ dOs,
                                                            const float *__restrict__ stats_kv, bf16_t *__restrict__ dK,
                                                            bf16_t *__restrict__ dV, float *__restrict__ parts, int Hq, int Hkv,
                                                            float scale) {
  dkv_workgroup<D>(int(blockIdx.x), units, slot_pos, nullptr, nullptr, 0, Qs, K, V, dOs, stats_kv, dK, dV, parts, Hq, Hkv, scale);
}

// dK/dV units and dQ half units (workgroups of 4 groups of 32 rows) in one launch, longest first.  For batches too small to
// fill the chip with either kernel: what a launch takes there is mostly its fixed part, and the dQ work finds CUs that the
// dK/dV units leave idle.  Measured, backward, two launches against one: 49 -> 30 us (384 rows, 8/1 heads, head_dim 128), 31 -> 22 us
// (1.5K tokens, 4/2 heads, head_dim 64), 356 -> 315 us (16K tokens of documents of about 2K, 8/2 heads, where the two kernels' last
// units leave CUs idle one after the other).  Batches that fill the chip gain 1 or 2 % or lose as much, 4 % at head_dim 64: the
// planner decides by a simulation of both and a limit (JOINT_MAX_US).
struct JointArgs {
  const int32_t *order;  // what each workgroup does (ca_plan::joint_order), or nullptr
  const BwdUnit *units;
  const FwdUnit *dq_units;
  const int32_t *slot_row, *slot_pos, *pos_kv;
  const bf16_t *q, *k, *v, *d_o, *q_sorted, *do_sorted;
  const float *l2_slot, *delta_slot, *stats_kv;
  bf16_t *dq, *dk, *dv;
  float *parts_dq, *parts_kv;
  int n_dkv, n_dq, hq, hkv;
  int64_t padded;
  float scale;
};
template <int D>
__global__ __launch_bounds__(256, 2) void ca_bwd_joint_kernel(const JointArgs a) {
  const int i = int(blockIdx.x) - a.n_dkv;
  int w = int(blockIdx.x);
  if (a.order) {
    w = a.order[blockIdx.x];
  } else if (i >= 0) {
    // (all second halves before all first ones: 4.50 against 4.27 ms on lone 64-row shards with contexts, 312 against 298 us on 4K
    // tokens of documents of about 1K)
    int unit = i, half;
    half_of_unit(unit, a.n_dq, half);
    w = -1 - (unit + half * a.n_dq);
  }
  if (w >= 0) {
    dkv_workgroup<D>(w, a.units, a.pos_kv, nullptr, nullptr, 0, a.q_sorted, a.k, a.v, a.do_sorted, a.stats_kv, a.dk, a.dv, a.parts_kv, a.hq, a.hkv, a.scale);
  } else {
    const int half = -1 - w >= a.n_dq ? 1 : 0;
    dq_workgroup<D, 4>(a.dq_units[-1 - w - half * a.n_dq], half, a.slot_row, a.slot_pos, nullptr, 0, a.q, a.k, a.v, a.d_o, a.l2_slot,
                       a.delta_slot, a.dq, a.parts_dq, a.hq, a.hkv, a.padded, a.scale);
  }
}

// Adds up the pieces of the cut units: dQ of the forward / dQ units (from parts_dq; 8 groups of 32 rows), then dK and dV of
// the dK/dV units (from parts_kv; 4 groups of 32 keys, two tensors).  One workgroup per (unit, group, 64 columns); see
// combine_parts.
template <int D>
__global__ __launch_bounds__(256) void ca_combine_bwd_kernel(const CombineUnit *__restrict__ units_dq, int n_dq,
                                                             const CombineUnit *__restrict__ units_kv,
                                                             const int32_t *__restrict__ slot_row,
                                                             const float *__restrict__ parts_dq,
                                                             const float *__restrict__ parts_kv,
                                                             bf16_t *__restrict__ dQ, bf16_t *__restrict__ dK,
                                                             bf16_t *__restrict__ dV, int Hq, int Hkv, float scale) {
  constexpr int NH = D / 64;  // 64-column halves
  __shared__ __attribute__((aligned(16))) float lds[COMBINE_LDS];
  __shared__ float ml[4][64][2];
  const int un = blockIdx.x / (8 * NH), h = blockIdx.x % NH, pair = (blockIdx.x / NH) % 8;
  const bool kv = un >= n_dq;
  const CombineUnit u = kv ? units_kv[un - n_dq] : units_dq[un];
  const float *src = (kv ? parts_kv : parts_dq) + size_t(u.part0) * (FWD_BM * D) + pair * (32 * D) + h * (8 * 256);
  const int row = threadIdx.x >> 3;  // the row of the tile this lane stores
  bf16_t *dst;
  float f = scale;
  if (kv) {  // pair: (32 keys, dK or dV)
    const int key = 32 * (pair >> 1) + row;
    if (pair & 1) f = 1.f;
    dst = key < u.b ? ((pair & 1) ? dV : dK) + (size_t(u.a + key) * Hkv + u.c) * D + 64 * h : nullptr;
  } else {
    const int head = u.b + (pair & (u.c - 1));
    const int rw = slot_row[u.a + (pair >> __builtin_ctz(u.c)) * 32 + row];
    dst = rw >= 0 ? dQ + (size_t(rw) * Hq + head) * D + 64 * h : nullptr;
  }
  float m, l;
  combine_parts<false>(src, FWD_BM * D, nullptr, 0, u.n_parts, f, lds, ml, m, l,
                       [&](int) __attribute__((always_inline)) { return dst; });
}

static void launch_fill(void *p, size_t bytes, hipStream_t st) {
  if (bytes == 0) return;
  const int64_t n16 = int64_t(bytes / 16);
  const unsigned blocks = unsigned(std::min<int64_t>((n16 + 255) / 256, 256 * 32));
  hipLaunchKernelGGL(ca_fill_zero_kernel, dim3(blocks), dim3(256), 0, st, static_cast<u32x4 *>(p), n16);
}

void fill_uncovered(const ca_plan_t *p, void *dq, void *dk, void *dv, hipStream_t st) {
  if (!p->kv_covered) {
    launch_fill(dk, size_t(p->total_kv) * p->hkv * p->d * 2, st);
    launch_fill(dv, size_t(p->total_kv) * p->hkv * p->d * 2, st);
  }
  if (!p->q_covered) launch_fill(dq, size_t(p->total_q) * p->hq * p->d * 2, st);
}

static void prepare_bwd(const ca_plan_t *p, const void *q, const void *o, const void *d_o, const float *lse, void *dq, void *dk, void *dv,
                        void *ws, bool fused, hipStream_t st) {
  char *const at = static_cast<char *>(ws);
  const int64_t padded = int64_t(p->slot_row.size());
  fill_uncovered(p, dq, dk, dv, st);
  if (padded > 0) {
    const int64_t threads = padded * p->hq * (p->d / 8);
    hipLaunchKernelGGL(ca_bwd_prep_kernel, dim3(unsigned((threads + 255) / 256)), dim3(256), 0, st, p->d_slot_row,
                       p->d_block_rpk, static_cast<const bf16_t *>(q), static_cast<const bf16_t *>(o),
                       static_cast<const bf16_t *>(d_o), lse, reinterpret_cast<float *>(at), reinterpret_cast<float *>(at + p->ws_off_l2),
                       reinterpret_cast<float *>(at + p->ws_off_stats_kv), reinterpret_cast<bf16_t *>(at + p->ws_off_qs),
                       reinterpret_cast<bf16_t *>(at + p->ws_off_dos), reinterpret_cast<u32x4 *>(at + p->ws_off_flags),
                       fused ? int64_t(p->ws_bwd_fused - p->ws_off_flags) / 16 : int64_t(0), padded, p->total_q, p->hq, p->hq / p->hkv, p->d);
  }
}

void combine_dkv(const ca_plan_t *p, const float *parts, void *dk, void *dv, hipStream_t st) {
  const unsigned n = unsigned(p->bwd_combine.size() * 8 * (p->d / 64));
  hipLaunchKernelGGL(p->d == 128 ? ca_combine_bwd_kernel<128> : ca_combine_bwd_kernel<64>, dim3(n), dim3(256), 0, st, nullptr, 0,
                     p->d_bwd_combine, p->d_slot_row, nullptr, parts, nullptr, static_cast<bf16_t *>(dk), static_cast<bf16_t *>(dv), p->hq,
                     p->hkv, p->scale);
}

template <int D>
static hipError_t launch_bwd_t(const ca_plan_t *p, const void *q, const void *k, const void *v, const void *o,
                               const void *d_o, const float *lse, void *dq, void *dk, void *dv, void *ws,
                               bool split, bool fused, hipStream_t st, hipEvent_t *ev) {
  if (ev) (void)hipEventRecord(ev[0], st);
  const int64_t padded = int64_t(p->slot_row.size());
  float *delta_slot = static_cast<float *>(ws);
  float *l2_slot = reinterpret_cast<float *>(static_cast<char *>(ws) + p->ws_off_l2);
  float *stats_kv = reinterpret_cast<float *>(static_cast<char *>(ws) + p->ws_off_stats_kv);
  bf16_t *q_sorted = reinterpret_cast<bf16_t *>(static_cast<char *>(ws) + p->ws_off_qs);
  bf16_t *do_sorted = reinterpret_cast<bf16_t *>(static_cast<char *>(ws) + p->ws_off_dos);
  // partial results of cut units, where the caller's workspace has room for them
  float *const parts_kv = split && p->n_bwd_parts > 0 ? reinterpret_cast<float *>(static_cast<char *>(ws) + p->ws_off_parts_kv) : nullptr;
  float *const parts_dq = split && p->n_fwd_parts > 0 ? reinterpret_cast<float *>(static_cast<char *>(ws) + p->ws_off_parts_dq) : nullptr;
  const int32_t n_dkv = parts_kv ? p->bwd_piece_workgroups : p->bwd_workgroups;
  auto combine = [&](bool dq_units, bool kv_units) {
    const int c_dq = dq_units && parts_dq ? int(p->fwd_combine.size()) : 0, c_kv = kv_units && parts_kv ? int(p->bwd_combine.size()) : 0;
    if (c_dq + c_kv > 0)
      hipLaunchKernelGGL(ca_combine_bwd_kernel<D>, dim3(unsigned((c_dq + c_kv) * 8 * (D / 64))), dim3(256), 0, st,
                         p->d_fwd_combine, c_dq, p->d_bwd_combine, p->d_slot_row, parts_dq, parts_kv,
                         static_cast<bf16_t *>(dq), static_cast<bf16_t *>(dk), static_cast<bf16_t *>(dv), p->hq, p->hkv,
                         p->scale);
  };
  prepare_bwd(p, q, o, d_o, lse, dq, dk, dv, ws, fused, st);
  if (ev) (void)hipEventRecord(ev[1], st);
  if (fused) {
    FusedArgs a = {};
    a.units = p->d_fused_units;
    std::copy(p->fused_queue, p->fused_queue + N_XCD + 1, a.queue);
    a.slot_row = p->d_slot_row, a.pos_kv = p->d_pos_kv;
    a.k = static_cast<const bf16_t *>(k), a.v = static_cast<const bf16_t *>(v), a.q_sorted = q_sorted, a.do_sorted = do_sorted;
    a.stats_kv = stats_kv, a.flag_bytes = uint32_t(p->ws_off_ctrl - p->ws_off_flags);
    a.copy_bytes = uint32_t(p->ws_off_dos - p->ws_off_qs), a.dq_bytes = uint32_t(p->ws_off_flags - p->ws_off_dq_sums);
    a.dq = static_cast<bf16_t *>(dq), a.dk = static_cast<bf16_t *>(dk), a.dv = static_cast<bf16_t *>(dv);
    a.dq_sums = reinterpret_cast<float *>(static_cast<char *>(ws) + p->ws_off_dq_sums);
    a.flags = reinterpret_cast<int *>(static_cast<char *>(ws) + p->ws_off_flags);
    a.ctrl = reinterpret_cast<int *>(static_cast<char *>(ws) + p->ws_off_ctrl);
    a.hq = p->hq, a.hkv = p->hkv, a.scale = p->scale;
    hipError_t e = launch_bwd_fused(a, D, p->device, st);
    if (e != hipSuccess) return e;
    if (ev) (void)hipEventRecord(ev[2], st), (void)hipEventRecord(ev[3], st);
    return hipGetLastError();
  }
  const FwdUnit *const dq_list = parts_dq ? p->d_fwd_pieces : p->d_fwd_units;
  const int n_dq = int(parts_dq ? p->fwd_pieces.size() : p->fwd_units.size());
  const bool joint = p->joint && (split || p->n_fwd_parts + p->n_bwd_parts == 0);
  JointArgs args = {};
  auto launch_joint = [&](int32_t workgroups) {
    constexpr int SMEM = std::max(DkvSmem<D>::TOTAL, DqSmem<D, 4>::TOTAL);
    hipLaunchKernelGGL(ca_bwd_joint_kernel<D>, dim3(unsigned(workgroups)), dim3(256), SMEM, st, args);
  };
  if (joint) {
    auto kern = ca_bwd_joint_kernel<D>;
    constexpr int SMEM = std::max(DkvSmem<D>::TOTAL, DqSmem<D, 4>::TOTAL);
    static std::atomic<bool> done[16];
    hipError_t e = set_smem(kern, SMEM, p->device, done);
    if (e != hipSuccess) return e;
    args = {p->joint_order.empty() || ev ? nullptr : p->d_joint_order, parts_kv ? p->d_bwd_pieces : p->d_bwd_units, dq_list,
            p->d_slot_row, p->d_slot_pos, p->d_pos_kv, static_cast<const bf16_t *>(q), static_cast<const bf16_t *>(k),
            static_cast<const bf16_t *>(v), static_cast<const bf16_t *>(d_o), q_sorted, do_sorted, l2_slot, delta_slot, stats_kv,
            static_cast<bf16_t *>(dq), static_cast<bf16_t *>(dk), static_cast<bf16_t *>(dv), parts_dq, parts_kv,
            n_dkv, n_dq, p->hq, p->hkv, padded, p->scale};
    // (with timing enabled the same workgroups run as two launches, so that each kind has a time)
    launch_joint(ev ? n_dkv : n_dkv + 2 * n_dq);
  } else if (!p->bwd_units.empty()) {
    auto kern = ca_bwd_dkv_kernel<D>;
    constexpr int SMEM = DkvSmem<D>::TOTAL;
    static std::atomic<bool> done[16];
    hipError_t e = set_smem(kern, SMEM, p->device, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3(unsigned(n_dkv)), dim3(256), SMEM, st,
                       parts_kv ? p->d_bwd_pieces : p->d_bwd_units, p->d_pos_kv, q_sorted, static_cast<const bf16_t *>(k), static_cast<const bf16_t *>(v), do_sorted,
                       stats_kv, static_cast<bf16_t *>(dk), static_cast<bf16_t *>(dv), parts_kv, p->hq, p->hkv, p->scale);
  }
  if (p->shared_parts) combine(false, true);  // before the dQ pieces write over them
  if (ev) (void)hipEventRecord(ev[2], st);
  if (joint) {
    args.n_dkv = 0;  // dQ halves only
    if (ev) launch_joint(2 * n_dq);
  } else if (n_dq > 0) {
    auto kern = ca_bwd_dq_kernel<D>;
    constexpr int SMEM = DqSmem<D, 8>::TOTAL;
    static std::atomic<bool> done[16];
    hipError_t e = set_smem(kern, SMEM, p->device, done);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3(unsigned(n_dq)), dim3(512), SMEM, st, dq_list, p->d_slot_row, p->d_slot_pos,
                       static_cast<const bf16_t *>(q), static_cast<const bf16_t *>(k), static_cast<const bf16_t *>(v),
                       static_cast<const bf16_t *>(d_o), l2_slot, delta_slot, static_cast<bf16_t *>(dq), parts_dq, p->hq,
                       p->hkv, padded, p->scale);
  }
  combine(true, !p->shared_parts);
  if (ev) (void)hipEventRecord(ev[3], st);
  return hipGetLastError();
}

hipError_t launch_bwd(const ca_plan_t *p, const void *q, const void *k, const void *v, const void *o, const void *d_o,
                      const float *lse, void *dq, void *dk, void *dv, void *ws, bool split, bool fused,
                      hipStream_t st, hipEvent_t *ev) {
  return p->d == 128 ? launch_bwd_t<128>(p, q, k, v, o, d_o, lse, dq, dk, dv, ws, split, fused, st, ev)
                     : launch_bwd_t<64>(p, q, k, v, o, d_o, lse, dq, dk, dv, ws, split, fused, st, ev);
}

}  // namespace ca

