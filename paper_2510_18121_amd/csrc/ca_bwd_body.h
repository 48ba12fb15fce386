// What the workgroups of the backward kernels of dQ and of dK and dV do (see ca_bwd.hip for what these are).
#pragma once
#include <type_traits>

#include "ca_device.h"
#include "ca_internal.h"

namespace ca {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float L2_PADDING = 1.0e30f;  // exp2(x - 1e30) == 0 for every finite score

// ------------------------------------------------------------------------------------------------ dQ
// Eight waves on a CU of their own have four stages; workgroups of four, two to a CU, share its LDS.
template <int D, int W, bool WINDOW = false>
struct DqSmem {
  static constexpr int NST = D == 128 && W == 4 ? 2 : WINDOW ? 3 : 4;
  static constexpr int TILE = FWD_BN * 2 * D;
  // a stage holds the K tile and then the V tile of one key block: both are reached from one address register
  // through the 16-bit offset field of the LDS instructions
  static constexpr int K_OFF = 0;
  static constexpr int V_OFF = TILE;
  static constexpr int STAGE = 2 * TILE;
  static constexpr int TOTAL = NST * STAGE;
};

// The workgroup of W waves: all eight 32-row groups of the unit (W = 8), or groups 4 half .. 4 half + 3 of them.  Both do the same
// arithmetic in the same order, so dQ does not depend on which of them computes it.
// The order of a 32-key block is written out: its fragments are fetched AHEAD of the MFMAs that use them through a ring of
// registers, the exponentials go between the MFMAs of dP, and fences keep the compiler from bunching either.  Left to the
// compiler, the same arithmetic waited for LDS in every pair of dQ's MFMAs: 77.3 -> 74.8 ms (128K tokens, 32/8 heads).
// WINDOW: as in the forward kernel.
template <int D, int W, bool WINDOW = false>
__device__ __forceinline__ void dq_workgroup(const FwdUnit &u, const int half, const int32_t *__restrict__ slot_row,
                                             const int32_t *__restrict__ slot_pos, const int32_t *__restrict__ slot_lo, const int sinks,
                                             const bf16_t *__restrict__ Q,
                                             const bf16_t *__restrict__ K, const bf16_t *__restrict__ V,
                                             const bf16_t *__restrict__ dO, const float *__restrict__ l2_slot,
                                             const float *__restrict__ delta_slot, bf16_t *__restrict__ dQ,
                                             float *__restrict__ parts, int Hq, int Hkv, int64_t padded, float scale) {
  using S = DqSmem<D, W, WINDOW>;
  constexpr int NK = D / 32, ND = D / 16, CH = D / 8, RPI = 64 / CH, NLD = FWD_BN / (W * RPI), NST = S::NST;
  constexpr int ROWB = 2 * D, HALF = 16 * ROWB;
  extern __shared__ __attribute__((aligned(1024))) char smem[];

  const uint32_t lds0 = (uint32_t)(uintptr_t)(CA_LDS char *)smem;  // LDS byte address of the dynamic segment
  const int tid = threadIdx.x, lane = tid & 63, j4 = lane >> 4, li = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hk = __builtin_amdgcn_readfirstlane(u.head / (Hq / Hkv));  // (uniform, for scalar K/V addresses)
  // (group of the unit) -> (32-slot group, query head) inside the unit, as in the forward kernel
  const int hp_lg = __builtin_ctz(u.hp), pair = W * half + wave;
  const int head = u.head + (pair & (u.hp - 1));
  const int slot = u.slot0 + (pair >> hp_lg) * 32 + li;  // the lane's first query row (the other is 16 further on)
  const int pos_base = WINDOW ? 0 : u.key0;
  int row[2], pos[2], lo[2] = {0, 0};
  float l2[2], dl[2];
#pragma unroll
  for (int rg = 0; rg < 2; ++rg) {
    row[rg] = slot_row[slot + 16 * rg];
    if (WINDOW) lo[rg] = slot_lo[slot + 16 * rg];
    pos[rg] = slot_pos[slot + 16 * rg] - pos_base;  // counted from the first key of a piece's window (below 0: sees none of it)
    l2[rg] = l2_slot[int64_t(head) * padded + slot + 16 * rg];
    dl[rg] = delta_slot[int64_t(head) * padded + slot + 16 * rg];
  }
  const int wmax = wave_max(max(pos[0], pos[1])), wmin = wave_min(min(pos[0], pos[1]));
  int lo_min = WINDOW ? wave_min(min(lo[0], lo[1])) : 0;
  if (WINDOW && lo_min > wmax) lo_min = INT_MAX;  // (all windows are empty)
  const int lo_max = WINDOW ? wave_max(max(lo[0], lo[1])) : 0;
  // tiles some row of the workgroup sees (positions are sorted; at least one, which then is masked)
  const int key_lo = WINDOW ? u.key0 : 0, first_key = WINDOW ? -1 - u.part : 0, n_sink = WINDOW ? min((sinks + FWD_BN - 1) / FWD_BN, key_lo / FWD_BN) : 0;
  auto key_of = [&](int tile) __attribute__((always_inline)) {  // the first key of a tile
    return tile < n_sink ? FWD_BN * tile : key_lo + FWD_BN * (tile - n_sink);
  };
  int n_tiles = n_sink + (u.n_keys - key_lo + FWD_BN - 1) / FWD_BN;
  if (W < 8) {
    const int last = slot_pos[u.slot0 + ((W * half + W - 1) >> hp_lg) * 32 + 31] - pos_base - key_lo;
    n_tiles = max(1, min(n_tiles, n_sink + last / FWD_BN + 1));
  }
  const float c = scale * LOG2E;

  // direct loads addressed as (scalar tile base) + (per-lane 32-bit offset); rows past the last key are fetched as the last key,
  // and with more than two stages tiles past the end as the last tile (the wait at the top of a tile counts loads)
  const uint32_t kv_row_bytes = uint32_t(Hkv) * D * 2;
  const int ld_row0 = RPI * wave + lane / CH;  // + W*RPI*n
  const uint32_t ld_cbytes = uint32_t((lane % CH) ^ tile_sw<D>(ld_row0)) * 16;
  const int last_tile = n_tiles - 1, last_key_in_tile = min(FWD_BN, u.n_keys - key_of(last_tile)) - 1;
  const uint32_t ld_off = uint32_t(ld_row0) * kv_row_bytes + ld_cbytes;  // + W*RPI*n rows (the swizzle repeats every 16)
  static_assert(W * RPI % 16 == 0);
  const char *kg = reinterpret_cast<const char *>(K + (size_t(u.kv_row0) * Hkv + hk) * D);
  const char *vg = reinterpret_cast<const char *>(V + (size_t(u.kv_row0) * Hkv + hk) * D);
  const size_t tile_bytes = size_t(FWD_BN) * kv_row_bytes;
  auto issue_kv = [&](int tile) __attribute__((always_inline)) {
    const bool last = tile >= last_tile, edge = last || (WINDOW && (tile == n_sink || tile == n_sink - 1));  // (see the forward)
    const size_t at = WINDOW ? size_t(key_of(last ? last_tile : tile)) * kv_row_bytes : size_t(last ? last_tile : tile) * tile_bytes;
    const uint32_t dst = lds0 + uint32_t((tile % NST) * S::STAGE + 1024 * wave);
    if (!edge) {
#pragma unroll
      for (int n = 0; n < NLD; ++n) {
        load_lds16_sbase(kg + at + n * W * RPI * kv_row_bytes, ld_off, dst + S::K_OFF + 1024 * W * n);
        load_lds16_sbase(vg + at + n * W * RPI * kv_row_bytes, ld_off, dst + S::V_OFF + 1024 * W * n);
      }
    } else {
#pragma unroll
      for (int n = 0; n < NLD; ++n) {
        int row = ld_row0 + W * RPI * n;
        if (WINDOW) row = seen_row(last ? last_key_in_tile : FWD_BN - 1, key_of(last ? last_tile : tile), first_key, sinks, row);
        else row = min(row, last_key_in_tile);
        const uint32_t off = uint32_t(row) * kv_row_bytes + ld_cbytes;
        load_lds16_sbase(kg + at, off, dst + S::K_OFF + 1024 * W * n);
        load_lds16_sbase(vg + at, off, dst + S::V_OFF + 1024 * W * n);
      }
    }
  };
#pragma unroll
  for (int t = 0; t < NST - 1; ++t) issue_kv(t);

  // Q and dO fragments (B operands); lane holds row's elements 32 s + 8 j4 .. +7
  bf16x8 qf[NK][2], dof[NK][2];
#pragma unroll
  for (int rg = 0; rg < 2; ++rg) {
    const size_t off = (size_t(row[rg] < 0 ? 0 : row[rg]) * Hq + head) * D + 8 * j4;
#pragma unroll
    for (int s = 0; s < NK; ++s) {
      qf[s][rg] = *reinterpret_cast<const bf16x8 *>(Q + off + 32 * s);
      dof[s][rg] = *reinterpret_cast<const bf16x8 *>(dO + off + 32 * s);
    }
  }
  int koff = lds0 + li * ROWB + 16 * (j4 ^ tile_sw<D>(li));
  int toff = lds0 + (4 * j4 + (li >> 2)) * ROWB + 16 * (((li >> 1) & 1) ^ tile_sw<D>(4 * j4 + (li >> 2))) + 8 * (li & 1);

  f32x4 acc[ND][2];
#pragma unroll
  for (int b = 0; b < ND; ++b) acc[b][0] = acc[b][1] = f32x4{0.f, 0.f, 0.f, 0.f};

  // All register loads above are complete from here on, so the compiler places no vector-memory waits
  // inside the loop (they would drain the direct-load queue every iteration).
  wait_vmcnt<0>();
  f32x4 nd[2];  // -Delta, from which the dP chains start
#pragma unroll
  for (int rg = 0; rg < 2; ++rg) {
#pragma unroll
    for (int s = 0; s < NK; ++s) pin(qf[s][rg]), pin(dof[s][rg]);
    pin(l2[rg]), pin(dl[rg]);
    nd[rg] = f32x4{dl[rg], dl[rg], dl[rg], dl[rg]};
  }

  for (int j = 0; j < n_tiles; ++j) {
    const int j0 = WINDOW ? key_of(j) : j * FWD_BN;
    wait_vmcnt<2 * (NST - 2) * NLD>();  // this wave's parts of K(j), V(j) have landed
    barrier_nofence();      // ... and everybody else's; everybody is done with tile j-1
    if (NST > 2 || j < last_tile) issue_kv(j + NST - 1);
    const bool seen = j0 <= wmax && (!WINDOW || j0 + FWD_BN > lo_min || j0 < sinks);  // some row of this wave sees the tile
    const bool masked = j0 + FWD_BN - 1 > wmin || (WINDOW && j0 < lo_max && j0 + FWD_BN > sinks);
    // one 64-key tile; MASKED is a compile-time constant in each of the two instantiations below
    auto tile = [&](const int KB0, const int KB1, const bool MASKED) __attribute__((always_inline)) {
      // Fragments come from LDS AHEAD fragments before the MFMAs that use them: per 32-key block 2 NK of K (scores), 2 NK of V
      // (dP) and ND of K transposed (dQ).
      constexpr int NF = 2 * NK + 2 * NK + ND, AHEAD = 4;
      bf16x8 fr[AHEAD];
      auto fetch = [&](int i) __attribute__((always_inline)) -> bf16x8 {
        const int kb = KB0 + i / NF, f = i % NF;
        const int KT = S::K_OFF + 32 * kb * ROWB, VT = S::V_OFF + 32 * kb * ROWB;
        if (f < 4 * NK) return lds_read8_at((f < 2 * NK ? KT : VT) + HALF * (f & 1) + (koff ^ (64 * (f % (2 * NK) / 2))));
        const int ta = toff ^ (32 * (f - 4 * NK));
        return join(lds_read_tr4_at(KT + ta), lds_read_tr4_at(KT + HALF + ta));
      };
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) fr[i] = fetch(i);
#pragma unroll
      for (int kb = KB0; kb < KB1; ++kb) {
        auto next = [&](int f) __attribute__((always_inline)) {  // fragment f is used: its registers take the one AHEAD later
          if (NF * (kb - KB0) + f + AHEAD < NF * (KB1 - KB0)) fr[f % AHEAD] = fetch(NF * (kb - KB0) + f + AHEAD);
        };
        static_assert(NF % AHEAD == 0);
        f32x4 sa[2][2], pa[2][2];  // [16 keys][16 rows]
#pragma unroll
        for (int f = 0; f < 2 * NK; ++f) {
#pragma unroll
          for (int rg = 0; rg < 2; ++rg) sa[f & 1][rg] = mfma16(fr[f % AHEAD], qf[f / 2][rg], f < 2 ? f32x4{0.f, 0.f, 0.f, 0.f} : sa[f & 1][rg]);
          next(f);
          __builtin_amdgcn_sched_barrier(0);
        }
        float p[2][2][4];
#pragma unroll
        for (int f = 0; f < 2 * NK; ++f) {
          const int kt = f & 1;
#pragma unroll
          for (int rg = 0; rg < 2; ++rg) pa[kt][rg] = mfma16(fr[f % AHEAD], dof[f / 2][rg], f < 2 ? nd[rg] : pa[kt][rg]);
          next(2 * NK + f);
          // 16 probabilities over 2 NK slots
#pragma unroll
          for (int i = 16 * f / (2 * NK); i < 16 * (f + 1) / (2 * NK); ++i) {
            const int e = i & 3, ekt = (i >> 2) & 1, rg = i >> 3;
            p[ekt][rg][e] = fast_exp2(fmaf(sa[ekt][rg][e], c, -l2[rg]));
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        uint32_t dw[2][4];
#pragma unroll
        for (int rg = 0; rg < 2; ++rg) {
          // register e of tile kt holds key j0 + 32 kb + 16 kt + 4 j4 + e: visible iff 16 kt + e <= vis
          const int vis = pos[rg] - (j0 + 32 * kb + 4 * j4), from = lo[rg] - (j0 + 32 * kb + 4 * j4);
          const int sink_end = sinks - (j0 + 32 * kb + 4 * j4);
          auto sees = [&](int i) __attribute__((always_inline)) { return i <= vis && (!WINDOW || i >= from || i < sink_end); };
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              float p0 = p[kt][rg][e], p1 = p[kt][rg][e + 1];
              if (MASKED) {
                p0 = sees(16 * kt + e) ? p0 : 0.f;
                p1 = sees(16 * kt + e + 1) ? p1 : 0.f;
              }
              dw[rg][2 * kt + e / 2] = pack_bf16(p0 * pa[kt][rg][e], p1 * pa[kt][rg][e + 1]);
            }
        }
        bf16x8 db[2];
#pragma unroll
        for (int rg = 0; rg < 2; ++rg) db[rg] = __builtin_bit_cast(bf16x8, u32x4{dw[rg][0], dw[rg][1], dw[rg][2], dw[rg][3]});
#pragma unroll
        for (int b = 0; b < ND; ++b) {
#pragma unroll
          for (int rg = 0; rg < 2; ++rg) acc[b][rg] = mfma16(fr[b % AHEAD], db[rg], acc[b][rg]);
          next(4 * NK + b);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    if (seen) {
      if (!masked) {
        tile(0, 2, false);
      } else if (!WINDOW) {
        tile(0, 2, true);
      } else {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const int k0 = j0 + 32 * kb;
          if (k0 <= wmax && (k0 + 32 > lo_min || k0 < sinks)) tile(kb, kb + 1, true);
        }
      }
    }
    // the offsets follow the stages round
    const int adv = (j % NST) == NST - 1 ? -(NST - 1) * S::STAGE : S::STAGE;
    koff += adv, toff += adv;
  }
  wait_vmcnt<0>();
  const int out_lane = lane_id_here();
  if (u.part >= 0) {  // a piece: the accumulators as they stand
    store_tile16_as_part<0>(parts + size_t(u.part) * (FWD_BM * D) + pair * (32 * D), acc, out_lane);
    return;
  }
  // dQ of the wave's 32 rows, as whole lines through a patch of LDS (the stages are free once every wave is past its
  // last tile)
  __syncthreads();
  static_assert(W * PATCH_BYTES <= S::TOTAL, "patches fit in the stages");
  store_tile16_as_lines<0>(lds0 + wave * PATCH_BYTES, acc, scale, scale, out_lane, [&](int p) __attribute__((always_inline)) -> bf16_t * {
    const int r0 = __shfl(row[0], p & 15), r1 = __shfl(row[1], p & 15);
    const int rw = p < 16 ? r0 : r1;
    return rw >= 0 ? dQ + (size_t(rw) * Hq + head) * D : nullptr;
  });
}

// ------------------------------------------------------------------------------------------------ dK, dV
// WINDOW: Q and dO come from where they are, by their rows, not from slot-ordered copies: few tiles of keys share a row (9 with a window
// of 1024), and the copies cost as much traffic as two fifths of them save.  The rows of a block are fetched NST - 1 tiles before the tile is.
template <int D, bool WINDOW = false>
struct DkvSmem {
  static constexpr int NST = D == 128 ? 2 : 3;      // two workgroups share a CU's LDS at head_dim 128, three at 64
  static constexpr int TILE = BWD_BQ * 2 * D;       // one Q or dO tile of 64 slots
  static constexpr int Q_OFF = 0;
  static constexpr int DO_OFF = TILE;
  static constexpr int L2_OFF = 2 * TILE;           // 64 floats each: 32 L2 and 32 -Delta of either half of the rows, positions, spare
  static constexpr int DL_OFF = L2_OFF + 128;
  static constexpr int POS_OFF = L2_OFF + 512;
  static constexpr int SPARE_OFF = POS_OFF + 256;
  static constexpr int STAGE = 2 * TILE + 1024;
  // WINDOW: packed rows of the tiles that are fetched next, [NROWS][64].  A wave that is ahead of the others before the first barrier has
  // issued NST - 1 tiles and fetched the rows of as many more, while another may not have read those of tile 0.
  static constexpr int NROWS = 2 * NST - 2, ROWS_OFF = NST * STAGE;
  static constexpr int TOTAL = ROWS_OFF + (WINDOW ? NROWS * 256 : 0);
  static_assert(4 * PATCH_BYTES <= NST * STAGE, "patches fit in the stages");
};

// A unit, or a chain of short units one after the other, in a workgroup of four waves, each of which owns 32 keys: K and V
// fragments (64 registers at head_dim 128) and dK / dV accumulators (128) stay in registers, and what is left of 256 holds one
// 32 x 32 tile of S and of dP and a ring of LDS fragments, so that two waves share a SIMD.  The two are of different workgroups
// and drift apart: one's exponentials, LDS latencies, barriers, first fetches and stores run under the other's MFMAs.  One wave
// per SIMD with 472 registers, its stream software-pipelined by hand across sub-blocks and across the units of a chain, did that
// less well everywhere (both with 32x32 MFMAs; dK/dV kernel, 32/8 heads unless noted): 222 -> 181 us on 4K tokens of documents
// of about 1K, 5.04 -> 4.76 ms on 64K tokens of about 2K, 112.7 -> 107.9 ms on 128K tokens of long and short documents, 3.85 ->
// 3.50 ms on the last 1000 rows of 130K, 3.55 -> 3.05 ms on lone 64-row shards with contexts (8/2).  Workgroups no longer wait for
// each other to share Q/dO tiles in L2.
// To stay within the registers, LDS addresses are one register per kind of read, from which an exclusive or makes the address of
// each fragment (4 cycles per 2 MFMAs), and what the lane index gives is derived again where it is needed.
template <int D, bool WINDOW = false>
__device__ __forceinline__ void dkv_workgroup(const int me /* index of the first unit */,
                                              const std::conditional_t<WINDOW, WindowUnit, BwdUnit> *__restrict__ units,
                                              const int32_t *__restrict__ slot_pos, const int32_t *__restrict__ slot_lo,
                                              const int32_t *__restrict__ slot_src, const int sinks, const bf16_t *__restrict__ Qs,
                                              const bf16_t *__restrict__ K, const bf16_t *__restrict__ V,
                                              const bf16_t *__restrict__ dOs, const float *__restrict__ stats_kv,
                                              bf16_t *__restrict__ dK,
                                              bf16_t *__restrict__ dV, float *__restrict__ parts, int Hq, int Hkv, float scale) {
  using S = DkvSmem<D, WINDOW>;
  constexpr int NK = D / 32, ND = D / 16, CH = D / 8, RPI = 64 / CH, NST = S::NST;
  constexpr int NLD = BWD_BQ / (4 * RPI);  // direct loads per wave per Q (or dO) tile
  constexpr int RPW = BWD_BQ / 4;          // tile rows fetched by one wave (contiguous)
  constexpr int ROWB = 2 * D;
  constexpr int LPI = 2 * NLD + 1 + WINDOW;  // loads per wave per iteration
  constexpr int SUB = 32 * ROWB, HALF = 16 * ROWB;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(CA_LDS char *)smem;  // LDS byte address of the dynamic segment
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = Hq / Hkv;
  const float c = scale * LOG2E;
  const int64_t head_stride = BWD_BQ * D * 2;            // bytes between the tiles of consecutive heads of a block
  const int64_t block_stride = int64_t(Hq) * head_stride;  // ... of consecutive blocks, same head
  auto *up = units + me;
  const int count = up->count, follow = up->follow;
  for (int done = 0;;) {
    const auto u = *up;
    const int lane = lane_id_here(), j = lane >> 4, li = lane & 15;
    const int kw0 = 32 * wave;
    const int hk = u.kv_head;
    const int n_blocks = (u.slot_end - u.slot_begin) / BWD_BQ;
    const int Gu = u.heads;  // tiles per block: the heads of the group, or fewer in a block of packed rows
    const int n_it = n_blocks * Gu;
    // Query blocks are walked from the document's LAST block backwards: the blocks that lie entirely below the diagonal of this KV
    // tile come first and need no mask, and workgroups that run side by side on an XCD (same KV head, neighbouring KV tiles)
    // start on the same Q/dO tiles.
    const int n_full = ((u.slot_end - u.slot_full) / BWD_BQ) * Gu;
    int n_edge = 0;  // WINDOW: the blocks at the end whose rows do not all have the whole tile in their window
    if constexpr (WINDOW) n_edge = ((u.slot_end - u.slot_edge) / BWD_BQ) * Gu;

    // Loads of one (block, head): this wave fetches tile rows RPW*wave .. of Q and of dO, RPI rows per load, plus one 64-float
    // auxiliary array: log2e*LSE and -Delta of 32 rows each (waves 0 and 1), slot positions (wave 2; wave 3 the same into a spare
    // area, so that every wave issues the same number of loads, or, WINDOW, where the rows' windows begin).  Q and dO come from their slot-ordered copies [block][head][64][D], in which
    // the tile of a (block, head) is one contiguous run: a load is (wave-uniform tile address) + (per-lane constant).
    const int trow = RPW * wave + lane / CH;
    const uint32_t ld_off = uint32_t(trow * ROWB + 16 * ((lane % CH) ^ tile_sw<D>(trow)));
    int left = n_it;  // tiles still to be fetched
    int ph = 0, pst = 0;
    const int64_t tile0 = (int64_t(u.slot_begin / BWD_BQ + n_blocks - 1) * Hq + hk * G) * head_stride;
    const char *q_tile = reinterpret_cast<const char *>(Qs) + tile0, *do_tile = reinterpret_cast<const char *>(dOs) + tile0;
    const int64_t aux_hstride = wave < 2 ? 128 : 0, aux_bstride = wave < 2 ? int64_t(Hq) * 128 : BWD_BQ;
    const float *aux_ptr = (wave < 2 ? stats_kv + hk * G * 128 + wave * 64 : reinterpret_cast<const float *>(WINDOW && wave == 3 ? slot_lo : slot_pos)) +
                           (u.slot_begin / BWD_BQ + n_blocks - 1) * aux_bstride;
    const uint32_t aux_lds = wave < 2 ? S::L2_OFF + 256 * wave : wave == 2 ? S::POS_OFF : S::SPARE_OFF;
    // WINDOW: the rows of tile t are fetched with tile t - NST + 1, every wave for itself (all write the same), and are there when t is
    // issued, NST - 1 steps later
    int row_block = u.slot_begin / BWD_BQ + n_blocks - 1, row_ph = 0, row_left = n_it, rst = 0, rd = 0;
    auto issue_rows = [&]() __attribute__((always_inline)) {
      load_lds4_sbase(slot_src + int64_t(row_block) * BWD_BQ, uint32_t(lane_id_here()) * 4, lds0 + S::ROWS_OFF + 256 * rst);
      rst = rst + 1 == S::NROWS ? 0 : rst + 1;
      if (--row_left > 0 && ++row_ph == Gu) row_ph = 0, --row_block;
    };
    auto issue_next = [&]() __attribute__((always_inline)) {
      const uint32_t st = lds0 + pst * S::STAGE;
      if constexpr (WINDOW) {
        const int l = lane_id_here(), r0 = RPW * wave + l / CH;
        const uint32_t chunk = 16 * ((l % CH) ^ tile_sw<D>(r0));
        const uint64_t head = (uint64_t)(uintptr_t)Qs + (uint64_t)(hk * G + ph) * ROWB, to_do = (uint64_t)(uintptr_t)dOs - (uint64_t)(uintptr_t)Qs;
#pragma unroll
        for (int n = 0; n < NLD; ++n) {
          const uint32_t row = lds_ld<uint32_t>(lds0 + S::ROWS_OFF + 256 * rd + 4 * (r0 + RPI * n));
          const uint64_t a = head + (uint64_t)row * uint32_t(Hq * ROWB) + (chunk ^ (D == 128 ? 16 * (2 * ((n & 1) ^ (n >> 1)) + (n >> 1)) : 48 * n));
          load_lds16_addr(a, st + S::Q_OFF + (RPW * wave + RPI * n) * ROWB);
          load_lds16_addr(a + to_do, st + S::DO_OFF + (RPW * wave + RPI * n) * ROWB);
        }
        load_lds4_sbase(aux_ptr, uint32_t(l) * 4, st + aux_lds);
        pst = pst + 1 == NST ? 0 : pst + 1;
        rd = rd + 1 == S::NROWS ? 0 : rd + 1;
        issue_rows();
        if (--left <= 0) return;
        if (ph + 1 < Gu) ++ph, aux_ptr += aux_hstride;
        else ph = 0, aux_ptr -= (Gu - 1) * aux_hstride + aux_bstride;
        return;
      }
      uint32_t ld0 = ld_off;
      asm volatile("" : "+v"(ld0));
#pragma unroll
      for (int n = 0; n < NLD; ++n) {
        // (rows RPI n further down; the swizzle of the row changes by an exclusive or)
        const uint32_t off = (ld0 ^ (D == 128 ? 16 * (2 * ((n & 1) ^ (n >> 1)) + (n >> 1)) : 48 * n)) + RPI * n * ROWB;
        load_lds16_sbase(q_tile, off, st + S::Q_OFF + (RPW * wave + RPI * n) * ROWB);
        load_lds16_sbase(do_tile, off, st + S::DO_OFF + (RPW * wave + RPI * n) * ROWB);
      }
      load_lds4_sbase(aux_ptr, uint32_t(lane_id_here()) * 4, st + aux_lds);
      pst = pst + 1 == NST ? 0 : pst + 1;
      if (--left <= 0) return;
      if (ph + 1 < Gu) {  // next tile of the group, same block
        ++ph;
        q_tile += head_stride, do_tile += head_stride, aux_ptr += aux_hstride;
      } else {  // first head of the group, previous block
        ph = 0;
        q_tile -= (Gu - 1) * head_stride + block_stride, do_tile -= (Gu - 1) * head_stride + block_stride;
        aux_ptr -= (Gu - 1) * aux_hstride + aux_bstride;
      }
    };
    if (n_it > 0) {
      if (WINDOW) {
#pragma unroll
        for (int i = 0; i < NST - 1; ++i) issue_rows();
        wait_vmcnt<0>();
      }
#pragma unroll
      for (int i = 0; i < NST - 1; ++i) issue_next();
    }

    // K, V fragments of the wave's 32 keys (B operands of S = Q K^T and dP = dO V^T).  Keys past the document's last key are
    // clamped; their positions exceed every query position, so they are masked.
    bf16x8 kf[NK][2], vf[NK][2];
#pragma unroll
    for (int kg = 0; kg < 2; ++kg) {
      const int key = min(kw0 + 16 * kg + li, u.n_valid - 1);
      const size_t off = (size_t(u.kv_row + key) * Hkv + hk) * D + 8 * j;
#pragma unroll
      for (int s = 0; s < NK; ++s) {
        kf[s][kg] = *reinterpret_cast<const bf16x8 *>(K + off + 32 * s);
        vf[s][kg] = *reinterpret_cast<const bf16x8 *>(V + off + 32 * s);
      }
    }
    wait_vmcnt<0>();  // (from here on the compiler places no vector-memory waits: they would drain the direct loads)
#pragma unroll
    for (int s = 0; s < NK; ++s) pin(kf[s][0]), pin(kf[s][1]), pin(vf[s][0]), pin(vf[s][1]);
    // natural reads, transposing reads and row statistics in the current stage
    int nb = lds0 + li * ROWB + 16 * (j ^ tile_sw<D>(li));
    int tb = lds0 + (4 * j + (li >> 2)) * ROWB + 16 * (((li >> 1) & 1) ^ tile_sw<D>(4 * j + (li >> 2))) + 8 * (li & 1);
    int auxo = lds0 + 16 * j, stage = 0;

    f32x4 acc_dk[ND][2], acc_dv[ND][2];
#pragma unroll
    for (int b = 0; b < ND; ++b)
#pragma unroll
      for (int kg = 0; kg < 2; ++kg) acc_dk[b][kg] = acc_dv[b][kg] = f32x4{0.f, 0.f, 0.f, 0.f};

    // Sub-blocks [QB0, QB1) of 32 rows each; MASK: some row of the block does not see some key of the tile.
    // Fragments come from LDS AHEAD fragments before the MFMAs that use them: per sub-block 2 NK of Q (scores), 2 NK of dO
    // (dP), ND of dO transposed (dV) and ND of Q transposed (dK).  The exponentials go between the MFMAs of dP, dS between those of
    // dV: 4.60 -> 4.31 ms on 64K tokens of documents of about 2K, 103.7 -> 99.9 ms on 128K tokens (32/8 heads), against
    // the compiler's order.  (3 ahead is within 0.5 %, and does not fit the registers.)
    constexpr int NF = 4 * NK + 2 * ND, AHEAD = 2;
    auto sub_blocks = [&](const int QB0, const int QB1, const bool MASK) __attribute__((always_inline)) {
      bf16x8 fr[AHEAD];
      auto fetch = [&](int i) __attribute__((always_inline)) -> bf16x8 {
        const int qb = i / NF, f = i % NF;
        const int QT = S::Q_OFF + qb * SUB, DOT = S::DO_OFF + qb * SUB;
        if (f < 4 * NK) return lds_read8_at((f < 2 * NK ? QT : DOT) + HALF * (f & 1) + (f % (2 * NK) < 2 ? nb : xor_here(nb, 64 * (f % (2 * NK) / 2))));
        const int t = (f < 4 * NK + ND ? DOT : QT) + ((f - 4 * NK) % ND == 0 ? tb : xor_here(tb, 32 * ((f - 4 * NK) % ND)));
        return join(lds_read_tr4_at(t), lds_read_tr4_at(HALF + t));
      };
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) fr[i] = fetch(NF * QB0 + i);
#pragma unroll
      for (int qb = QB0; qb < QB1; ++qb) {
        int at = NF * (qb - QB0);  // the fragment in use, counted from the first
        auto next = [&]() __attribute__((always_inline)) {  // it has been used: its registers take the one AHEAD later
          if (at + AHEAD < NF * (QB1 - QB0)) fr[at % AHEAD] = fetch(NF * QB0 + at + AHEAD);
          ++at;
          __builtin_amdgcn_sched_barrier(0);
        };
        f32x4 sa[2][2], pa[2][2];  // [16 rows][16 keys]: S, and dP - Delta: its chain starts from -Delta
        f32x4 nd[2], l2v[2];
#pragma unroll
        for (int f = 0; f < 2 * NK; ++f) {
          if (f == 2 * NK - 2) {
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) nd[rt] = lds_ld<f32x4>(S::DL_OFF + 256 * qb + 64 * rt + auxo);
          }
          if (f == 2 * NK - 1) {
#pragma unroll
            for (int rt = 0; rt < 2; ++rt) l2v[rt] = lds_ld<f32x4>(S::L2_OFF + 256 * qb + 64 * rt + auxo);
          }
#pragma unroll
          for (int kg = 0; kg < 2; ++kg) sa[f & 1][kg] = mfma16(fr[at % AHEAD], kf[f / 2][kg], f < 2 ? f32x4{0.f, 0.f, 0.f, 0.f} : sa[f & 1][kg]);
          next();
        }
#pragma unroll
        for (int f = 0; f < 2 * NK; ++f) {
#pragma unroll
          for (int kg = 0; kg < 2; ++kg) pa[f & 1][kg] = mfma16(fr[at % AHEAD], vf[f / 2][kg], f < 2 ? nd[f & 1] : pa[f & 1][kg]);
          // P, in place of S: 16 values over 2 NK slots
#pragma unroll
          for (int i = 16 * f / (2 * NK); i < 16 * (f + 1) / (2 * NK); ++i) {
            const int e = i & 3, kg = (i >> 2) & 1, rt = i >> 3;
            sa[rt][kg][e] = fast_exp2(fmaf(sa[rt][kg][e], c, -l2v[rt][e]));
          }
          next();
        }
        if (MASK) {
#pragma unroll
          for (int rt = 0; rt < 2; ++rt) {
            const int key_pos = u.key_pos0 + kw0 + (lane_id_here() & 15);  // position of this lane's first key (the other is 16 further on)
            const u32x4 pv = lds_ld<u32x4>(S::POS_OFF + (32 * qb + 16 * rt) * 4 + auxo);
            u32x4 lv = {0, 0, 0, 0};
            if (WINDOW) lv = lds_ld<u32x4>(S::SPARE_OFF + (32 * qb + 16 * rt) * 4 + auxo);
#pragma unroll
            for (int kg = 0; kg < 2; ++kg)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int key = key_pos + 16 * kg;
                const bool sees = key <= int(pv[e]) && (!WINDOW || key >= int(lv[e]) || key < sinks);
                sa[rt][kg][e] = sees ? sa[rt][kg][e] : 0.f;
              }
          }
        }
        bf16x8 pb[2], db[2];
        uint32_t dw[2][4];
#pragma unroll
        for (int kg = 0; kg < 2; ++kg)
          pb[kg] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16(sa[0][kg][0], sa[0][kg][1]), pack_bf16(sa[0][kg][2], sa[0][kg][3]),
                                                    pack_bf16(sa[1][kg][0], sa[1][kg][1]), pack_bf16(sa[1][kg][2], sa[1][kg][3])});
#pragma unroll
        for (int b = 0; b < ND; ++b) {
#pragma unroll
          for (int kg = 0; kg < 2; ++kg) acc_dv[b][kg] = mfma16(fr[at % AHEAD], pb[kg], acc_dv[b][kg]);
          // dS: 8 pairs over ND slots
#pragma unroll
          for (int i = 8 * b / ND; i < 8 * (b + 1) / ND; ++i) {
            const int e = 2 * (i & 1), rt = (i >> 1) & 1, kg = i >> 2;
            // (values of keys that nobody sees may be anything: 0 times it is 0)
            auto times = [&](float x, float y) { return WINDOW && MASK && x == 0.f ? 0.f : x * y; };
            dw[kg][2 * rt + e / 2] = pack_bf16(times(sa[rt][kg][e], pa[rt][kg][e]), times(sa[rt][kg][e + 1], pa[rt][kg][e + 1]));
          }
          next();
        }
#pragma unroll
        for (int kg = 0; kg < 2; ++kg) db[kg] = __builtin_bit_cast(bf16x8, u32x4{dw[kg][0], dw[kg][1], dw[kg][2], dw[kg][3]});
#pragma unroll
        for (int b = 0; b < ND; ++b) {
#pragma unroll
          for (int kg = 0; kg < 2; ++kg) acc_dk[b][kg] = mfma16(fr[at % AHEAD], db[kg], acc_dk[b][kg]);
          next();
        }
      }
    };
    int it = 0;
    auto step = [&](const bool MASK) __attribute__((always_inline)) {
      wait_vmcnt<(NST - 2) * LPI>();  // block `it` has landed (this wave's part); block it+1 may be in flight
      barrier_nofence();              // ... and everybody else's; everybody is done with block it-1
      if (NST > 2 || left > 0) issue_next();
      if (!MASK) {
        sub_blocks(0, 2, false);
      } else {
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {  // (a sub-block entirely above the diagonal for this wave's keys is left out: positions are sorted)
          if (WINDOW) {  // (or one whose windows have all passed them by, where they are no sinks)
            const uint32_t at = lds0 + stage * S::STAGE + (32 * qb + (lane_id_here() & 31)) * 4;
            const int hi = lds_ld<int>(at + S::POS_OFF), lo = lds_ld<int>(at + S::SPARE_OFF), key = u.key_pos0 + kw0;
            if (__any(hi >= key && (lo <= key + 31 || key < sinks))) sub_blocks(qb, qb + 1, true);
          } else {
            const int sub_max_pos = lds_ld<int>(lds0 + stage * S::STAGE + S::POS_OFF + (32 * qb + 31) * 4);
            if (sub_max_pos >= u.key_pos0 + kw0) sub_blocks(qb, qb + 1, true);
          }
        }
      }
      const int adv = stage == NST - 1 ? -(NST - 1) * S::STAGE : S::STAGE;
      stage = stage == NST - 1 ? 0 : stage + 1;
      nb += adv, tb += adv, auxo += adv;
    };
    if (WINDOW) {
      for (; it < n_edge; ++it) step(true);
      for (; it < n_full; ++it) step(false);
      for (; it < n_it; ++it) step(true);
    } else {
      for (; it < n_full; ++it) step(false);
      for (; it < n_it; ++it) step(true);
    }
    wait_vmcnt<0>();  // nothing may still be writing LDS
    const int ol = lane_id_here();
    if (count <= 1 && follow < 0) {  // a piece of a unit's query blocks: the accumulators as they stand
      float *const dst = parts + size_t(-1 - follow) * (FWD_BM * D) + 2 * wave * (32 * D);
      store_tile16_as_part<0>(dst, acc_dk, ol);
      store_tile16_as_part<0>(dst + 32 * D, acc_dv, ol);
      return;
    }
    __syncthreads();  // every wave is done with the stages
#pragma unroll
    for (int t = 0; t < 2; ++t)
      store_tile16_as_lines<0>(lds0 + wave * PATCH_BYTES, t == 0 ? acc_dk : acc_dv, t == 0 ? scale : 1.0f, t == 0 ? scale : 1.0f, ol,
                                [&](int p) __attribute__((always_inline)) -> bf16_t * {
        const int key = kw0 + p;
        return key < u.n_valid ? (t == 0 ? dK : dV) + (size_t(u.kv_row + key) * Hkv + hk) * D : nullptr;
      });
    if (++done >= count) return;
    __syncthreads();  // ... and with its patch
    up = units + follow + done - 1;
  }
}

}  // namespace ca
