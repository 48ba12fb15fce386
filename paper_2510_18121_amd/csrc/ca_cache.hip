// A paged cache of keys and values in 8 bits, and the attention that reads it (serving: single tokens and chunks of prompts).
//
// A page holds 64 tokens.  Of a page and KV head: the keys as e4m3 codes [64][D], the values as e4m3 codes [D][64], and one fp32
// scale each; a code stands for code * scale.  With that layout every operand of the two products is a run of 16 bytes per lane
// straight from global memory, with no transposition and no trip through LDS:
//   S^T = K Q^T (v_mfma_f32_16x16x32_bf16, 16 keys x 16 rows): row i of tile t of a page is key 16 (i / 4) + 4 t + i % 4, so that lane
//   (r, j) of the results holds keys 16 j .. 16 j + 15 of query row r, in order, over the four tiles;
//   O^T += V^T P^T: the probabilities of two tiles are the B operand as they stand, and the lane's A operand is 8 consecutive
//   tokens of a V^T row.
// e4m3 is exact in bf16; the scales go into the exponent's factor (K) and into the probabilities (V).
//
// O = softmax(scale Q K^T) V and LSE need the codes once, 2 D bytes per (token, KV head): reading them bounds single tokens, and
// matrix products bound chunks.  Measured (kernel times under rocprofv3, medians over four sets of inputs in turn, of which the last cache holds none
// of the large ones; 8 KV heads of 128 unless noted):
//   attend   64 sequences of about 4096 tokens, 32 heads      144 us, 6.2 TB/s (a large copy: 4.97 read and written)
//            4 sequences of 130K tokens, 64 heads             173 us, 6.2 TB/s
//            32 sequences, window 4096, 16/16 heads of 64      54 us, 4.9 TB/s (47 us on one set of inputs)
//            one sequence of 901 tokens                      11.6 us (15 pages of 16 KiB, one CU per KV head: 9 bytes per cycle and
//                                                             CU; 15 from the first page to the last, the rest is the way there and back)
//   chunk    4 chunks of 500 rows behind 8192 tokens          246 us, 0.78 PFLOP/s (222 and 0.87 in a call without the profiler)
//   combine  of these                                         4 to 5 us, 13 us
//   append   128 tokens; 16 prompts of up to 2048             6.6 us; 41 us, 3.4 TB/s (32 us on one set of inputs)
//   copy     4000 pages of 128 KiB                            212 us, 4.9 TB/s
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <sstream>

#include "ca_cache.h"
#include "ca_cache_attend.h"
#include "ca_device.h"
#include "ca_internal.h"
#include "ca_launch.h"

namespace ca {

// ------------------------------------------------------------------------------------------------ attention
template <int D, int NR, int W>
__global__ __launch_bounds__(64 * W, NR == 1 || D == 64 ? 2 : 1) void ca_cache_attend_kernel(const AttendArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  WorkSplit<WHOLE> split;
  split.count<64 * W>(smem + AttendShape<D, NR, W>::MERGE, a, 16 * NR);
  split.deal(gridDim.y, a.by_workers, W);
  attend_workgroup<WHOLE, D, NR, W>(a, smem, split, blockIdx.x, blockIdx.y, a.parts);
}

template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void ca_cache_chunk_kernel(const AttendArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  WorkSplit<WHOLE> split;
  split.count<256>(smem + ChunkSmem<D>::TOTAL, a, 128);
  split.deal(gridDim.y, a.by_workers, 4);
  chunk_workgroup<WHOLE, D, false>(a, smem, split, blockIdx.x, blockIdx.y, a.parts);
}

// Adds up the parts of the tiles that were cut, in their order: a wave takes RW rows, and two (four) parts of each at a time.  4 to 5 us, of which
// most is the way to the first load (13 us for chunks: 29 MB of parts; of those a wave takes two rows, one or four: +1 %); a worker adding them up in the first kernel would need counters that
// somebody clears.
template <int D, int NR>
__global__ __launch_bounds__(256) void ca_cache_combine_kernel(const AttendArgs a) {
  constexpr int R = 16 * NR, LANES = D / 4, AT_A_TIME = 64 / LANES, RW = NR == 8 ? 2 : 1;
  const int hk = blockIdx.x, worker = blockIdx.y;
  int4 head = a.heads[worker * a.hkv + hk];  // {parts, first row of the sequence, first row of the tile, last row of the tile}
  head.x = min(head.x, int(gridDim.y) - worker);  // (sequences that overlap, against their description, may have more units than are counted)
  const int G = a.G, lane = threadIdx.x & 63, r0 = RW * (4 * blockIdx.z + (threadIdx.x >> 6));
  if (head.x < 2 || head.z + r0 > head.w) return;
  const size_t stride = size_t(2 * a.hkv) * (R * (D + 2));
  const float *const first = a.parts + size_t((worker * 2 + 1) * a.hkv + hk) * (R * (D + 2));
  const float *const others = first + stride - size_t(a.hkv) * (R * (D + 2));
  auto part = [&](int i) { return i == 0 ? first : others + size_t(i - 1) * stride; };
  const int mine = lane / LANES, col = 4 * (lane % LANES);
  f32x4 y[RW];
  float top[RW], sum[RW];
#pragma unroll
  for (int x = 0; x < RW; ++x) top[x] = NO_MAX, sum[x] = 0.f, y[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto add = [&](int x, float m, float l, const f32x4 &z) __attribute__((always_inline)) {
    const float grown = fmaxf(top[x], m), old = fast_exp2(top[x] - grown), w = fast_exp2(m - grown);
    top[x] = grown, sum[x] = sum[x] * old + w * l;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[x][e] = y[x][e] * old + w * z[e];
  };
  // (rows behind the tile's last one are read and not stored: their parts are whatever the workers left there)
#pragma unroll RW == 1 ? 8 : 2
  for (int i = mine; i < head.x; i += AT_A_TIME) {
    const float *const p = part(i) + r0 * D + col, *const ml = part(i) + R * D + 2 * r0;
#pragma unroll
    for (int x = 0; x < RW; ++x) add(x, ml[2 * x], ml[2 * x + 1], *reinterpret_cast<const f32x4 *>(p + x * D));
  }
#pragma unroll
  for (int x = 0; x < RW; ++x) {
#pragma unroll
    for (int o = LANES; o < 64; o <<= 1) {
      f32x4 z;
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = __shfl_xor(y[x][e], o);
      add(x, __shfl_xor(top[x], o), __shfl_xor(sum[x], o), z);
    }
    const int at = head.z + r0 + x, token = a.token_of(at), h = hk * G + at - token * G;
    if (mine != 0 || at > head.w) continue;
    const float inv = sum[x] == 0.f ? 0.f : 1.0f / sum[x];
    *reinterpret_cast<u32x2 *>(a.o + (size_t(head.y + token) * a.hq + h) * D + col) =
        u32x2{pack_bf16(y[x][0] * inv, y[x][1] * inv), pack_bf16(y[x][2] * inv, y[x][3] * inv)};
    if (col == 0 && a.lse) a.lse[size_t(h) * a.s.total + head.y + token] = 0.6931471805599453f * (top[x] + fast_log2(sum[x]));
  }
}

// ------------------------------------------------------------------------------------------------ append
struct AppendArgs {
  SeqArgs s;
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  const bf16_t *new_k, *new_v;
  int hkv;
};

// The smallest power of two that is at least top / 448, the largest e4m3 value (448 = 1.75 * 2^8), and at least 2^-126.
__device__ __forceinline__ float scale_for(float top) {
  const uint32_t u = __builtin_bit_cast(uint32_t, top);
  const int e = int(u >> 23) - 8 + ((u & 0x7FFFFF) > 0x600000);  // the exponent field of the scale
  return __builtin_bit_cast(float, uint32_t(max(e, 1)) << 23);
}
// The smallest power of two that is at least x (of a positive normal number).
__device__ __forceinline__ float next_power(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  return __builtin_bit_cast(float, (u & 0x7FFFFF) ? ((u >> 23) + 1) << 23 : u);
}
__device__ __forceinline__ float inverse_power(float s) {  // of a power of two from 2^-126 to 2^126
  return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, s));
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
// four values to four codes, nearest, ties to even (no finite value here is beyond 448; Inf and NaN become NaN)
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}
__device__ __forceinline__ uint32_t scaled_codes(uint32_t w, float f) {
  return to_codes(__builtin_amdgcn_cvt_f32_fp8(int(w), 0) * f, __builtin_amdgcn_cvt_f32_fp8(int(w), 1) * f,
                  __builtin_amdgcn_cvt_f32_fp8(int(w), 2) * f, __builtin_amdgcn_cvt_f32_fp8(int(w), 3) * f);
}
// the larger of the finite magnitudes of a word's two values and `top` (bits of a bf16)
__device__ __forceinline__ uint32_t top_of(uint32_t top, uint32_t w) {
  const uint32_t a = w & 0x7FFF, b = (w >> 16) & 0x7FFF;
  return max(top, max(a < 0x7F80 ? a : 0u, b < 0x7F80 ? b : 0u));
}
__device__ __forceinline__ float wave_top(uint32_t top) { return __builtin_bit_cast(float, uint32_t(wave_max(int(top))) << 16); }

// One wave per (page that gets new tokens, KV head, K or V): the largest magnitude of the new tokens, the scale, the codes.  A page that
// is all new (of a prompt) passes through registers once; of any other the new tokens are read twice, a few at a time, the second time
// from the caches.  Where such a page's scale grows, all that it holds is rounded again, from old / new of the scales: exact but for codes
// that leave the normal range.
// K: D / 8 lanes per token, 8 columns each.  V: a lane has two columns; at head_dim 64 the wave's halves take tokens of their own.
// (128 single tokens: 22 us with a workgroup per page, K and V one after the other; 8.6 with a wave each; 6.8 with the sequences in lanes or LDS.
// 16 prompts of up to 2048 tokens: 47, 40.7 and 32 us on one set of inputs, which the last cache holds; 41 where it does not.)
template <int D>
__global__ __launch_bounds__(256) void ca_cache_append_kernel(const AppendArgs a) {
  constexpr int LPT = D / 8, TPI = 64 / LPT, NI = PAGE / TPI;  // K: lanes per token, tokens per load, loads per page
  constexpr int VL = D / 2, VT = 64 / VL, NV = PAGE / VT;      // V: lanes per token, halves, tokens per half of a whole page
  extern __shared__ __attribute__((aligned(16))) char smem[];
  SeqTable tab;
  auto first_pos = [](const Seq &q) { return max(0, q.len - q.n); };
  const int total = tab.fill<256>(smem, a.s, [&](const Seq &q) { return q.n > 0 && q.len > 0 ? (q.len - 1) / PAGE - first_pos(q) / PAGE + 1 : 0; });
  const int unit = int(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int touch = unit / (2 * a.hkv), h = unit / 2 % a.hkv, lane = threadIdx.x & 63;
  if (touch >= total) return;
  const int s = tab.find(touch);
  const Seq q = tab.at(s);
  const int index = first_pos(q) / PAGE + touch - tab.before(s);
  const int page = a.s.table[size_t(s) * a.s.width + index];
  if (page < 0 || page >= a.s.n_pages) return;
  const int begin = max(first_pos(q) - index * PAGE, 0), end = min(q.len - index * PAGE, PAGE);  // the page's tokens that are new
  const int64_t row0 = int64_t(q.row0) + index * PAGE - (q.len - q.n);                           // the row of the page's token 0
  const size_t at = size_t(page) * a.hkv + h, row = size_t(a.hkv) * D;
  // 1 / the new scale and old / new; stores the new scale
  auto scales = [&](uint32_t top, float old, float *scale, float &f, float &again) {
    const float need = scale_for(wave_top(top)), now = old > 0.f ? fmaxf(need, next_power(old)) : need;
    f = inverse_power(now), again = old > 0.f ? old * f : 1.f;
    if (lane == 0) *scale = now;
  };
  float f, again;

  if (unit % 2 == 0) {
    const bf16_t *const src = a.new_k + row0 * int64_t(row) + size_t(h) * D + 8 * (lane % LPT);
    uint8_t *const dst = a.k + at * (PAGE * D) + 8 * (lane % LPT);
    auto codes = [&](const u32x4 &x) {
      return u32x2{to_codes(bf16_lo(x[0]) * f, bf16_hi(x[0]) * f, bf16_lo(x[1]) * f, bf16_hi(x[1]) * f),
                   to_codes(bf16_lo(x[2]) * f, bf16_hi(x[2]) * f, bf16_lo(x[3]) * f, bf16_hi(x[3]) * f)};
    };
    uint32_t top = 0;
    if (end - begin == PAGE) {
      u32x4 x[NI];
#pragma unroll
      for (int i = 0; i < NI; ++i) x[i] = *reinterpret_cast<const u32x4 *>(src + (TPI * i + lane / LPT) * row);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) top = top_of(top, x[i][w]);
      scales(top, 0.f, a.k_scale + at, f, again);
#pragma unroll
      for (int i = 0; i < NI; ++i) *reinterpret_cast<u32x2 *>(dst + (TPI * i + lane / LPT) * D) = codes(x[i]);
      return;
    }
    const float old = begin > 0 ? a.k_scale[at] : 0.f;
    for (int t0 = begin; t0 < end; t0 += 4 * TPI) {
      u32x4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = t0 + TPI * i + lane / LPT;
        x[i] = u32x4{0, 0, 0, 0};
        if (t < end) x[i] = *reinterpret_cast<const u32x4 *>(src + t * row);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) top = top_of(top, x[i][w]);
    }
    scales(top, old, a.k_scale + at, f, again);
    if (again != 1.f) {
#pragma unroll 4
      for (int t = lane / LPT; t < PAGE; t += TPI) {
        const u32x2 w = *reinterpret_cast<const u32x2 *>(dst + t * D);
        if (t < begin || t >= end) *reinterpret_cast<u32x2 *>(dst + t * D) = u32x2{scaled_codes(w[0], again), scaled_codes(w[1], again)};
      }
    }
#pragma unroll 4
    for (int t = begin + lane / LPT; t < end; t += TPI) *reinterpret_cast<u32x2 *>(dst + t * D) = codes(*reinterpret_cast<const u32x4 *>(src + t * row));
    return;
  }

  const bf16_t *const src = a.new_v + row0 * int64_t(row) + size_t(h) * D + 2 * (lane % VL);
  uint8_t *const dst = a.v + at * (PAGE * D) + 2 * (lane % VL) * PAGE;
  auto codes = [&](int c, const uint32_t *x) {  // of column c of four tokens
    return c == 0 ? to_codes(bf16_lo(x[0]) * f, bf16_lo(x[1]) * f, bf16_lo(x[2]) * f, bf16_lo(x[3]) * f)
                  : to_codes(bf16_hi(x[0]) * f, bf16_hi(x[1]) * f, bf16_hi(x[2]) * f, bf16_hi(x[3]) * f);
  };
  uint32_t top = 0;
  if (end - begin == PAGE) {
    const int t0 = NV * (lane / VL);
    uint32_t x[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) x[i] = *reinterpret_cast<const uint32_t *>(src + (t0 + i) * row);
#pragma unroll
    for (int i = 0; i < NV; ++i) top = top_of(top, x[i]);
    scales(top, 0.f, a.v_scale + at, f, again);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < NV; i += 16)
        *reinterpret_cast<u32x4 *>(dst + c * PAGE + t0 + i) = u32x4{codes(c, x + i), codes(c, x + i + 4), codes(c, x + i + 8), codes(c, x + i + 12)};
    return;
  }
  const float old = begin > 0 ? a.v_scale[at] : 0.f;
  for (int t0 = begin; t0 < end; t0 += 8 * VT) {
    uint32_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = t0 + VT * i + lane / VL;
      x[i] = 0;
      if (t < end) x[i] = *reinterpret_cast<const uint32_t *>(src + t * row);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) top = top_of(top, x[i]);
  }
  scales(top, old, a.v_scale + at, f, again);
  // words of four tokens: all of the page's where it is rounded again, those with new tokens otherwise
  const bool all = again != 1.f;
#pragma unroll 2
  for (int t = (all ? 0 : begin & ~3) + 4 * (lane / VL); t < (all ? PAGE : end); t += 4 * VT) {
    uint32_t x[4], mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool is_new = t + e >= begin && t + e < end;
      x[e] = 0;
      if (is_new) x[e] = *reinterpret_cast<const uint32_t *>(src + (t + e) * row);
      mine |= is_new ? 0xFFu << (8 * e) : 0u;
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      uint32_t *const word = reinterpret_cast<uint32_t *>(dst + c * PAGE + t);
      const uint32_t w = codes(c, x);
      if (mine == 0xFFFFFFFFu || all) {
        *word = (w & mine) | (mine == 0xFFFFFFFFu ? 0u : scaled_codes(*word, again) & ~mine);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if ((mine >> (8 * e)) & 1) dst[c * PAGE + t + e] = uint8_t(w >> (8 * e));
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ copies
// 16 KiB of a page's keys, then of its values, per workgroup, all loads before the stores, which pass the caches by (4000 pages of 128 KiB 202 -> 198 us,
// 1400 pages 69 -> 55).  At the rate of a large copy; 16 pages take 3.4 us.
constexpr int COPY_BYTES = 16384;
__global__ __launch_bounds__(256) void ca_cache_copy_kernel(uint8_t *__restrict__ k, uint8_t *__restrict__ v, float *__restrict__ k_scale,
                                                            float *__restrict__ v_scale, const int32_t *__restrict__ src,
                                                            const int32_t *__restrict__ dst, int n_pages, int hkv, int page_bytes,
                                                            int chunks) {
  const int pair = blockIdx.x / (2 * chunks), rest = blockIdx.x % (2 * chunks), at = rest % chunks * COPY_BYTES;
  const int from = src[pair], to = dst[pair];
  if (from < 0 || from >= n_pages || to < 0 || to >= n_pages || from == to) return;
  uint8_t *const p = rest < chunks ? k : v;
  const u32x4 *const x = reinterpret_cast<const u32x4 *>(p + size_t(from) * page_bytes + at);
  u32x4 *const y = reinterpret_cast<u32x4 *>(p + size_t(to) * page_bytes + at);
  const int n = min(COPY_BYTES, page_bytes - at) / 16;
  u32x4 r[COPY_BYTES / 4096];
#pragma unroll
  for (int i = 0; i < COPY_BYTES / 4096; ++i)
    if (256 * i + int(threadIdx.x) < n) r[i] = x[256 * i + threadIdx.x];
#pragma unroll
  for (int i = 0; i < COPY_BYTES / 4096; ++i)
    if (256 * i + int(threadIdx.x) < n) __builtin_nontemporal_store(r[i], y + 256 * i + threadIdx.x);
  if (at == 0) {
    float *const scale = rest < chunks ? k_scale : v_scale;
    for (int h = threadIdx.x; h < hkv; h += 256) scale[size_t(to) * hkv + h] = scale[size_t(from) * hkv + h];
  }
}

// ------------------------------------------------------------------------------------------------ calls
template <int D, int NR, int W>
static int launch_attend(AttendArgs a, void *ws, hipStream_t st) {
  const int workers = n_workers<D, NR, W>(a.hkv, a.s.width > CUT);
  a.by_workers = 1.0001f / float(workers);
  a.heads = static_cast<int4 *>(ws);
  a.parts = reinterpret_cast<float *>(a.heads + size_t(workers) * a.hkv);
  void (*kern)(AttendArgs);
  size_t bytes;  // of LDS, but for the table of sequences
  if constexpr (NR == 8) kern = ca_cache_chunk_kernel<D>, bytes = ChunkSmem<D>::TOTAL;
  else kern = ca_cache_attend_kernel<D, NR, W>, bytes = AttendShape<D, NR, W>::MERGE;
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  static std::atomic<bool> done[16];
  if (e == hipSuccess) e = set_smem(kern, int(bytes + seq_table_bytes(MAX_SEQS)), device, done);
  if (e != hipSuccess) return launched("cache attention", e);
  hipLaunchKernelGGL(kern, dim3(unsigned(a.hkv), unsigned(workers)), dim3(64 * W), bytes + seq_table_bytes(a.s.n_seqs), st, a);
  // (no tile has more pages than the table is wide, and none of up to CUT pages is cut)
  if (a.s.width > CUT) hipLaunchKernelGGL((ca_cache_combine_kernel<D, NR>), dim3(unsigned(a.hkv), unsigned(workers), NR == 8 ? 16 : 4 * NR), dim3(256), 0, st, a);
  return launched("cache attention", hipSuccess);
}

// Rows per tile from the average sequence: up to 32 rows a page is converted by the wave that reads it; with more it is converted once
// per 128 rows, through LDS.
// Waves per worker.  With two or more tiles per CU pairs of waves (four workers per CU, two with 32 rows): while one worker looks its tile up or its waves'
// sums meet, others read (200 sequences of 500 tokens, 8 KV heads of 128: 67 us with eight waves, 48 with four, 41 with two, 41 with one; 64 of 500: 27, 24, 19,
// 25; 32 rows a tile, 200 of 500: 87 with four, 72 with two; contexts of thousands: level).  With fewer tiles a CU has one of its own, which its waves share: four
// where contexts are short (32 sequences of 500: 17.3, 13.5, 15.8, 18.6; one of 901: 12.2, 11.6, 13.6, 20), eight otherwise (16 of 4000: 33, 36, 37, 38).  More
// sequences than fit LDS four times leave pairs to themselves on a CU.
// One kernel serves a call, by this average, also where single tokens and a chunk come together: 32/8 heads of 128, 63 tokens at 4096 (alone 93 us) with a
// chunk of 400 rows (59) take 172 us, with one of 512 (61) 178; 127 tokens (172) with one of 500 (61) 278; 200 tokens at 1000 (81) with one of 500 (40) 107.
template <int D>
static int attend_by_rows(const AttendArgs &a, void *ws, hipStream_t st) {
  const int64_t rows = int64_t(a.s.total) * a.G / a.s.n_seqs, tiles = int64_t(a.s.n_seqs) * a.hkv;
  if (rows > 32) return launch_attend<D, 8, 4>(a, ws, st);
  const bool pairs = tiles >= 2 * N_CU && 4 * (AttendShape<D, 1, 2>::MERGE + seq_table_bytes(a.s.n_seqs)) <= 160 * 1024;
  if (rows > 16) return pairs ? launch_attend<D, 2, 2>(a, ws, st) : launch_attend<D, 2, 4>(a, ws, st);
  return pairs ? launch_attend<D, 1, 2>(a, ws, st) : a.s.width <= 2 * CUT ? launch_attend<D, 1, 4>(a, ws, st) : launch_attend<D, 1, 8>(a, ws, st);
}

}  // namespace ca

extern "C" {

int ca_cache_attend_workspace_bytes(const ca_cache *c, int32_t n_q_heads, size_t *bytes) {
  using namespace ca;
  if (const int rc = check_cache(c); rc != CA_OK) return rc;
  if (!bytes) return fail(CA_ERR_INVALID_ARG, "output is null");
  if (n_q_heads < 1 || n_q_heads % c->n_kv_heads != 0) return fail(CA_ERR_UNSUPPORTED, "n_q_heads is not a multiple of n_kv_heads");
  *bytes = attend_bytes(c);
  return CA_OK;
}

int ca_cache_attend(const ca_cache *c, const ca_cache_batch *b, int32_t n_q_heads, float softmax_scale, int64_t window, int64_t sinks,
                    const void *q, void *o, float *lse, void *ws, size_t ws_bytes, void *hip_stream) {
  using namespace ca;
  if (const int rc = check_cache(c); rc != CA_OK) return rc;
  if (const int rc = check_batch(b); rc != CA_OK) return rc;
  if (n_q_heads < 1 || n_q_heads % c->n_kv_heads != 0) return fail(CA_ERR_UNSUPPORTED, "n_q_heads is not a multiple of n_kv_heads");
  if (window < 0 || sinks < 0) return fail(CA_ERR_INVALID_ARG, "negative window or sinks");
  if (b->n_seqs == 0 || b->total_rows == 0) return CA_OK;
  if (!q || !o) return fail(CA_ERR_INVALID_ARG, "q or o is null");
  if (!aligned(q) || !aligned(o)) return fail(CA_ERR_INVALID_ARG, "q or o is not 16-byte aligned");
  const size_t need = attend_bytes(c);
  if (!ws || ws_bytes < need || reinterpret_cast<uintptr_t>(ws) % 256 != 0) {
    std::ostringstream os;
    os << "workspace of " << (ws ? ws_bytes : 0) << " bytes given, " << need << " needed, 256-byte aligned";
    return fail(CA_ERR_WORKSPACE, os.str());
  }
  const int64_t g = n_q_heads / c->n_kv_heads;
  if ((b->total_rows * g / 16 + b->n_seqs) * std::max(1, b->table_width) >= int64_t(1) << 30)
    return fail(CA_ERR_UNSUPPORTED, "batch: rows times pages beyond 2^30");
  if ((b->total_rows * g + 128) * g >= int64_t(1) << 32) return fail(CA_ERR_UNSUPPORTED, "batch: rows times the square of the heads per KV head beyond 2^32");
  AttendArgs a = {};
  a.s = seq_args(c, b);
  a.k = static_cast<const uint8_t *>(c->k), a.v = static_cast<const uint8_t *>(c->v), a.k_scale = c->k_scale, a.v_scale = c->v_scale;
  a.q = static_cast<const bf16_t *>(q), a.o = static_cast<bf16_t *>(o), a.lse = lse;
  a.hq = n_q_heads, a.hkv = c->n_kv_heads, a.G = int(g), a.by_g = uint32_t(((uint64_t(1) << 32) + uint64_t(g) - 1) / uint64_t(g));
  a.window = window == 0 ? 1 << 30 : int(std::min<int64_t>(window, 1 << 30));
  a.sinks = window == 0 ? 0 : int(std::min<int64_t>(sinks, 1 << 30));
  a.c = (softmax_scale > 0.f ? softmax_scale : c->head_dim == 128 ? 0.08838834764831845f : 0.125f) * 1.4426950408889634f;
  // Codes that the last cache (256 MiB) does not hold until the next call pass it by: 64 sequences of about 4096 tokens, 8 KV heads of 128 (0.9 GB)
  // 166 -> 150 us, 48 of 4096 (0.4 GB) 80 -> 76; those that it holds are read from there (36 of 4096, 0.3 GB: 57 against 60 us; 28: 42, 49).
  // (As many as there may be: what the device's lengths say, the host does not know.)
  const int64_t pages = std::min<int64_t>(int64_t(b->n_seqs) * std::min<int64_t>(b->table_width, (int64_t(a.window) + a.sinks) / PAGE + 3), c->n_pages);
  a.stream = pages * c->n_kv_heads * (2 * PAGE * c->head_dim) > int64_t(384) << 20;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return c->head_dim == 128 ? attend_by_rows<128>(a, ws, st) : attend_by_rows<64>(a, ws, st);
}

int ca_cache_append(const ca_cache *c, const ca_cache_batch *b, const void *k, const void *v, void *hip_stream) {
  using namespace ca;
  if (const int rc = check_cache(c); rc != CA_OK) return rc;
  if (const int rc = check_batch(b); rc != CA_OK) return rc;
  if (b->n_seqs == 0 || b->total_rows == 0 || b->table_width == 0) return CA_OK;
  if (!k || !v) return fail(CA_ERR_INVALID_ARG, "k or v is null");
  if (!aligned(k) || !aligned(v)) return fail(CA_ERR_INVALID_ARG, "k or v is not 16-byte aligned");
  const AppendArgs a = {seq_args(c, b), static_cast<uint8_t *>(c->k), static_cast<uint8_t *>(c->v), c->k_scale, c->v_scale,
                        static_cast<const bf16_t *>(k), static_cast<const bf16_t *>(v), c->n_kv_heads};
  // pages that n rows of a sequence can touch: at most (n - 1) / 64 + 2, and no more than n
  const int64_t touches = std::min<int64_t>(b->total_rows, b->total_rows / PAGE + 2 * int64_t(b->n_seqs));
  const int64_t groups = (touches * 2 * c->n_kv_heads + 3) / 4;
  if (groups > MOST_GROUPS) return fail(CA_ERR_UNSUPPORTED, "batch: rows times KV heads too many");
  const size_t smem = seq_table_bytes(b->n_seqs);
  auto kern = c->head_dim == 128 ? ca_cache_append_kernel<128> : ca_cache_append_kernel<64>;
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  static std::atomic<bool> done[2][16];
  if (e == hipSuccess) e = set_smem(kern, int(seq_table_bytes(MAX_SEQS)), device, done[c->head_dim == 128]);
  if (e != hipSuccess) return launched("cache append", e);
  hipLaunchKernelGGL(kern, dim3(unsigned(groups)), dim3(256), smem, static_cast<hipStream_t>(hip_stream), a);
  return launched("cache append", hipSuccess);
}

int ca_cache_copy_pages(const ca_cache *c, const int32_t *src, const int32_t *dst, int64_t n, void *hip_stream) {
  using namespace ca;
  if (const int rc = check_cache(c); rc != CA_OK) return rc;
  if (n < 0) return fail(CA_ERR_INVALID_ARG, "negative number of pages");
  if (n == 0) return CA_OK;
  if (!src || !dst) return fail(CA_ERR_INVALID_ARG, "src or dst is null");
  // (a workgroup per 16 KiB)
  const int64_t page_bytes = int64_t(c->n_kv_heads) * PAGE * c->head_dim, chunks = (page_bytes + COPY_BYTES - 1) / COPY_BYTES;
  if (n > MOST_GROUPS || 2 * chunks * n > MOST_GROUPS) return fail(CA_ERR_UNSUPPORTED, "too many pages");
  hipLaunchKernelGGL(ca_cache_copy_kernel, dim3(unsigned(2 * chunks * n)), dim3(256), 0, static_cast<hipStream_t>(hip_stream),
                     static_cast<uint8_t *>(c->k), static_cast<uint8_t *>(c->v), c->k_scale, c->v_scale, src, dst, c->n_pages, c->n_kv_heads,
                     int(page_bytes), int(chunks));
  return launched("cache copy", hipSuccess);
}

}  // extern "C"
