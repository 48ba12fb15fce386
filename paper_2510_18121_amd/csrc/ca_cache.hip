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

#include "ca_device.h"
#include "ca_internal.h"
#include "ca_launch.h"

namespace ca {

constexpr int PAGE = CA_CACHE_PAGE_TOKENS;
static_assert(PAGE == 64);
constexpr int MAX_SEQS = 4096;  // their prefix sums lie in LDS
constexpr float NO_MAX = -3.402823466e38f;
constexpr float OUTGROWN = 0x1p20f;
constexpr float LEAST_SCALE = 1.17549435e-38f;  // (a hidden score is -infinity, and that times a scale of 0 would be NaN)

// ------------------------------------------------------------------------------------------------ sequences
// The batch as the kernels see it.  What the device arrays say is clamped to the tensors' sizes: no value reads or writes beyond them.
struct SeqArgs {
  const int32_t *q_start, *kv_len, *table;
  int n_seqs, width, total, n_pages;
};
struct Seq {
  int row0, n, len;  // rows row0 .. row0 + n - 1, at positions len - n .. len - 1
};
__device__ __forceinline__ Seq seq_of(const SeqArgs &a, int s) {
  Seq q;
  q.row0 = min(max(a.q_start[s], 0), a.total);
  q.n = min(max(a.q_start[s + 1], q.row0), a.total) - q.row0;
  q.len = min(max(a.kv_len[s], 0), a.width * PAGE);
  return q;
}

// The sequences as a wave finds them: how many units of work lie before each, and itself, without a trip to memory.  Up to 64 are in
// the lanes of every wave (one token of one sequence: 2.7K cycles to the first unit fewer than through LDS and its barriers), more in LDS.
// (Sums stop growing at MOST_UNITS: only sequences that overlap, against their description, come so far, and then nothing overflows.)
constexpr int MOST_UNITS = (1 << 30) - 1;
__device__ __forceinline__ int sum_units(int a, int b) { return min(a + b, MOST_UNITS); }
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_lanes(int x) {
  return sum_units(x, __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ int wave_prefix(int x) {  // inclusive
  x = add_lanes<0x111, 0xF>(x);  // row_shr 1, 2, 4, 8: inside each 16 lanes
  x = add_lanes<0x112, 0xF>(x);
  x = add_lanes<0x114, 0xF>(x);
  x = add_lanes<0x118, 0xF>(x);
  x = add_lanes<0x142, 0xA>(x);         // the last lane of the 16 before
  return add_lanes<0x143, 0xC>(x);      // ... and of the 32 before
}
constexpr size_t seq_table_bytes(int n_seqs) { return n_seqs <= 64 ? 0 : 64 + size_t(n_seqs + 4) / 4 * 16 * 4; }
struct SeqTable {
  int n_seqs;
  Seq mine;         // up to 64 sequences: of this lane,
  int upto;         // and the units up to it and with it
  int *wave_sums, *pre, *row0, *n, *len;  // more

  // for all threads of the workgroup (T); returns the sum of all units
  template <int T, class F>
  __device__ __forceinline__ int fill(void *lds, const SeqArgs &a, F units) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    n_seqs = a.n_seqs;
    if (n_seqs <= 64) {
      mine = seq_of(a, min(lane, n_seqs - 1));
      upto = wave_prefix(lane < n_seqs ? units(mine) : 0);
      return __builtin_amdgcn_readlane(upto, 63);
    }
    const int stride = (n_seqs + 4) / 4 * 4;
    wave_sums = static_cast<int *>(lds), pre = wave_sums + 16, row0 = pre + stride, n = row0 + stride, len = n + stride;
    int carry = 0;
    for (int base = 0; base < n_seqs; base += T) {
      const int i = base + int(threadIdx.x);
      int x = 0;
      if (i < n_seqs) {
        const Seq q = seq_of(a, i);
        row0[i] = q.row0, n[i] = q.n, len[i] = q.len;
        x = units(q);
      }
      x = wave_prefix(x);
      if (lane == 63) wave_sums[wave] = x;
      __syncthreads();
      int before = carry;
#pragma unroll
      for (int w = 0; w < T / 64; ++w) {
        const int sum = wave_sums[w];
        before = sum_units(before, w < wave ? sum : 0);
        carry = sum_units(carry, sum);
      }
      if (i < n_seqs) pre[i + 1] = sum_units(before, x);
      if (i == 0) pre[0] = 0;
      __syncthreads();
    }
    return __builtin_amdgcn_readfirstlane(carry);
  }
  __device__ __forceinline__ Seq at(int s) const {
    if (n_seqs <= 64) return {__builtin_amdgcn_readlane(mine.row0, s), __builtin_amdgcn_readlane(mine.n, s), __builtin_amdgcn_readlane(mine.len, s)};
    return {__builtin_amdgcn_readfirstlane(row0[s]), __builtin_amdgcn_readfirstlane(n[s]), __builtin_amdgcn_readfirstlane(len[s])};
  }
  __device__ __forceinline__ int before(int s) const {  // units of the sequences before s
    if (n_seqs <= 64) return s == 0 ? 0 : __builtin_amdgcn_readlane(upto, s - 1);
    return __builtin_amdgcn_readfirstlane(pre[s]);
  }
  __device__ __forceinline__ int find(int u) const {  // the sequence that has unit u (less than all units)
    if (n_seqs <= 64) return __builtin_popcountll(__ballot(upto <= u));
    int lo = 0, hi = n_seqs;  // pre[lo] <= u < pre[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid] <= u) lo = mid;
      else hi = mid;
    }
    return __builtin_amdgcn_readfirstlane(lo);
  }
};

// ------------------------------------------------------------------------------------------------ attention
struct AttendArgs {
  SeqArgs s;
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  const bf16_t *q;
  bf16_t *o;
  float *lse;
  float *parts;  // [worker][2][KV head][R rows][D] and then [R][2] {running maximum, sum}
  int4 *heads;   // [worker][KV head], of the tile that begins in this worker and is cut: {parts, first row of its sequence, first and last row}
  int hq, hkv, window, sinks;
  int G;          // query heads per KV head
  uint32_t by_g;  // 2^32 / G, rounded up: x / G is the high word of x * by_g for x < 2^32 / G (G > 1)
  float c;        // softmax_scale * log2(e)
  float by_workers;  // a little more than 1 / (workers per KV head)
  int stream;        // codes pass the caches by

  __device__ __forceinline__ int token_of(int row) const { return G == 1 ? row : int(__umulhi(uint32_t(row), by_g)); }
};

// Rows of a sequence and KV head, token by token and then by head of the group, make up tiles of R = 16 NR; a unit of work is a page
// of a tile.  The units of all sequences, in order, are dealt to the workers in equal runs, whatever the sequences' lengths
// are; a run that ends inside a tile of at most CUT pages is moved to the tile's nearer end, longer tiles are cut.  (A CU takes 1100
// cycles per page that it reads alone, of head_dim 128, and what adding up the parts takes 10 thousand, most of it between launches.)
// Every tile of a sequence counts as many units as the sequence has pages (or the window spans), also where its rows sit early and do not see the
// later ones, which are passed over: a prompt from its first token is dealt unevenly (32/8 heads of 128: one of 2048 rows 91 us, sixteen 1010; their flops
// need 25 and 407), one behind a long context is not.
constexpr int CUT = 16;
__device__ __forceinline__ int tile_pages(int len, int R, int G, int window, int sinks) {
  const int pages = (len + PAGE - 1) / PAGE;
  if (window >= len) return max(1, pages);
  const int tokens = (R + G - 2) / G + 1;  // at most, of a tile
  return max(1, min(pages, (sinks + PAGE - 1) / PAGE + (window + tokens - 2) / PAGE + 2));
}

__device__ __forceinline__ bf16x8 codes_to_bf16(uint32_t a, uint32_t b) {
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  const v2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  const v2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  return bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

// x / y of two uniform numbers, x >= 0, y > 0.  (A 32-bit division is 40 dependent instructions; below 2^24 a quotient in fp32 is off by
// at most one.)
__device__ __forceinline__ int quotient(int x, int y) {
  if (x >= 1 << 24) return x / y;
  const int q = int(float(x) * __builtin_amdgcn_rcpf(float(y))), r = x - q * y;
  return __builtin_amdgcn_readfirstlane(q + (r >= y) - (r < 0));
}

// The workers' shares of the units: worker w has units bound(w) .. bound(w + 1) - 1.
struct WorkSplit {
  SeqTable tab;
  int total, run, R, G, window, sinks;
  template <int T>
  __device__ __forceinline__ void make(void *lds, const AttendArgs &a, int rows, int n_workers, int least) {
    R = rows, G = a.G, window = a.window, sinks = a.sinks;
    total = tab.fill<T>(lds, a.s, [&](const Seq &q) { return (q.n * G + R - 1) / R * tile_pages(q.len, R, G, window, sinks); });
    run = max(least, n_workers == 1 ? total : __builtin_amdgcn_readfirstlane(int(float(total) * a.by_workers)) + 1);
  }
  __device__ __forceinline__ int bound(int w) const {
    const int u = min(w * run, total);
    if (u >= total || u == 0) return u;
    const int s = tab.find(u), n = tile_pages(tab.at(s).len, R, G, window, sinks);
    if (n > CUT) return u;
    const int x = u - tab.before(s), into = x - quotient(x, n) * n;
    return 2 * into < n ? u - into : u - into + n;
  }
};

// Scores x of a page (of row group rg; -infinity where a key is not seen) to the operand of P V; ks and vs: the page's scales, ks with
// the softmax's factor in base 2.  The reference m moves when some row's maximum has grown by more than 2^8 (see the forward kernel).
// P is the sum of two bf16 operands (hi + lo): rounded once more to one alone, O would be off by 1.4 times what its own rounding costs, and
// the matrix pipe is idle most of the time here.
template <int NB, int NR>
__device__ __forceinline__ void softmax_page(const f32x4 (&x)[4][NR], int rg, float ks, float vs, float &m, float &l, f32x4 (&acc)[NB][NR],
                                             bf16x8 (&pb)[2][NR], bf16x8 (&pl)[2][NR]) {
  float top = x[0][rg][0];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = fmaxf(top, x[t][rg][e]);
  top *= ks;
  if (__any(top > m + 8.f)) {
    const float grown = fmaxf(m, quad_max(top)), f = m == NO_MAX ? 0.f : fast_exp2(m - grown);
    m = grown, l *= f;
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b][rg] *= f;
  }
  uint32_t w[2][4], r[2][4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = fast_exp2(fmaf(x[t][rg][e], ks, -m));
    l += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      const float a = p[e] * vs, b = p[e + 1] * vs;
      const uint32_t hi = pack_bf16(a, b);
      w[t >> 1][2 * (t & 1) + e / 2] = hi;
      r[t >> 1][2 * (t & 1) + e / 2] = pack_bf16(a - __builtin_bit_cast(float, hi << 16), b - __builtin_bit_cast(float, hi & 0xFFFF0000u));
    }
  }
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    pb[kk][rg] = __builtin_bit_cast(bf16x8, u32x4{w[kk][0], w[kk][1], w[kk][2], w[kk][3]});
    pl[kk][rg] = __builtin_bit_cast(bf16x8, u32x4{r[kk][0], r[kk][1], r[kk][2], r[kk][3]});
  }
}

template <int D, int NR, int W>
struct AttendShape {
  static constexpr int R = 16 * NR, CW = NR == 1 ? D : 32, ROW = CW + 4;
  static constexpr int MERGE = (W * R * ROW + W * R * 2) * 4;
};

// Single tokens and the like: tiles of 16 NR rows.  A wave has pages of its own, every W-th of the worker's run: codes come to registers
// in 16-byte runs, the next page's K while this one's scores are multiplied, its V behind this one's (a page further ahead took 5 % longer on 64 sequences
// of about 4096 tokens, 7 % on 4 of 130K).  No barrier before the waves' sums meet.
template <int D, int NR, int W>
__global__ __launch_bounds__(64 * W, NR == 1 || D == 64 ? 2 : 1) void ca_cache_attend_kernel(const AttendArgs a) {
  using S = AttendShape<D, NR, W>;
  constexpr int R = S::R, NH = D / 64, NB = D / 16;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float *const merge = reinterpret_cast<float *>(smem), *const merge_ml = merge + W * R * S::ROW;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j4 = lane >> 4, li = lane & 15;
  const int G = a.G, n_workers = gridDim.y, worker = blockIdx.y, hk = blockIdx.x;
  WorkSplit split;
  split.make<64 * W>(smem + S::MERGE, a, R, n_workers, W);
  const SeqTable &tab = split.tab;
  const int begin = split.bound(worker), end = split.bound(worker + 1);
  int4 head = {0, 0, 0, 0};
  const uint32_t k_lane = uint32_t(16 * (li >> 2) + (li & 3)) * D + 16 * j4, v_lane = uint32_t(li) * PAGE + 16 * j4;

  for (int u = begin; u < end;) {
    const int s = tab.find(u), in_seq = u - tab.before(s);
    const Seq q = tab.at(s);
    const int per_tile = tile_pages(q.len, R, G, a.window, a.sinks);
    const int tile = quotient(in_seq, per_tile), first = in_seq - tile * per_tile;
    const int n = min(end - u, per_tile - first);
    u += n;
    // the rows
    const int last_row = min((tile + 1) * R, q.n * G) - 1, pos0 = q.len - q.n;
    const int p0 = pos0 + a.token_of(tile * R), p1 = pos0 + a.token_of(last_row);  // of the tile's first and last row
    const int from = max(0, p0 - a.window + 1);                                    // the first key of a window that some row has
    const int n_sink = min((a.sinks + PAGE - 1) / PAGE, from / PAGE);
    int hi[NR], lo[NR];
    bf16x8 qf[2 * NH][NR];
    f32x4 acc[NB][NR];
    float m[NR], l[NR];
#pragma unroll
    for (int rg = 0; rg < NR; ++rg) {
      m[rg] = NO_MAX, l[rg] = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b][rg] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // pages first + wave, first + wave + W, ..: their ids and scales, 64 at a time, one per lane
    const int n_mine = (n - wave + W - 1) / W;
    for (int base = 0; base == 0 || base < n_mine; base += 64) {
      int id = -1, at = 0;
      if (base + lane < n_mine) {
        const int i = first + wave + W * (base + lane);
        at = i < n_sink ? i : from / PAGE + i - n_sink;
        if (at * PAGE <= p1) id = a.s.table[size_t(s) * a.s.width + at];
        if (id >= a.s.n_pages) id = -1;
      }
      if (base == 0) {
#pragma unroll
        for (int rg = 0; rg < NR; ++rg) {
          const int r = tile * R + 16 * rg + li, ok = r <= last_row, i = ok ? a.token_of(r) : 0, h = hk * G + (ok ? r - i * G : 0);
          hi[rg] = ok ? pos0 + i : -1, lo[rg] = max(0, pos0 + i - a.window + 1);
          const bf16_t *const qp = a.q + (size_t(q.row0 + i) * a.hq + h) * D + 16 * j4;
#pragma unroll
          for (int f = 0; f < 2 * NH; ++f) qf[f][rg] = *reinterpret_cast<const bf16x8 *>(qp + 64 * (f >> 1) + 8 * (f & 1));
        }
      }
      uint64_t left = __ballot(id >= 0);
      auto pop = [&]() __attribute__((always_inline)) {
        if (!left) return -1;
        const int i = __builtin_ctzll(left);
        left &= left - 1;
        return i;
      };
      u32x4 kr[4 * NH], vr[NB];
      auto load_k = [&](int i) __attribute__((always_inline)) {
        const uint8_t *const p = a.k + (size_t(__builtin_amdgcn_readlane(id, i)) * a.hkv + hk) * (PAGE * D);
        if (a.stream) {
          asm volatile("" ::: "memory");  // (two branches, or the loads become one kind)
#pragma unroll
          for (int f = 0; f < 4 * NH; ++f) kr[f] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p + k_lane + 4 * (f / NH) * D + 64 * (f % NH)));
          asm volatile("" ::: "memory");
        } else {
#pragma unroll
          for (int f = 0; f < 4 * NH; ++f) kr[f] = *reinterpret_cast<const u32x4 *>(p + k_lane + 4 * (f / NH) * D + 64 * (f % NH));
        }
      };
      auto load_v = [&](int i) __attribute__((always_inline)) {
        const uint8_t *const p = a.v + (size_t(__builtin_amdgcn_readlane(id, i)) * a.hkv + hk) * (PAGE * D);
        if (a.stream) {
          asm volatile("" ::: "memory");
#pragma unroll
          for (int b = 0; b < NB; ++b) vr[b] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p + v_lane + 16 * PAGE * b));
          asm volatile("" ::: "memory");
        } else {
#pragma unroll
          for (int b = 0; b < NB; ++b) vr[b] = *reinterpret_cast<const u32x4 *>(p + v_lane + 16 * PAGE * b);
        }
      };
      int cur = pop(), next;
      if (cur >= 0) load_k(cur), load_v(cur);
      float ks = 0.f, vs = 0.f;  // (behind the first codes: they are needed later)
      if (id >= 0) ks = fmaxf(a.k_scale[size_t(id) * a.hkv + hk] * a.c, LEAST_SCALE), vs = a.v_scale[size_t(id) * a.hkv + hk];
      for (; cur >= 0; cur = next) {
        next = pop();
        const int i = cur;
        const int key0 = __builtin_amdgcn_readlane(at, i) * PAGE;
        const float ksi = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, ks), i));
        const float vsi = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, vs), i));
        f32x4 x[4][NR];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int f = 0; f < NH; ++f) {
            const u32x4 w = kr[t * NH + f];
            const bf16x8 k0 = codes_to_bf16(w[0], w[1]), k1 = codes_to_bf16(w[2], w[3]);
#pragma unroll
            for (int rg = 0; rg < NR; ++rg) {
              x[t][rg] = mfma16(k0, qf[2 * f][rg], f == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : x[t][rg]);
              x[t][rg] = mfma16(k1, qf[2 * f + 1][rg], x[t][rg]);
            }
          }
        if (next >= 0) load_k(next);
        // some row does not see some key: lane (r, j) holds keys key0 + 16 j + 4 t + e
        if (key0 + PAGE - 1 > p0 || (key0 < p1 - a.window + 1 && key0 + PAGE > a.sinks)) {
          asm volatile("");  // (a branch)
          const int key = key0 + 16 * j4;
#pragma unroll
          for (int rg = 0; rg < NR; ++rg)
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int j = key + 4 * t + e;
                x[t][rg][e] = j <= hi[rg] && (j >= lo[rg] || j < a.sinks) ? x[t][rg][e] : -INFINITY;
              }
          // values of tokens that no row sees count nothing, whatever stands there
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t keep = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = key + 4 * w + e;
              keep |= j <= p1 && (j >= from || j < a.sinks) ? 0xFFu << (8 * e) : 0u;
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) vr[b][w] &= keep;
          }
        }
        bf16x8 pb[2][NR], pl[2][NR];
#pragma unroll
        for (int rg = 0; rg < NR; ++rg) softmax_page<NB>(x, rg, ksi, vsi, m[rg], l[rg], acc, pb, pl);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const bf16x8 v0 = codes_to_bf16(vr[b][0], vr[b][1]), v1 = codes_to_bf16(vr[b][2], vr[b][3]);
#pragma unroll
          for (int rg = 0; rg < NR; ++rg) {
            acc[b][rg] = mfma16(v0, pb[0][rg], acc[b][rg]);
            acc[b][rg] = mfma16(v1, pb[1][rg], acc[b][rg]);
            acc[b][rg] = mfma16(v0, pl[0][rg], acc[b][rg]);
            acc[b][rg] = mfma16(v1, pl[1][rg], acc[b][rg]);
          }
        }
        if (next >= 0) load_v(next);
      }
    }
    // The waves' sums meet in LDS, CW columns at a time.  A tile that this worker has from its first page to its last is done; of
    // any other the sums go to the workspace.
    float sum[NR];
#pragma unroll
    for (int rg = 0; rg < NR; ++rg) {
      sum[rg] = quad_sum(l[rg]);
      if (j4 == 0) merge_ml[wave * R + 16 * rg + li] = m[rg];
    }
    __syncthreads();
    const bool whole = n == per_tile;
    const int slot = first == 0 ? 1 : 0;
    float *const part = a.parts + size_t((worker * 2 + slot) * a.hkv + hk) * (R * (D + 2));
    if (!whole && slot == 1) head = int4{(u - n + per_tile - 1) / split.run - worker + 1, q.row0, tile * R, last_row};
    float factor[NR];
#pragma unroll
    for (int rg = 0; rg < NR; ++rg) {
      float top = NO_MAX;
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, merge_ml[w * R + 16 * rg + li]);
      factor[rg] = m[rg] == NO_MAX ? 0.f : fast_exp2(m[rg] - top);
      if (j4 == 0) merge_ml[(W + wave) * R + 16 * rg + li] = sum[rg] * factor[rg];
    }
    for (int c0 = 0; c0 < D; c0 += S::CW) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
        if (S::CW == D || (b >= c0 / 16 && b < c0 / 16 + S::CW / 16))
#pragma unroll
          for (int rg = 0; rg < NR; ++rg)
            *reinterpret_cast<f32x4 *>(&merge[(wave * R + 16 * rg + li) * S::ROW + 16 * b - c0 + 4 * j4]) = acc[b][rg] * factor[rg];
      __syncthreads();
      for (int i = threadIdx.x; i < R * S::CW / 4; i += 64 * W) {
        const int r = i / (S::CW / 4), col = 4 * (i % (S::CW / 4)), at = tile * R + r;
        if (at > last_row) break;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
          all += merge_ml[(W + w) * R + r];
          y += *reinterpret_cast<const f32x4 *>(&merge[(w * R + r) * S::ROW + col]);
        }
        const bool stats = c0 + col == 0;
        float top = NO_MAX;
        if (stats) {
#pragma unroll
          for (int w = 0; w < W; ++w) top = fmaxf(top, merge_ml[w * R + r]);
        }
        if (!whole) {
          *reinterpret_cast<f32x4 *>(part + r * D + c0 + col) = y;
          if (stats) part[R * D + 2 * r] = top, part[R * D + 2 * r + 1] = all;
          continue;
        }
        const int token = a.token_of(at), h = hk * G + at - token * G;
        const float inv = all == 0.f ? 0.f : 1.0f / all;  // (a row that sees nothing: O = 0, LSE = -inf)
        *reinterpret_cast<u32x2 *>(a.o + (size_t(q.row0 + token) * a.hq + h) * D + c0 + col) =
            u32x2{pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv)};
        if (stats && a.lse) a.lse[size_t(h) * a.s.total + q.row0 + token] = 0.6931471805599453f * (top + fast_log2(all));
      }
      if (c0 + S::CW < D || u < end) __syncthreads();
    }
  }
  if (threadIdx.x == 0) a.heads[worker * a.hkv + hk] = head;
}

// ------------------------------------------------------------------------------------------------ attention of chunks
// Tiles of 128 rows, 32 to a wave.  The waves share a page: each converts a quarter of it to bf16 and puts it into LDS, so that a code is
// converted once per 128 rows, and all read its fragments from there.  The page after the next is on its way to registers, the
// next one is written to the other stage while this one is multiplied; one barrier per page.  K's rows stand in the order of
// the four tiles' rows, V^T's chunks of 8 keys in the order of its fragments, both swizzled as the other kernels' tiles are.
// (4 chunks of 500 rows behind 8192 tokens, 32/8 heads of 128, the whole call: 412 us with 64 rows to a wave of the kernel above, 305 through
// LDS, 258 with fragments fetched ahead and exponentials between MFMAs, 235 now.  MFMAs 38 % busy, vector instructions issue 46 %: conversions,
// exponentials and packing beside them bound it.)  P is one bf16 operand here (its rounding is as large as O's own), not two as above.
template <int D>
struct ChunkSmem {
  static constexpr int V_OFF = PAGE * 2 * D, STAGE = 2 * PAGE * 2 * D;
  static constexpr int TOTAL = 2 * STAGE;
  static_assert(4 * PATCH_BYTES <= TOTAL, "patches fit in the stages");
};

template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void ca_cache_chunk_kernel(const AttendArgs a) {
  using S = ChunkSmem<D>;
  constexpr int R = 128, NK = D / 32, NB = D / 16, ROWB = 2 * D, NL = D / 64;  // NL: loads of K, and of V, of a wave per page
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(CA_LDS char *)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j4 = lane >> 4, li = lane & 15;
  const int G = a.G, n_workers = gridDim.y, worker = blockIdx.y, hk = blockIdx.x;
  WorkSplit split;
  split.make<256>(smem + S::TOTAL, a, R, n_workers, 4);
  const SeqTable &tab = split.tab;
  const int begin = split.bound(worker), end = split.bound(worker + 1);
  int4 head = {0, 0, 0, 0};
  // where the wave's codes come from in a page, and where they go: K row i of tile `wave` is key 16 (i / 4) + 4 wave + i % 4
  uint32_t k_src[NL], k_dst[NL], v_src[NL], v_dst[NL];
#pragma unroll
  for (int n = 0; n < NL; ++n) {
    constexpr int KL = D / 16;  // lanes per row of K
    const int i = 64 / KL * n + lane / KL, piece = lane % KL, d = D / 4 * wave + 16 * n + lane / 4, j = lane % 4;
    k_src[n] = uint32_t(16 * (i >> 2) + 4 * wave + (i & 3)) * D + 16 * piece;
    k_dst[n] = lds0 + (16 * wave + i) * ROWB + 16 * ((2 * piece) ^ tile_sw<D>(i));  // (the second half of the codes: ^ 16)
    v_src[n] = uint32_t(d) * PAGE + 16 * j;
    v_dst[n] = lds0 + S::V_OFF + d * (2 * PAGE) + 16 * (j ^ tile_sw<64>(d));        // (... ^ 64)
  }
  uint32_t koff = lds0 + li * ROWB + 16 * (j4 ^ tile_sw<D>(li)), voff = lds0 + S::V_OFF + li * (2 * PAGE) + 16 * (j4 ^ tile_sw<64>(li)), stage = 0;

  for (int u = begin; u < end;) {
    const int s = tab.find(u), in_seq = u - tab.before(s);
    const Seq q = tab.at(s);
    const int per_tile = tile_pages(q.len, R, G, a.window, a.sinks);
    const int tile = quotient(in_seq, per_tile), first = in_seq - tile * per_tile;
    const int n = min(end - u, per_tile - first);
    u += n;
    // the rows: of the tile, and of the wave (w..)
    const int last_row = min((tile + 1) * R, q.n * G) - 1, pos0 = q.len - q.n, row_w = tile * R + 32 * wave;
    const int p0 = pos0 + a.token_of(tile * R), p1 = pos0 + a.token_of(last_row);
    const int from = max(0, p0 - a.window + 1), n_sink = min((a.sinks + PAGE - 1) / PAGE, from / PAGE);
    const int p0w = pos0 + a.token_of(row_w), p1w = row_w <= last_row ? pos0 + a.token_of(min(row_w + 31, last_row)) : -1;
    const int from_w = max(0, p0w - a.window + 1);
    int hi[2], lo[2];
    bf16x8 qf[NK][2];
#pragma unroll
    for (int rg = 0; rg < 2; ++rg) {
      const int r = row_w + 16 * rg + li, ok = r <= last_row, i = ok ? a.token_of(r) : 0, h = hk * G + (ok ? r - i * G : 0);
      hi[rg] = ok ? pos0 + i : -1, lo[rg] = max(0, pos0 + i - a.window + 1);
      const bf16_t *const qp = a.q + (size_t(q.row0 + i) * a.hq + h) * D + 8 * j4;
#pragma unroll
      for (int f = 0; f < NK; ++f) qf[f][rg] = *reinterpret_cast<const bf16x8 *>(qp + 32 * f);
    }
    f32x4 acc[NB][2];
    float m[2], l[2];
#pragma unroll
    for (int rg = 0; rg < 2; ++rg) {
      m[rg] = NO_MAX, l[rg] = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b) acc[b][rg] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int base = 0; base < n; base += 64) {  // 64 pages at a time: their ids and scales, one per lane
      int id = -1, at = 0;
      float ks = 0.f, vs = 1.f, lv = 0.f, iv = 1.f;
      if (base + lane < n) {
        const int i = first + base + lane;
        at = i < n_sink ? i : from / PAGE + i - n_sink;
        if (at * PAGE <= p1) id = a.s.table[size_t(s) * a.s.width + at];
        if (id >= a.s.n_pages) id = -1;
        if (id >= 0) ks = fmaxf(a.k_scale[size_t(id) * a.hkv + hk] * a.c, LEAST_SCALE), vs = a.v_scale[size_t(id) * a.hkv + hk];
        // The scale of V goes into the exponent: exp2(x - m + lv) = P vs, and their sum times iv is that of P.  Not where that could
        // leave the normal range.
        if (vs > 0x1p-40f && vs < 0x1p40f) lv = fast_log2(vs), iv = fast_exp2(-lv);
      }
      uint64_t left = __ballot(id >= 0);
      u32x4 kr[NL], vr[NL];
      auto pop = [&]() __attribute__((always_inline)) {
        if (!left) return -1;
        const int i = __builtin_ctzll(left);
        left &= left - 1;
        return i;
      };
      auto load = [&](int i) __attribute__((always_inline)) {
        const size_t p = (size_t(__builtin_amdgcn_readlane(id, i)) * a.hkv + hk) * (PAGE * D);
#pragma unroll
        for (int x = 0; x < NL; ++x) kr[x] = *reinterpret_cast<const u32x4 *>(a.k + p + k_src[x]), vr[x] = *reinterpret_cast<const u32x4 *>(a.v + p + v_src[x]);
      };
      auto put = [&](uint32_t stage, int i) __attribute__((always_inline)) {
        const int key0 = __builtin_amdgcn_readlane(at, i) * PAGE;
        if (key0 + PAGE - 1 > p1 || (key0 < from && key0 + PAGE > a.sinks)) {  // values of tokens that no row sees count nothing, whatever stands there
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t keep = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = key0 + 16 * (lane % 4) + 4 * w + e;
              keep |= j <= p1 && (j >= from || j < a.sinks) ? 0xFFu << (8 * e) : 0u;
            }
#pragma unroll
            for (int x = 0; x < NL; ++x) vr[x][w] &= keep;
          }
        }
#pragma unroll
        for (int x = 0; x < NL; ++x) {
          *(CA_LDS bf16x8 *)(stage + k_dst[x]) = codes_to_bf16(kr[x][0], kr[x][1]);
          *(CA_LDS bf16x8 *)(stage + (k_dst[x] ^ 16)) = codes_to_bf16(kr[x][2], kr[x][3]);
          *(CA_LDS bf16x8 *)(stage + v_dst[x]) = codes_to_bf16(vr[x][0], vr[x][1]);
          *(CA_LDS bf16x8 *)(stage + (v_dst[x] ^ 64)) = codes_to_bf16(vr[x][2], vr[x][3]);
        }
      };
      int cur = pop(), next = pop();
      if (cur >= 0) load(cur), put(0, cur);
      if (next >= 0) load(next);
      koff -= stage, voff -= stage, stage = 0;
      barrier_nofence();
      while (cur >= 0) {
        const int after = pop();
        const int key0 = __builtin_amdgcn_readlane(at, cur) * PAGE;
        if (key0 <= p1w && (key0 + PAGE > from_w || key0 < a.sinks)) {
          auto of_page = [&](float x) __attribute__((always_inline)) {
            return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), cur));
          };
          const float ksi = of_page(ks), vsi = of_page(vs), lvi = of_page(lv), ivi = of_page(iv);
          const bool hidden = key0 + PAGE - 1 > p0w || (key0 < p1w - a.window + 1 && key0 + PAGE > a.sinks);  // some row does not see some key
          // Fragments come from LDS AHEAD fragments before the MFMAs that use them: per half of 32 keys 2 NK of K and NB of V^T.  The
          // exponentials of the first tile go between the score MFMAs of the second; fences keep that order.
          constexpr int NF = 2 * NK + NB, AHEAD = 4;
          {
            bf16x8 fr[AHEAD];
            auto fetch = [&](int i) __attribute__((always_inline)) -> bf16x8 {
              const int kk = i / NF, f = i % NF;
              return f < 2 * NK ? lds_read8_at((koff ^ (64 * (f % NK))) + 16 * (2 * kk + f / NK) * ROWB)
                                : lds_read8_at((voff ^ (64 * kk)) + 16 * (f - 2 * NK) * (2 * PAGE));
            };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) fr[i] = fetch(i);
            int now = 0;  // the fragment in use
            auto advance = [&]() __attribute__((always_inline)) {
              if (now + AHEAD < 2 * NF) fr[now % AHEAD] = fetch(now + AHEAD);
              ++now;
              __builtin_amdgcn_sched_barrier(0);
            };
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
              f32x4 x[2][2];
              uint32_t w[2][4];
              float sum[2] = {0.f, 0.f};
              // probabilities times the scale of V of tile t and row group rg, relative to the reference as it stands
              auto expo = [&](int t, int rg) __attribute__((always_inline)) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = fast_exp2(fmaf(x[t][rg][e], ksi, lvi - m[rg]));
                sum[rg] += (p[0] + p[1]) + (p[2] + p[3]);
                w[rg][2 * t] = pack_bf16(p[0], p[1]), w[rg][2 * t + 1] = pack_bf16(p[2], p[3]);
              };
              auto mask = [&](int t) __attribute__((always_inline)) {  // lane (r, j) holds keys key0 + 16 j + 8 kk + 4 t + e
                if (!hidden) return;
                asm volatile("");  // (a branch, not 16 selects on every page)
#pragma unroll
                for (int rg = 0; rg < 2; ++rg) {
                  const int base = key0 + 16 * j4 + 8 * kk + 4 * t, vis = hi[rg] - base, begins = lo[rg] - base, sink_end = a.sinks - base;
#pragma unroll
                  for (int e = 0; e < 4; ++e) x[t][rg][e] = e <= vis && (e >= begins || e < sink_end) ? x[t][rg][e] : -INFINITY;
                }
              };
#pragma unroll
              for (int f = 0; f < 2 * NK; ++f) {
                const int t = f / NK;
                if (f == NK) mask(0);
#pragma unroll
                for (int rg = 0; rg < 2; ++rg) x[t][rg] = mfma16(fr[now % AHEAD], qf[f % NK][rg], f % NK == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : x[t][rg]);
                if (t == 1) {
#pragma unroll
                  for (int rg = 2 * (f - NK) / NK; rg < 2 * (f - NK + 1) / NK; ++rg) expo(0, rg);
                }
                advance();
              }
              mask(1);
#pragma unroll
              for (int rg = 0; rg < 2; ++rg) {
                expo(1, rg);
                __builtin_amdgcn_sched_barrier(0);
              }
              // The reference is moved when it has been outgrown by far (or there is none yet): probabilities relative to a stale one are
              // merely larger numbers.
              if (__any(!(sum[0] * ivi < OUTGROWN && sum[1] * ivi < OUTGROWN))) {
#pragma unroll
                for (int rg = 0; rg < 2; ++rg) {
                  float top = x[0][rg][0];
#pragma unroll
                  for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, x[t][rg][e]);
                  const float grown = fmaxf(m[rg], quad_max(top * ksi)), f = m[rg] == NO_MAX ? 0.f : fast_exp2(m[rg] - grown);
                  m[rg] = grown, l[rg] *= f, sum[rg] = 0.f;
#pragma unroll
                  for (int b = 0; b < NB; ++b) acc[b][rg] *= f;
                  expo(0, rg), expo(1, rg);
                }
              }
              bf16x8 pb[2];
#pragma unroll
              for (int rg = 0; rg < 2; ++rg) {
                l[rg] = fmaf(sum[rg], ivi, l[rg]);
                pb[rg] = __builtin_bit_cast(bf16x8, u32x4{w[rg][0], w[rg][1], w[rg][2], w[rg][3]});
              }
              if (lvi == 0.f && vsi != 1.f) {  // a scale of V that the exponent does not take
#pragma unroll
                for (int rg = 0; rg < 2; ++rg)
#pragma unroll
                  for (int i = 0; i < 8; ++i) pb[rg][i] = bf16_t(float(pb[rg][i]) * vsi);
              }
#pragma unroll
              for (int b = 0; b < NB; ++b) {
#pragma unroll
                for (int rg = 0; rg < 2; ++rg) acc[b][rg] = mfma16(fr[now % AHEAD], pb[rg], acc[b][rg]);
                advance();
              }
            }
          }
        }
        if (next >= 0) {
          put(S::STAGE - stage, next);
          if (after >= 0) load(after);
        }
        cur = next, next = after;
        koff += S::STAGE - 2 * stage, voff += S::STAGE - 2 * stage;
        stage = S::STAGE - stage;
        barrier_nofence();
      }
    }
    const float sum[2] = {quad_sum(l[0]), quad_sum(l[1])};
    if (n == per_tile) {
      const float f0 = sum[0] == 0.f ? 0.f : 1.0f / sum[0], f1 = sum[1] == 0.f ? 0.f : 1.0f / sum[1];
      store_tile16_as_lines<0>(lds0 + wave * PATCH_BYTES, acc, f0, f1, lane, [&](int p) __attribute__((always_inline)) -> bf16_t * {
        const int r = row_w + p, i = a.token_of(r);
        return r <= last_row ? a.o + (size_t(q.row0 + i) * a.hq + hk * G + r - i * G) * D : nullptr;
      });
      const int r = row_w + lane, i = a.token_of(r);
      if (lane < 32 && r <= last_row && a.lse)
        a.lse[size_t(hk * G + r - i * G) * a.s.total + q.row0 + i] = 0.6931471805599453f * ((lane < 16 ? m[0] : m[1]) + fast_log2(lane < 16 ? sum[0] : sum[1]));
    } else {
      const int slot = first == 0 ? 1 : 0;
      if (slot == 1) head = int4{(u - n + per_tile - 1) / split.run - worker + 1, q.row0, tile * R, last_row};
      float *const part = a.parts + size_t((worker * 2 + slot) * a.hkv + hk) * (R * (D + 2)) + 32 * wave * D;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int rg = 0; rg < 2; ++rg) *reinterpret_cast<f32x4 *>(part + (16 * rg + li) * D + 16 * b + 4 * j4) = acc[b][rg];
      float *const ml = a.parts + size_t((worker * 2 + slot) * a.hkv + hk) * (R * (D + 2)) + R * D + 64 * wave;
      if (lane < 32) ml[2 * lane] = lane < 16 ? m[0] : m[1], ml[2 * lane + 1] = lane < 16 ? sum[0] : sum[1];
    }
    if (u < end) __syncthreads();  // the patches lie in the stages
  }
  if (threadIdx.x == 0) a.heads[worker * a.hkv + hk] = head;
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
static int fail(int code, const std::string &msg) {
  set_error(msg);
  return code;
}
static bool aligned(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
constexpr int64_t MOST_GROUPS = (int64_t(1) << 24) - 1;  // workgroups of 256 threads of a launch, whose threads number less than 2^32
static int check_cache(const ca_cache *c) {
  if (!c) return fail(CA_ERR_INVALID_ARG, "cache is null");
  if (c->head_dim != 64 && c->head_dim != 128) return fail(CA_ERR_UNSUPPORTED, "head_dim not supported (64 or 128)");
  if (c->n_pages < 0 || c->n_kv_heads < 1) return fail(CA_ERR_INVALID_ARG, "cache: n_pages must not be negative, n_kv_heads at least 1");
  if (c->n_kv_heads > 1024) return fail(CA_ERR_UNSUPPORTED, "cache: more than 1024 KV heads");
  if (c->n_pages > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return fail(CA_ERR_INVALID_ARG, "cache: k, v, k_scale or v_scale is null");
  if (!aligned(c->k) || !aligned(c->v)) return fail(CA_ERR_INVALID_ARG, "cache: k or v is not 16-byte aligned");
  return CA_OK;
}
static int check_batch(const ca_cache_batch *b) {
  if (!b) return fail(CA_ERR_INVALID_ARG, "batch is null");
  if (b->n_seqs < 0 || b->table_width < 0 || b->total_rows < 0) return fail(CA_ERR_INVALID_ARG, "batch: negative size");
  if (b->n_seqs > MAX_SEQS) return fail(CA_ERR_UNSUPPORTED, "batch: more than 4096 sequences");
  if (b->table_width > (1 << 23)) return fail(CA_ERR_UNSUPPORTED, "batch: table_width beyond 2^23 pages");
  if (b->total_rows >= (int64_t(1) << 30)) return fail(CA_ERR_UNSUPPORTED, "batch: total_rows beyond 2^30");
  if (b->n_seqs > 0 && (!b->q_start || !b->kv_len || (b->table_width > 0 && !b->page_table)))
    return fail(CA_ERR_INVALID_ARG, "batch: q_start, kv_len or page_table is null");
  return CA_OK;
}
static SeqArgs seq_args(const ca_cache *c, const ca_cache_batch *b) {
  return {b->q_start, b->kv_len, b->page_table, b->n_seqs, b->table_width, int(b->total_rows), c->n_pages};
}
static int launched(const char *what, hipError_t e) {
  if (e == hipSuccess) e = hipGetLastError();
  if (e == hipSuccess) return CA_OK;
  return fail(CA_ERR_HIP, std::string(what) + ": " + hipGetErrorName(e) + " (" + hipGetErrorString(e) + ")");
}

// Workers of W waves per KV head: as many as are on the chip at a time (NR: 16-row groups of a tile; 8: chunks), eight waves to a CU.  Of tiles of
// 32 rows at head_dim 128 four (352 registers: in 256, 23 of them spill, and 64 sequences of about 4096 tokens with 8 rows each take 204 us, not 197;
// at head_dim 64 eight waves take 110, four 176).  Of chunks at head_dim 64 twelve, where tiles are long (4 chunks of 500 rows behind 8192 tokens, 32/8 heads: 224 us
// with eight, 200 with twelve).  Where they are short it goes by how the tiles fill the chip, which this rule does not know: one prompt of 1000, 32/32 heads, 26 us with
// eight and 33 with twelve, sixteen with 8/8 55 and 65; but eight of 512 with 32/8 48 and 36, sixteen of 1000 with 16/16 98 and 74.
template <int D, int NR, int W>
static int n_workers(int hkv, bool long_tiles = true) {
  return std::max(1, N_CU * (NR == 2 && D == 128 ? 4 : NR == 8 && D == 64 && long_tiles ? 12 : 8) / W / hkv);
}
template <int D, int NR, int W>
static size_t attend_bytes(int hkv) {
  const size_t workers = size_t(n_workers<D, NR, W>(hkv));
  return workers * hkv * sizeof(int4) + workers * 2 * hkv * (16 * NR * (D + 2)) * 4;
}
template <int D>
static size_t attend_bytes(int hkv) {
  return std::max({attend_bytes<D, 1, 2>(hkv), attend_bytes<D, 2, 2>(hkv), attend_bytes<D, 8, 4>(hkv)});
}
static size_t attend_bytes(const ca_cache *c) { return c->head_dim == 128 ? attend_bytes<128>(c->n_kv_heads) : attend_bytes<64>(c->n_kv_heads); }

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
