// The workgroups of attention over the cache: of single tokens and the like, and of chunks.
#pragma once
#include <algorithm>

#include "ca_cache.h"

namespace ca {

// ------------------------------------------------------------------------------------------------ attention
template <class S>
struct AttendArgsOf {
  S s;
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
using AttendArgs = AttendArgsOf<SeqArgs>;
// PREFIX and TAIL: of tiles that one worker had from their first page to their last, a row and head's sums with {m, l} behind them.
struct SharedArgs : AttendArgsOf<GroupedSeqs> {
  float *row_sums[2];  // [total_rows][n_q_heads][row_floats(D)]
};
constexpr int row_floats(int d) { return d + 4; }

// Rows of a sequence and KV head, token by token and then by head of the group, make up tiles of R = 16 NR; a unit of work is a page
// of a tile.  The units of all sequences, in order, are dealt to the workers in equal runs, whatever the sequences' lengths
// are; a run that ends inside a tile of at most CUT pages is moved to the tile's nearer end, longer tiles are cut.  (A CU takes 1100
// cycles per page that it reads alone, of head_dim 128, and what adding up the parts takes 10 thousand, most of it between launches.)
// Every tile of a sequence counts as many units as the sequence has pages (or the window spans), also where its rows sit early and do not see the
// later ones, which are passed over: a prompt from its first token is dealt unevenly (32/8 heads of 128: one of 2048 rows 91 us, sixteen 1010; their flops
// need 25 and 407), one behind a long context is not.
constexpr int CUT = 16;
constexpr int FAR = 1 << 29;  // the position of rows that see every token there is
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
template <Part P>
struct WorkSplit {
  SeqTableOf<P> tab;
  int total, run, cut, R, G, window, sinks;
  bool stream;  // TAIL: codes pass the caches by
  template <int T, class A>
  __device__ __forceinline__ void count(void *lds, const A &a, int rows) {
    R = rows, G = a.G, window = a.window, sinks = a.sinks;
    total = tab.template fill<T>(lds, a.s, [&](const Seq &q) { return (q.n * G + R - 1) / R * tile_pages(q.len, R, G, window, sinks); });
  }
  // by_workers: a little more than 1 / n_workers
  __device__ __forceinline__ void deal(int n_workers, float by_workers, int least, int longest_whole = CUT) {
    cut = longest_whole;
    run = max(least, n_workers == 1 ? total : __builtin_amdgcn_readfirstlane(int(float(total) * by_workers)) + 1);
  }
  __device__ __forceinline__ int bound(int w) const {
    const int u = min(w * run, total);
    if (u >= total || u == 0) return u;
    const int s = tab.find(u), n = tile_pages(tab.at(s).len, R, G, window, sinks);
    if (n > cut) return u;
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

// Single tokens and the like: tiles of 16 NR rows.  The worker is a workgroup of W waves, or, with W = 1, a wave of any.  A wave has pages of its own, every W-th of the worker's run: codes come to registers
// in 16-byte runs, the next page's K while this one's scores are multiplied, its V behind this one's (a page further ahead took 5 % longer on 64 sequences
// of about 4096 tokens, 7 % on 4 of 130K).  No barrier before the waves' sums meet.
template <Part P, int D, int NR, int W, class A>
__device__ __forceinline__ void attend_workgroup(const A &a, char *smem, const WorkSplit<P> &split, int hk, int worker, float *parts) {
  using S = AttendShape<D, NR, W>;
  constexpr int R = S::R, NH = D / 64, NB = D / 16;
  float *const merge = reinterpret_cast<float *>(smem), *const merge_ml = merge + W * R * S::ROW;
  const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), thread = W == 1 ? lane : threadIdx.x;
  auto sync = [&]() __attribute__((always_inline)) {
    if constexpr (W == 1) wave_sync();
    else __syncthreads();
  };
  const int j4 = lane >> 4, li = lane & 15;
  const int G = a.G;
  const SeqTableOf<P> &tab = split.tab;
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
    const int last_row = min((tile + 1) * R, q.n * G) - 1, pos0 = P == PREFIX ? FAR : q.len - q.n;
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
        if (at * PAGE <= p1) id = a.s.table[size_t(P == PREFIX ? q.more : s) * a.s.width + (P == TAIL ? q.more : 0) + at];
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
        if (P == WHOLE ? a.stream : P == TAIL && split.stream) {
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
        if (P == WHOLE ? a.stream : P == TAIL && split.stream) {
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
    sync();
    const bool whole = n == per_tile;
    const int slot = first == 0 ? 1 : 0;
    float *const part = parts + size_t((worker * 2 + slot) * a.hkv + hk) * (R * (D + 2));
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
      sync();
      for (int i = thread; i < R * S::CW / 4; i += 64 * W) {
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
        if constexpr (P != WHOLE) {
          if (P == PREFIX || q.more > 0) {
            float *const sums = a.row_sums[P == TAIL] + (size_t(q.row0 + token) * a.hq + h) * row_floats(D);
            *reinterpret_cast<f32x4 *>(sums + c0 + col) = y;
            if (stats) sums[D] = top, sums[D + 1] = all;
            continue;
          }
        }
        const float inv = all == 0.f ? 0.f : 1.0f / all;  // (a row that sees nothing: O = 0, LSE = -inf)
        *reinterpret_cast<u32x2 *>(a.o + (size_t(q.row0 + token) * a.hq + h) * D + c0 + col) =
            u32x2{pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv)};
        if (stats && a.lse) a.lse[size_t(h) * a.s.total + q.row0 + token] = 0.6931471805599453f * (top + fast_log2(all));
      }
      if (c0 + S::CW < D || u < end) sync();
    }
  }
  if (P == WHOLE && threadIdx.x == 0) a.heads[worker * a.hkv + hk] = head;
}

// ------------------------------------------------------------------------------------------------ attention of chunks
// Tiles of 128 rows, 32 to a wave.  The waves share a page: each converts a quarter of it to bf16 and puts it into LDS, so that a code is
// converted once per 128 rows, and all read its fragments from there.  The page after the next is on its way to registers, the
// next one is written to the other stage while this one is multiplied; one barrier per page.  K's rows stand in the order of
// the four tiles' rows, V^T's chunks of 8 keys in the order of its fragments, both swizzled as the other kernels' tiles are.
// (4 chunks of 500 rows behind 8192 tokens, 32/8 heads of 128, the whole call: 412 us with 64 rows to a wave of the kernel above, 305 through
// LDS, 258 with fragments fetched ahead and exponentials between MFMAs, 235 now.  MFMAs 38 % busy, vector instructions issue 46 %: conversions,
// exponentials and packing beside them bound it.)  P is one bf16 operand here (its rounding is as large as O's own), or, TWO, two as above: where the rows are
// those of a group of sequences with few rows each, which have two wherever else they are attended.
template <int D>
struct ChunkSmem {
  static constexpr int V_OFF = PAGE * 2 * D, STAGE = 2 * PAGE * 2 * D;
  static constexpr int TOTAL = 2 * STAGE;
  static_assert(4 * PATCH_BYTES <= TOTAL, "patches fit in the stages");
};

template <Part P, int D, bool TWO, class A>
__device__ __forceinline__ void chunk_workgroup(const A &a, char *smem, const WorkSplit<P> &split, int hk, int worker, float *parts) {
  using S = ChunkSmem<D>;
  constexpr int R = 128, NK = D / 32, NB = D / 16, ROWB = 2 * D, NL = D / 64;  // NL: loads of K, and of V, of a wave per page
  const uint32_t lds0 = (uint32_t)(uintptr_t)(CA_LDS char *)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int j4 = lane >> 4, li = lane & 15;
  const int G = a.G;
  const SeqTableOf<P> &tab = split.tab;
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
    const int last_row = min((tile + 1) * R, q.n * G) - 1, pos0 = P == PREFIX ? FAR : q.len - q.n, row_w = tile * R + 32 * wave;
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
        if (at * PAGE <= p1) id = a.s.table[size_t(P == PREFIX ? q.more : s) * a.s.width + (P == TAIL ? q.more : 0) + at];
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
              uint32_t w[2][4], rest[2][4];  // (rest: the second operand, TWO)
              float sum[2] = {0.f, 0.f};
              // probabilities times the scale of V of tile t and row group rg, relative to the reference as it stands
              auto expo = [&](int t, int rg) __attribute__((always_inline)) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = fast_exp2(fmaf(x[t][rg][e], ksi, lvi - m[rg]));
                sum[rg] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                  const uint32_t hi = pack_bf16(p[e], p[e + 1]);
                  w[rg][2 * t + e / 2] = hi;
                  if (TWO) rest[rg][2 * t + e / 2] = pack_bf16(p[e] - __builtin_bit_cast(float, hi << 16), p[e + 1] - __builtin_bit_cast(float, hi & 0xFFFF0000u));
                }
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
              bf16x8 pb[2], pl[2];
#pragma unroll
              for (int rg = 0; rg < 2; ++rg) {
                l[rg] = fmaf(sum[rg], ivi, l[rg]);
                pb[rg] = __builtin_bit_cast(bf16x8, u32x4{w[rg][0], w[rg][1], w[rg][2], w[rg][3]});
                if (TWO) pl[rg] = __builtin_bit_cast(bf16x8, u32x4{rest[rg][0], rest[rg][1], rest[rg][2], rest[rg][3]});
              }
              if (lvi == 0.f && vsi != 1.f) {  // a scale of V that the exponent does not take
#pragma unroll
                for (int rg = 0; rg < 2; ++rg)
#pragma unroll
                  for (int i = 0; i < 8; ++i) {
                    const float x = (TWO ? float(pb[rg][i]) + float(pl[rg][i]) : float(pb[rg][i])) * vsi;
                    pb[rg][i] = bf16_t(x);
                    if (TWO) pl[rg][i] = bf16_t(x - float(pb[rg][i]));
                  }
              }
#pragma unroll
              for (int b = 0; b < NB; ++b) {
#pragma unroll
                for (int rg = 0; rg < 2; ++rg) acc[b][rg] = mfma16(fr[now % AHEAD], pb[rg], acc[b][rg]);
                if (TWO) {
#pragma unroll
                  for (int rg = 0; rg < 2; ++rg) acc[b][rg] = mfma16(fr[now % AHEAD], pl[rg], acc[b][rg]);
                }
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
    bool joined = false;  // (with the other part of what its rows see)
    if constexpr (P != WHOLE) {
      joined = n == per_tile && (P == PREFIX || q.more > 0);
      if (joined) {
#pragma unroll
        for (int rg = 0; rg < 2; ++rg) {
          const int r = row_w + 16 * rg + li, i = a.token_of(r);
          if (r > last_row) continue;
          float *const sums = a.row_sums[P == TAIL] + (size_t(q.row0 + i) * a.hq + hk * G + r - i * G) * row_floats(D);
#pragma unroll
          for (int b = 0; b < NB; ++b) *reinterpret_cast<f32x4 *>(sums + 16 * b + 4 * j4) = acc[b][rg];
          if (j4 == 0) sums[D] = m[rg], sums[D + 1] = sum[rg];
        }
      }
    }
    if (joined) {
    } else if (n == per_tile) {
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
      float *const part = parts + size_t((worker * 2 + slot) * a.hkv + hk) * (R * (D + 2)) + 32 * wave * D;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int rg = 0; rg < 2; ++rg) *reinterpret_cast<f32x4 *>(part + (16 * rg + li) * D + 16 * b + 4 * j4) = acc[b][rg];
      float *const ml = parts + size_t((worker * 2 + slot) * a.hkv + hk) * (R * (D + 2)) + R * D + 64 * wave;
      if (lane < 32) ml[2 * lane] = lane < 16 ? m[0] : m[1], ml[2 * lane + 1] = lane < 16 ? sum[0] : sum[1];
    }
    if (u < end) __syncthreads();  // the patches lie in the stages
  }
  if (P == WHOLE && threadIdx.x == 0) a.heads[worker * a.hkv + hk] = head;
}

// ------------------------------------------------------------------------------------------------ launches
// Workers of W waves per KV head: as many as are on the chip at a time (NR: 16-row groups of a tile; 8: chunks), eight waves to a CU.  Of tiles of
// 32 rows at head_dim 128 four (352 registers: in 256, 23 of them spill, and 64 sequences of about 4096 tokens with 8 rows each take 204 us, not 197;
// at head_dim 64 eight waves take 110, four 176).  Of chunks at head_dim 64 twelve, where tiles are long (4 chunks of 500 rows behind 8192 tokens, 32/8 heads: 224 us
// with eight, 200 with twelve).  Where they are short it goes by how the tiles fill the chip, which this rule does not know: one prompt of 1000, 32/32 heads, 26 us with
// eight and 33 with twelve, sixteen with 8/8 55 and 65; but eight of 512 with 32/8 48 and 36, sixteen of 1000 with 16/16 98 and 74.
template <int D, int NR, int W>
inline int n_workers(int hkv, bool long_tiles = true) {
  return std::max(1, N_CU * (NR == 2 && D == 128 ? 4 : NR == 8 && D == 64 && long_tiles ? 12 : 8) / W / hkv);
}
template <int D, int NR, int W>
inline size_t attend_bytes(int hkv) {
  const size_t workers = size_t(n_workers<D, NR, W>(hkv));
  return workers * hkv * sizeof(int4) + workers * 2 * hkv * (16 * NR * (D + 2)) * 4;
}
template <int D>
inline size_t attend_bytes(int hkv) {
  return std::max({attend_bytes<D, 1, 2>(hkv), attend_bytes<D, 2, 2>(hkv), attend_bytes<D, 8, 4>(hkv)});
}
inline size_t attend_bytes(const ca_cache *c) { return c->head_dim == 128 ? attend_bytes<128>(c->n_kv_heads) : attend_bytes<64>(c->n_kv_heads); }

}  // namespace ca
