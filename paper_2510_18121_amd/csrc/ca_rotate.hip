// Queries and keys on their way to attention: the norm of each head and the turn by the row's position, in one pass, and its gradients.
//
// Of a head x of D columns at position p, with gain g:
//   u = g x / sqrt(mean(x^2) + eps)  (u = x without a gain);   y = R(p) u
// R(p) turns pair i < rot / 2 of the first rot columns, (i, i + rot / 2) or (2 i, 2 i + 1), by the angle p f_i and multiplies it by `factor`; the
// other columns stay.  Backward, with dy: du = R(p)^T dy;  dg = sum over rows and heads of du xh, xh = x / sqrt(..);
//   dx = (g du - xh mean(g du xh)) / sqrt(..)  (dx = du without a gain).
// Frequencies are turns per position in units of 2^-64, so that p f mod 1 is exact for every p, also a million tokens on, where an angle in fp32 is off by
// 0.06; of it 32 bits are taken, reduced to an eighth of a turn and put into the series of sine and cosine (below 3e-8 off).
//
// Bound by HBM: 4 bytes per element forward, 6 backward (4 without a gain), some ten operations for each.  A wave holds 1024 elements, 16 to a lane, so that
// a pair is a lane's own (HALF: two runs of 8 columns half the turned ones apart; INTERLEAVED: neighbours), and a row's sines and cosines are computed once, one per
// lane, and handed out through the wave's LDS.  Measured (32/8 heads of 128 unless noted; a copy of 512 MB in turn: 5.3 to 5.6 TB/s):
//   forward    65536 rows with gains 228 to 238 us, 5.6 to 5.9 TB/s; 40001 out of a joint projection 140 to 148
//   backward   65536 rows with gains 357 to 367 us, 5.5 TB/s; 16411 rows of 16/16 heads of 64: 27 forward, 38 to 48 backward
//   half of each head of 128 turned in halves 298 and 420, whose lanes read runs that are further apart; a number of pairs that is no multiple of 8, through LDS:
//   120 or 38 columns of 128 250 to 257 forward, 407 to 419 backward; 58 or 26 of 64 of the 16411 rows 32 and 61 to 64
//   without gains 65536 rows 232 and 235, 16411 rows 24 and 24
//   one row 3.1 us, 250 rows of 64/8 heads 5.1 (a launch, and the trips to memory for the position and the row)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <sstream>

#include "ca_device.h"
#include "ca_internal.h"

namespace ca {

// Workgroups of a tensor.  (Half of them or twice as many: within 3 % on 65536 rows of 40 heads of 128, 29 to 30 us on 16411 of 32 of 64; a bound of 6 waves per
// SIMD spills: 810 us backward.)
constexpr int MOST_BLOCKS = N_CU * 4;
// What is read and written together beyond this passes the last cache (256 MiB) by.  (65536 rows of 40 heads of 128, 1.3 GB: 252 -> 237 us forward, 390 -> 367 backward;
// 16411 of 32 of 64, 0.13 GB, which the cache does hold: 29 -> 32 and 48 -> 50.)
constexpr int64_t STREAM_BYTES = int64_t(384) << 20;

enum Layout { HALF, INTERLEAVED, HALF_ANY };  // HALF: rot / 2 is a multiple of 8; HALF_ANY: of anything

struct RotateTensor {
  const bf16_t *x, *dy;  // (dy: backward)
  bf16_t *y;             // forward: y; backward: dx
  const float *gain;
  float *dgain;        // partial sums [workgroup][D], backward
  const int32_t *pos;  // or nullptr: by the sequences
  int64_t rows, x_stride, y_stride, dy_stride;
  int heads, segments, blocks;  // waves per row; workgroups
  int gaps;                     // rows at position CA_ROTATE_GAP are of nobody
};
struct RotateArgs {
  RotateTensor t[2];
  const uint64_t *turns;
  const int32_t *q_start, *kv_len;
  int n_seqs, rot;
  float eps, factor;
};

// The position of a row of the sequences; false where it is of none.  A wave looks at 64 sequences at a time.
__device__ __forceinline__ bool position_in_sequence(const RotateArgs &a, int64_t rows, int64_t row, int lane, int &pos) {
  int base = 0;
  if (a.n_seqs >= 64) {
    const int n = __builtin_popcountll(__ballot(lane * 64 <= a.n_seqs && a.q_start[min(lane * 64, a.n_seqs)] <= row));
    // (with 4096 sequences the last entry, the end of them all, is none of the 64)
    if (n == 0) return false;
    base = (n - 1) * 64;
  }
  const int n = __builtin_popcountll(__ballot(base + lane <= a.n_seqs && a.q_start[min(base + lane, a.n_seqs)] <= row));
  const int s = base + n - 1;
  if (n == 0 || s >= a.n_seqs) return false;
  const int64_t end = min(int64_t(a.q_start[s + 1]), rows);
  if (row >= end) return false;
  pos = int(a.kv_len[s] - (end - row));
  return true;
}

// Sine and cosine of p f: of the angle's 64 bits of a turn the upper 32, less the nearest quarter.  (The series end where they are 3e-8 off, at an
// eighth of a turn.)
__device__ __forceinline__ f32x2 cos_sin(int pos, uint64_t turns) {
  const uint32_t lo = uint32_t(turns), hi = uint32_t(turns >> 32);
  const uint32_t t = uint32_t(pos) * hi + __umulhi(uint32_t(pos), lo) - (pos < 0 ? lo : 0u);
  const uint32_t quarter = (t + 0x20000000u) >> 30;
  const float x = float(int32_t(t - (quarter << 30))) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float z = x * x;
  const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), x);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 2.4801587e-5f, -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
  const bool swap = quarter & 1;
  const float cc = swap ? s : c, ss = swap ? c : s;
  return f32x2{quarter == 1 || quarter == 2 ? -cc : cc, quarter >= 2 ? -ss : ss};
}

__device__ __forceinline__ void unpack(const u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = __builtin_bit_cast(float, w[i] << 16), x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
}
__device__ __forceinline__ u32x4 packed(const float (&x)[8]) {
  return u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}

template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
// the sum over the lanes of a head (4 or 8 neighbours)
template <int LANES>
__device__ __forceinline__ float head_sum(float x) {
  x = add_dpp<0xB1>(x);                           // lane ^ 1
  x = add_dpp<0x4E>(x);                           // lane ^ 2
  return LANES == 8 ? add_dpp<0x141>(x) : x;      // 7 - lane: of the other four
}

// A wave's own LDS: cosines and sines of the row's pairs, and, for HALF_ANY, the heads in flight.
template <int D, Layout L>
struct RotateSmem {
  f32x2 cs[D / 2];
  float x[L == HALF_ANY ? 1024 : 1];
};

// What a lane holds of a head: 8 columns from col_a on and 8 from col_b on, of D / 16 lanes.  HALF: the two are pairs (or none is turned).
template <int D, Layout L>
struct Turner {
  int col_a, col_b, rot, slot;
  bool turned;
  f32x2 cs[L == HALF_ANY ? 16 : 8];
  __device__ __forceinline__ Turner(int lane, int r) : rot(r), slot(lane / (D / 16)) {
    const int p = lane % (D / 16), h = r / 16;
    if (L == HALF) {
      turned = p < h;
      col_a = 8 * (turned ? p : p + h), col_b = 8 * (turned ? p + h : p + D / 16);
    } else {
      turned = true;
      col_a = 8 * p, col_b = 8 * p + D / 2;
    }
  }
  // takes the row's cosines and sines
  __device__ __forceinline__ void take(const f32x2 *row) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (L == HALF) cs[e] = turned ? row[col_a + e] : f32x2{1.f, 0.f};
      if (L == INTERLEAVED) cs[e] = row[(e < 4 ? col_a : col_b) / 2 + e % 4];
      if (L == HALF_ANY)
        for (int s = 0; s < 2; ++s) {
          const int c = (s ? col_b : col_a) + e, half = rot / 2;
          cs[8 * s + e] = row[c < half ? c : c < rot ? c - half : 0];
        }
    }
  }
  // turns a head's columns by SIGN times the angles
  template <int SIGN>
  __device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], float *lds) const {
    if (L == HALF) {
      if (!turned) return;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float c = cs[e][0], s = SIGN * cs[e][1], x = a[e], y = b[e];
        a[e] = x * c - y * s, b[e] = x * s + y * c;
      }
    } else if (L == INTERLEAVED) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float *const v = e < 4 ? a : b;
        const int i = 2 * (e % 4), col = (e < 4 ? col_a : col_b) + i;
        const float c = cs[e][0], s = SIGN * cs[e][1], x = v[i], y = v[i + 1];
        if (col < rot) v[i] = x * c - y * s, v[i + 1] = x * s + y * c;
      }
    } else {
      float *const head = lds + slot * D;
      const int half = rot / 2;
#pragma unroll
      for (int e = 0; e < 8; ++e) head[col_a + e] = a[e], head[col_b + e] = b[e];
      wave_sync();
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        float &v = k < 8 ? a[k % 8] : b[k % 8];
        const int col = (k < 8 ? col_a : col_b) + k % 8;
        const float c = cs[k][0], s = SIGN * cs[k][1];
        const float other = head[col < half ? col + half : col < rot ? col - half : col];
        if (col < half) v = v * c - other * s;
        else if (col < rot) v = v * c + other * s;
      }
      wave_sync();
    }
  }
};

// A wave takes a row's heads, or a run of them, 1024 elements at a time, and then those of a row further on; the elements after the next are on their
// way while it works.  STREAM: tensors that the last cache does not hold until somebody reads them pass it by.
template <int D, Layout L, bool BACKWARD, bool STREAM>
__global__ __launch_bounds__(256) void ca_rotate_kernel(const RotateArgs a) {
  constexpr int LANES = D / 16, SLOTS = 64 / LANES;  // of a head; heads at a time
  __shared__ RotateSmem<D, L> smem[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool second = int(blockIdx.x) >= a.t[0].blocks;
  const RotateTensor &t = a.t[second];
  const int block = int(blockIdx.x) - (second ? a.t[0].blocks : 0);
  const int w = block * 4 + wave, segments = t.segments, segment = w % segments;
  const int chunks = (t.heads + SLOTS - 1) / SLOTS, per = (chunks + segments - 1) / segments;
  const int first = segment * per * SLOTS, end = min(t.heads, first + per * SLOTS);
  const int64_t stride = max(1, t.blocks * 4 / segments);
  Turner<D, L> turner(lane, a.rot);
  const uint64_t turns = lane < a.rot / 2 ? a.turns[lane] : 0;
  RotateSmem<D, L> &mine = smem[wave];
  float ga[8], gb[8], da[8], db[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    ga[e] = t.gain ? t.gain[turner.col_a + e] : 1.f, gb[e] = t.gain ? t.gain[turner.col_b + e] : 1.f;
    da[e] = db[e] = 0.f;
  }
  auto get = [&](const bf16_t *p) __attribute__((always_inline)) {
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
    else return *reinterpret_cast<const u32x4 *>(p);
  };
  auto put = [&](bf16_t *p, const u32x4 &v) __attribute__((always_inline)) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p));
    else *reinterpret_cast<u32x4 *>(p) = v;
  };
  struct Raw {
    u32x4 a, b, xa, xb;  // x, or dy and with a gain x
  };
  auto load = [&](int64_t row, int h0) __attribute__((always_inline)) {
    const int h = h0 + turner.slot;
    const int64_t at = int64_t(h < end ? h : h0) * D;
    const bf16_t *const src = (BACKWARD ? t.dy + row * t.dy_stride : t.x + row * t.x_stride) + at;
    Raw r;
    r.a = get(src + turner.col_a), r.b = get(src + turner.col_b);
    if (BACKWARD && t.gain) {
      const bf16_t *const xs = t.x + row * t.x_stride + at;
      r.xa = get(xs + turner.col_a), r.xb = get(xs + turner.col_b);
    }
    return r;
  };
  int64_t row = w / segments;
  int h0 = first;
  bool more = row < t.rows && w / segments < stride && first < end, known = false;
  Raw next = {};
  int pos = 0, next_pos = 0;
  if (more) {
    next = load(row, h0);
    if (t.pos) next_pos = t.pos[row];
  }
  while (more) {
    const Raw now = next;
    const int64_t this_row = row;
    const int this_h0 = h0;
    const bool new_row = h0 == first;
    if (new_row) {
      pos = next_pos, known = !t.gaps || pos != CA_ROTATE_GAP;
      if (!t.pos) known = position_in_sequence(a, t.rows, row, lane, pos);
    }
    h0 += SLOTS;
    if (h0 >= end) h0 = first, row += stride;
    more = row < t.rows;
    if (more) {
      next = load(row, h0);
      if (t.pos && h0 == first) next_pos = t.pos[row];
    }
    if (!known) continue;  // a row of no sequence, a gap
    if (new_row) {
      if (lane < D / 2) mine.cs[lane] = cos_sin(pos, turns) * a.factor;
      wave_sync();
      turner.take(mine.cs);
      wave_sync();
    }
    const int h = this_h0 + turner.slot;
    const bool there = h < end;
    float xa[8], xb[8];
    unpack(now.a, xa), unpack(now.b, xb);
    if (!BACKWARD) {
      if (t.gain) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], sum));
        const float r = rsqrtf(fmaf(head_sum<LANES>(sum), 1.f / D, a.eps));
#pragma unroll
        for (int e = 0; e < 8; ++e) xa[e] *= r * ga[e], xb[e] *= r * gb[e];
      }
      turner.template turn<1>(xa, xb, mine.x);
    } else {
      turner.template turn<-1>(xa, xb, mine.x);
      if (t.gain) {
        float va[8], vb[8];
        unpack(now.xa, va), unpack(now.xb, vb);
        float sum = 0.f, dot = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sum = fmaf(va[e], va[e], fmaf(vb[e], vb[e], sum));
          dot = fmaf(xa[e] * ga[e], va[e], fmaf(xb[e] * gb[e], vb[e], dot));
        }
        const float r = rsqrtf(fmaf(head_sum<LANES>(sum), 1.f / D, a.eps));
        const float mean = head_sum<LANES>(dot) * (r * r) * (1.f / D);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (there) da[e] = fmaf(xa[e] * r, va[e], da[e]), db[e] = fmaf(xb[e] * r, vb[e], db[e]);
          xa[e] = r * fmaf(-mean, va[e], xa[e] * ga[e]), xb[e] = r * fmaf(-mean, vb[e], xb[e] * gb[e]);
        }
      }
    }
    if (there) {
      bf16_t *const dst = t.y + this_row * t.y_stride + int64_t(h) * D;
      put(dst + turner.col_a, packed(xa)), put(dst + turner.col_b, packed(xb));
    }
  }
  if (!BACKWARD || !t.gain) return;
  // the workgroup's sum of dg: over the wave's heads, then over the waves, in order
  __shared__ float sums[4][D];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int o = LANES; o < 64; o <<= 1) da[e] += __shfl_xor(da[e], o), db[e] += __shfl_xor(db[e], o);
    if (lane < LANES) sums[wave][turner.col_a + e] = da[e], sums[wave][turner.col_b + e] = db[e];
  }
  __syncthreads();
  if (threadIdx.x < D)
    t.dgain[size_t(block) * D + threadIdx.x] = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
}

// dg of each tensor from the workgroups' sums, four columns to a workgroup, in a fixed order.  (4 to 5.5 us; 16 columns to a workgroup of 1024 threads, which
// read one sum after the other, 11 and 19.)
struct GainSums {
  const float *parts[2];
  float *out[2];
  int n[2];
};
template <int D>
__global__ __launch_bounds__(256) void ca_rotate_gain_kernel(const GainSums a) {
  __shared__ f32x4 sums[256];
  const int which = blockIdx.y, i0 = threadIdx.x;
  if (!a.out[which]) return;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < MOST_BLOCKS / 256; ++k) {
    const int i = i0 + 256 * k;
    if (i < a.n[which]) sum += *reinterpret_cast<const f32x4 *>(a.parts[which] + size_t(i) * D + 4 * blockIdx.x);
  }
  sums[i0] = sum;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (i0 < o) sums[i0] += sums[i0 + o];
    __syncthreads();
  }
  if (i0 < 4) a.out[which][4 * blockIdx.x + i0] = sums[0][i0];
}

// ------------------------------------------------------------------------------------------------ calls
static int refuse(int code, const std::string &msg) {
  set_error(msg);
  return code;
}
static bool whole_lines(const void *p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0; }

static int check_rotation(const ca_rotation *r) {
  if (!r) return refuse(CA_ERR_INVALID_ARG, "rotation is null");
  if (r->head_dim != 64 && r->head_dim != 128) return refuse(CA_ERR_UNSUPPORTED, "head_dim not supported (64 or 128)");
  if (r->rot_dim < 0 || r->rot_dim > r->head_dim || r->rot_dim % 2 != 0) return refuse(CA_ERR_INVALID_ARG, "rotation: rot_dim is not an even number up to head_dim");
  if (r->rot_dim > 0 && !r->turns) return refuse(CA_ERR_INVALID_ARG, "rotation: turns is null");
  return CA_OK;
}

// One tensor of a call, checked; rows, and heads where there are rows.
static int check_tensor(const ca_rotate_tensor &s, int d, bool backward, bool by_sequences, const char *name) {
  auto say = [&](int code, const char *what) { return refuse(code, std::string(name) + ": " + what); };
  if (s.rows < 0) return say(CA_ERR_INVALID_ARG, "negative number of rows");
  if (s.rows == 0) return CA_OK;
  if (s.heads < 1 || s.heads > 65536) return say(CA_ERR_INVALID_ARG, "heads: 1 to 65536");
  if (s.rows >= int64_t(1) << 31) return say(CA_ERR_UNSUPPORTED, "rows beyond 2^31");
  const int64_t width = int64_t(s.heads) * d;
  if ((!backward || s.gain) && (!s.x || !whole_lines(s.x, s.x_stride) || s.x_stride < width))
    return say(CA_ERR_INVALID_ARG, "x is null, not 16-byte aligned, or its rows are (a stride is a multiple of 8 elements, at least heads x head_dim)");
  if (!s.y || !whole_lines(s.y, s.y_stride) || s.y_stride < width)
    return say(CA_ERR_INVALID_ARG, "the output is null, not 16-byte aligned, or its rows are (a stride is a multiple of 8 elements, at least heads x head_dim)");
  if (backward && (!s.dy || !whole_lines(s.dy, s.dy_stride) || s.dy_stride < width))
    return say(CA_ERR_INVALID_ARG, "dy is null, not 16-byte aligned, or its rows are (a stride is a multiple of 8 elements, at least heads x head_dim)");
  if (!by_sequences && !s.pos) return say(CA_ERR_INVALID_ARG, "pos is null, and there are no sequences");
  return CA_OK;
}

// Workgroups and waves per row of a tensor.
static void shape(RotateTensor &t, int d) {
  if (t.rows == 0) {
    t.segments = 1, t.blocks = 0;
    return;
  }
  const int chunks = (t.heads + 1024 / d - 1) / (1024 / d);
  const int64_t room = MOST_BLOCKS * 4;
  t.segments = int(std::min<int64_t>(chunks, std::max<int64_t>(1, room / t.rows)));
  const int64_t waves = std::min<int64_t>(t.rows * t.segments, room);
  t.blocks = int((waves + 3) / 4);
}

static int rotate(const ca_rotation *r, const ca_rotate_tensor *tensors, int n, const ca_cache_batch *where, float eps, bool backward, void *ws,
                  size_t ws_bytes, hipStream_t st) {
  if (const int rc = check_rotation(r); rc != CA_OK) return rc;
  if (n < 1 || n > 2 || !tensors) return refuse(CA_ERR_INVALID_ARG, "tensors: one or two");
  if (!(eps >= 0.f)) return refuse(CA_ERR_INVALID_ARG, "eps is negative or not a number");
  if (where) {
    if (where->n_seqs < 0 || where->n_seqs > 4096) return refuse(CA_ERR_UNSUPPORTED, "batch: 0 to 4096 sequences");
    if (where->n_seqs > 0 && (!where->q_start || !where->kv_len)) return refuse(CA_ERR_INVALID_ARG, "batch: q_start or kv_len is null");
  }
  const int d = r->head_dim;
  RotateArgs a = {};
  a.turns = r->turns, a.rot = r->rot_dim, a.factor = r->factor, a.eps = eps;
  if (where) a.q_start = where->q_start, a.kv_len = where->kv_len, a.n_seqs = where->n_seqs;
  GainSums g = {};
  float *parts = static_cast<float *>(ws);
  size_t need = 0;
  int64_t bytes = 0;  // of what is read and written
  static const char *const names[] = {"first tensor", "second tensor"};
  for (int i = 0; i < n; ++i) {
    const ca_rotate_tensor &s = tensors[i];
    if (const int rc = check_tensor(s, d, backward, where != nullptr, names[i]); rc != CA_OK) return rc;
    RotateTensor &t = a.t[i];
    t.x = static_cast<const bf16_t *>(s.x), t.dy = static_cast<const bf16_t *>(s.dy), t.y = static_cast<bf16_t *>(s.y);
    t.gain = s.gain, t.pos = where ? nullptr : s.pos, t.rows = where && where->n_seqs == 0 ? 0 : s.rows;
    t.x_stride = s.x_stride, t.y_stride = s.y_stride, t.dy_stride = s.dy_stride, t.heads = s.heads;
    t.gaps = !where && s.gaps;
    shape(t, d);
    bytes += t.rows * t.heads * d * (backward && t.gain ? 6 : 4);
    if (backward && s.gain) {
      if (!s.dgain) return refuse(CA_ERR_INVALID_ARG, std::string(names[i]) + ": dgain is null");
      t.dgain = parts + need / 4, g.parts[i] = t.dgain, g.out[i] = s.dgain, g.n[i] = t.blocks;
      need += size_t(t.blocks) * d * 4;
    }
  }
  if (need > 0 && (!ws || ws_bytes < need || reinterpret_cast<uintptr_t>(ws) % 16 != 0)) {
    std::ostringstream os;
    os << "workspace of " << (ws ? ws_bytes : 0) << " bytes given, " << need << " needed, 16-byte aligned";
    return refuse(CA_ERR_WORKSPACE, os.str());
  }
  const unsigned blocks = unsigned(a.t[0].blocks + a.t[1].blocks);
  if (blocks == 0 && !g.out[0] && !g.out[1]) return CA_OK;
  if (blocks > 0) {
    const Layout l = r->interleaved ? INTERLEAVED : r->rot_dim % 16 == 0 ? HALF : HALF_ANY;
    auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, st, a); };
    auto by_layout = [&](auto dim, auto back, auto past) {
      constexpr int D = decltype(dim)::value;
      constexpr bool B = decltype(back)::value, S = decltype(past)::value;
      if (l == INTERLEAVED) launch(ca_rotate_kernel<D, INTERLEAVED, B, S>);
      else if (l == HALF) launch(ca_rotate_kernel<D, HALF, B, S>);
      else launch(ca_rotate_kernel<D, HALF_ANY, B, S>);
    };
    auto by_size = [&](auto dim, auto back) { bytes > STREAM_BYTES ? by_layout(dim, back, std::true_type{}) : by_layout(dim, back, std::false_type{}); };
    auto by_direction = [&](auto dim) { backward ? by_size(dim, std::true_type{}) : by_size(dim, std::false_type{}); };
    d == 128 ? by_direction(std::integral_constant<int, 128>{}) : by_direction(std::integral_constant<int, 64>{});
  }
  if (g.out[0] || g.out[1]) {
    if (d == 128) hipLaunchKernelGGL(ca_rotate_gain_kernel<128>, dim3(128 / 4, 2), dim3(256), 0, st, g);
    else hipLaunchKernelGGL(ca_rotate_gain_kernel<64>, dim3(64 / 4, 2), dim3(256), 0, st, g);
  }
  if (const hipError_t e = hipGetLastError(); e != hipSuccess)
    return refuse(CA_ERR_HIP, std::string("rotation: ") + hipGetErrorName(e) + " (" + hipGetErrorString(e) + ")");
  return CA_OK;
}

}  // namespace ca

extern "C" {

int ca_rotate(const ca_rotation *r, const ca_rotate_tensor *tensors, int32_t n, const ca_cache_batch *where, float eps, void *hip_stream) {
  return ca::rotate(r, tensors, n, where, eps, false, nullptr, 0, static_cast<hipStream_t>(hip_stream));
}

int ca_rotate_backward(const ca_rotation *r, const ca_rotate_tensor *tensors, int32_t n, const ca_cache_batch *where, float eps, void *ws,
                       size_t ws_bytes, void *hip_stream) {
  return ca::rotate(r, tensors, n, where, eps, true, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
}

size_t ca_rotate_backward_workspace_bytes(void) { return size_t(2) * ca::MOST_BLOCKS * 128 * 4; }

}  // extern "C"
