// Reading a cache back: the rows of a call's sequences from their pages to bf16, code * scale, rounded once.
//
// Bound by HBM: 2 bytes of codes in and 4 out per (token, KV head, column).  V lies [D][64] in a page and leaves as rows of tokens: words of four
// tokens of eight columns are transposed in registers.
#include <hip/hip_runtime.h>

#include "ca_cache.h"
#include "ca_device.h"
#include "ca_internal.h"
#include "ca_launch.h"

namespace ca {

struct ReadArgs {
  SeqArgs s;
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  bf16_t *out_k, *out_v;
  int hkv;
};

// 8 codes, times f, as 8 bf16
__device__ __forceinline__ u32x4 codes_times(uint32_t a, uint32_t b, float f) {
  typedef float v2 __attribute__((ext_vector_type(2)));
  const v2 x = __builtin_amdgcn_cvt_pk_f32_fp8(int(a), false), y = __builtin_amdgcn_cvt_pk_f32_fp8(int(a), true);
  const v2 z = __builtin_amdgcn_cvt_pk_f32_fp8(int(b), false), w = __builtin_amdgcn_cvt_pk_f32_fp8(int(b), true);
  return u32x4{pack_bf16(x[0] * f, x[1] * f), pack_bf16(y[0] * f, y[1] * f), pack_bf16(z[0] * f, z[1] * f), pack_bf16(w[0] * f, w[1] * f)};
}

// Words of four bytes, rows of a 4 x 4 matrix, transposed.
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602);  // w0.0 w1.0 w0.1 w1.1, ..
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
  w[0] = __builtin_amdgcn_perm(c, a, 0x05040100), w[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
  w[2] = __builtin_amdgcn_perm(d, b, 0x05040100), w[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}

// One wave per (page with tokens that are asked for, KV head, K or V).  K: a lane has 8 columns of a token; V: 8 columns of 16 (head_dim 64: 8) tokens.
// STREAM: rows that the last cache does not hold until somebody reads them are stored past it.
// (8 sequences of about 16K tokens, 8 heads of 128, 1.08 GB: 223 us, 215 past the cache, 5.0 TB/s; with the codes' loads past it too 220.  16 columns of a token
// to a lane of K, whose stores are then halves of lines: 233 and 287.  A copy of 512 MB: 5.3 to 5.6 TB/s.)
template <int D, bool STREAM>
__global__ __launch_bounds__(256) void ca_cache_read_kernel(const ReadArgs a) {
  auto put = [](u32x4 *p, const u32x4 &v) __attribute__((always_inline)) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
  };
  extern __shared__ __attribute__((aligned(16))) char smem[];
  SeqTable tab;
  auto first_pos = [](const Seq &q) { return max(0, q.len - q.n); };
  const int total = tab.fill<256>(smem, a.s, [&](const Seq &q) { return q.n > 0 && q.len > 0 ? (q.len - 1) / PAGE - first_pos(q) / PAGE + 1 : 0; });
  const int unit = int(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int touch = unit / (2 * a.hkv), h = unit / 2 % a.hkv, lane = threadIdx.x & 63;
  const bool is_k = unit % 2 == 0;
  if (touch >= total || !(is_k ? a.out_k : a.out_v)) return;
  const int s = tab.find(touch);
  const Seq q = tab.at(s);
  const int index = first_pos(q) / PAGE + touch - tab.before(s);
  int page = a.s.table[size_t(s) * a.s.width + index];
  if (page >= a.s.n_pages) page = -1;
  const int begin = max(first_pos(q) - index * PAGE, 0), end = min(q.len - index * PAGE, PAGE);  // the page's tokens that are asked for
  const int64_t row0 = int64_t(q.row0) + index * PAGE - (q.len - q.n);                           // the row of the page's token 0
  const size_t at = size_t(max(page, 0)) * a.hkv + h, row = size_t(a.hkv) * D;
  const float f = page < 0 ? 0.f : (is_k ? a.k_scale : a.v_scale)[at];
  if (is_k) {
    constexpr int LPT = D / 8, TPI = 64 / LPT;  // lanes per token, tokens per load
    const uint8_t *const src = a.k + at * (PAGE * D) + 8 * (lane % LPT);
    bf16_t *const dst = a.out_k + row0 * int64_t(row) + size_t(h) * D + 8 * (lane % LPT);
#pragma unroll
    for (int i = 0; i < PAGE / TPI; ++i) {
      const int t = TPI * i + lane / LPT;
      if (t < begin || t >= end) continue;
      u32x2 w = {0, 0};
      if (page >= 0) w = *reinterpret_cast<const u32x2 *>(src + t * D);
      put(reinterpret_cast<u32x4 *>(dst + t * int64_t(row)), codes_times(w[0], w[1], f));
    }
    return;
  }
  constexpr int G = D / 8, NT = G;  // groups of columns; tokens of a lane
  const int g = lane % G, t0 = NT * (lane / G);
  const uint8_t *const src = a.v + at * (PAGE * D) + 8 * g * PAGE + t0;
  bf16_t *const dst = a.out_v + row0 * int64_t(row) + size_t(h) * D + 8 * g;
  if (t0 >= end || t0 + NT <= begin) return;
  uint32_t w[8][NT / 4];
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    if (page < 0) {
#pragma unroll
      for (int i = 0; i < NT / 4; ++i) w[c][i] = 0;
    } else if constexpr (NT == 16) {
      const u32x4 x = *reinterpret_cast<const u32x4 *>(src + c * PAGE);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[c][i] = x[i];
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2 *>(src + c * PAGE);
      w[c][0] = x[0], w[c][1] = x[1];
    }
  }
#pragma unroll
  for (int i = 0; i < NT / 4; ++i) {
    uint32_t lo[4] = {w[0][i], w[1][i], w[2][i], w[3][i]}, hi[4] = {w[4][i], w[5][i], w[6][i], w[7][i]};
    transpose4(lo), transpose4(hi);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = t0 + 4 * i + e;
      if (t >= begin && t < end) put(reinterpret_cast<u32x4 *>(dst + t * int64_t(row)), codes_times(lo[e], hi[e], f));
    }
  }
}

}  // namespace ca

extern "C" int ca_cache_read(const ca_cache *c, const ca_cache_batch *b, void *k, void *v, void *hip_stream) {
  using namespace ca;
  if (const int rc = check_cache(c); rc != CA_OK) return rc;
  if (const int rc = check_batch(b); rc != CA_OK) return rc;
  if (b->n_seqs == 0 || b->total_rows == 0 || b->table_width == 0) return CA_OK;
  if (!k && !v) return fail(CA_ERR_INVALID_ARG, "k and v are null");
  if (!aligned(k) || !aligned(v)) return fail(CA_ERR_INVALID_ARG, "k or v is not 16-byte aligned");
  const ReadArgs a = {seq_args(c, b), static_cast<const uint8_t *>(c->k), static_cast<const uint8_t *>(c->v), c->k_scale, c->v_scale,
                      static_cast<bf16_t *>(k), static_cast<bf16_t *>(v), c->n_kv_heads};
  // pages that n rows of a sequence can touch: at most (n - 1) / 64 + 2, and no more than n
  const int64_t touches = std::min<int64_t>(b->total_rows, b->total_rows / PAGE + 2 * int64_t(b->n_seqs));
  const int64_t groups = (touches * 2 * c->n_kv_heads + 3) / 4;
  if (groups > MOST_GROUPS) return fail(CA_ERR_UNSUPPORTED, "batch: rows times KV heads too many");
  const bool past = b->total_rows * c->n_kv_heads * c->head_dim * 6 > int64_t(384) << 20;
  auto kern = c->head_dim == 128 ? (past ? ca_cache_read_kernel<128, true> : ca_cache_read_kernel<128, false>)
                                 : (past ? ca_cache_read_kernel<64, true> : ca_cache_read_kernel<64, false>);
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  static std::atomic<bool> done[4][16];
  if (e == hipSuccess) e = set_smem(kern, int(seq_table_bytes(MAX_SEQS)), device, done[2 * past + (c->head_dim == 128)]);
  if (e != hipSuccess) return launched("cache read", e);
  hipLaunchKernelGGL(kern, dim3(unsigned(groups)), dim3(256), seq_table_bytes(b->n_seqs), static_cast<hipStream_t>(hip_stream), a);
  return launched("cache read", hipSuccess);
}
