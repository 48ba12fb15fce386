// What the kernels of the cache share: a call's sequences as they see them, codes, and the checks of the entry points.
#pragma once
#include <hip/hip_runtime.h>

#include <sstream>
#include <string>

#include "ca_device.h"
#include "ca_internal.h"

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
  int more;          // PREFIX: whose row of the table has the pages; TAIL: pages that are left out
};
// Where groups of sequences share their first pages, attention runs over two kinds of sequences in place of the batch's (WHOLE) own.  PREFIX: each
// group's rows, all of which see all of the shared pages.  TAIL: each sequence's rows over the tokens behind them, counted from there.  A sequence of
// which some row would see less than all of the shared pages takes no part: its tail is all of it, and what PREFIX makes of its rows is left.
enum Part { WHOLE, PREFIX, TAIL };
struct GroupedSeqs : SeqArgs {
  const int32_t *group_start, *prefix_pages;
  int n_groups;
};
template <Part P, class A>
__device__ __forceinline__ int n_entries(const A &a) {
  if constexpr (P == PREFIX) return a.n_groups;
  else return a.n_seqs;
}
template <Part P = WHOLE, class A>
__device__ __forceinline__ Seq seq_of(const A &a, int s) {
  Seq q;
  if constexpr (P == PREFIX) {
    q.more = min(max(a.group_start[s], 0), a.n_seqs);
    const int end = min(max(a.group_start[s + 1], q.more), a.n_seqs);
    q.row0 = min(max(a.q_start[q.more], 0), a.total);
    q.n = min(max(a.q_start[end], q.row0), a.total) - q.row0;
    q.len = min(max(a.prefix_pages[s], 0), a.width) * PAGE;
    if (q.len == 0 || end == q.more) q.n = 0;
    return q;
  }
  q.row0 = min(max(a.q_start[s], 0), a.total);
  q.n = min(max(a.q_start[s + 1], q.row0), a.total) - q.row0;
  q.len = min(max(a.kv_len[s], 0), a.width * PAGE);
  q.more = 0;
  if constexpr (P == TAIL) {
    if (a.n_groups > 0) {
      int lo = 0, hi = a.n_groups;  // the last group that begins at s or before
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.group_start[mid] <= s) lo = mid;
        else hi = mid;
      }
      const int shared = a.group_start[lo] <= s && s < a.group_start[lo + 1] ? min(max(a.prefix_pages[lo], 0), a.width) : 0;
      if (q.len - q.n >= shared * PAGE) q.more = shared, q.len -= shared * PAGE;
    }
  }
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
constexpr size_t seq_table_bytes(int n_seqs, Part part = WHOLE) {
  return n_seqs <= 64 ? 0 : 64 + size_t(n_seqs + 4) / 4 * 16 * (part == TAIL ? 5 : 4);
}
template <Part P>
struct SeqTableOf {
  int n_seqs;
  Seq mine;         // up to 64 sequences: of this lane,
  int upto;         // and the units up to it and with it
  int *wave_sums, *pre, *row0, *n, *len, *more;  // more than 64
  const int32_t *group_start;
  int last;

  // for all threads of the workgroup (T); returns the sum of all units
  template <int T, class A, class F>
  __device__ __forceinline__ int fill(void *lds, const A &a, F units) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    n_seqs = n_entries<P>(a);
    if constexpr (P == PREFIX) {
      if (n_seqs == 0) return 0;
      group_start = a.group_start, last = a.n_seqs;
    }
    if (n_seqs <= 64) {
      mine = seq_of<P>(a, min(lane, n_seqs - 1));
      upto = wave_prefix(lane < n_seqs ? units(mine) : 0);
      return __builtin_amdgcn_readlane(upto, 63);
    }
    const int stride = (n_seqs + 4) / 4 * 4;
    wave_sums = static_cast<int *>(lds), pre = wave_sums + 16, row0 = pre + stride, n = row0 + stride, len = n + stride, more = len + stride;
    int carry = 0;
    for (int base = 0; base < n_seqs; base += T) {
      const int i = base + int(threadIdx.x);
      int x = 0;
      if (i < n_seqs) {
        const Seq q = seq_of<P>(a, i);
        row0[i] = q.row0, n[i] = q.n, len[i] = q.len;
        if (P == TAIL) more[i] = q.more;
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
    if (n_seqs <= 64)
      return {__builtin_amdgcn_readlane(mine.row0, s), __builtin_amdgcn_readlane(mine.n, s), __builtin_amdgcn_readlane(mine.len, s),
              P == WHOLE ? 0 : __builtin_amdgcn_readlane(mine.more, s)};
    return {__builtin_amdgcn_readfirstlane(row0[s]), __builtin_amdgcn_readfirstlane(n[s]), __builtin_amdgcn_readfirstlane(len[s]),
            P == WHOLE ? 0 : __builtin_amdgcn_readfirstlane(P == TAIL ? more[s] : min(max(group_start[s], 0), last))};
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
  __device__ __forceinline__ int find_row(int row) const {  // the last one that begins at the row or before, or -1
    if (n_seqs <= 64) return __builtin_popcountll(__ballot(int(threadIdx.x & 63) < n_seqs && mine.row0 <= row)) - 1;
    if (row0[0] > row) return -1;
    int lo = 0, hi = n_seqs;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (row0[mid] <= row) lo = mid;
      else hi = mid;
    }
    return __builtin_amdgcn_readfirstlane(lo);
  }
};
using SeqTable = SeqTableOf<WHOLE>;

// ------------------------------------------------------------------------------------------------ calls
inline int fail(int code, const std::string &msg) {
  set_error(msg);
  return code;
}
inline bool aligned(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
constexpr int64_t MOST_GROUPS = (int64_t(1) << 24) - 1;  // workgroups of 256 threads of a launch, whose threads number less than 2^32
inline int check_cache(const ca_cache *c) {
  if (!c) return fail(CA_ERR_INVALID_ARG, "cache is null");
  if (c->head_dim != 64 && c->head_dim != 128) return fail(CA_ERR_UNSUPPORTED, "head_dim not supported (64 or 128)");
  if (c->n_pages < 0 || c->n_kv_heads < 1) return fail(CA_ERR_INVALID_ARG, "cache: n_pages must not be negative, n_kv_heads at least 1");
  if (c->n_kv_heads > 1024) return fail(CA_ERR_UNSUPPORTED, "cache: more than 1024 KV heads");
  if (c->n_pages > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return fail(CA_ERR_INVALID_ARG, "cache: k, v, k_scale or v_scale is null");
  if (!aligned(c->k) || !aligned(c->v)) return fail(CA_ERR_INVALID_ARG, "cache: k or v is not 16-byte aligned");
  return CA_OK;
}
inline int check_batch(const ca_cache_batch *b) {
  if (!b) return fail(CA_ERR_INVALID_ARG, "batch is null");
  if (b->n_seqs < 0 || b->table_width < 0 || b->total_rows < 0) return fail(CA_ERR_INVALID_ARG, "batch: negative size");
  if (b->n_seqs > MAX_SEQS) return fail(CA_ERR_UNSUPPORTED, "batch: more than 4096 sequences");
  if (b->table_width > (1 << 23)) return fail(CA_ERR_UNSUPPORTED, "batch: table_width beyond 2^23 pages");
  if (b->total_rows >= (int64_t(1) << 30)) return fail(CA_ERR_UNSUPPORTED, "batch: total_rows beyond 2^30");
  if (b->n_seqs > 0 && (!b->q_start || !b->kv_len || (b->table_width > 0 && !b->page_table)))
    return fail(CA_ERR_INVALID_ARG, "batch: q_start, kv_len or page_table is null");
  return CA_OK;
}
inline SeqArgs seq_args(const ca_cache *c, const ca_cache_batch *b) {
  return {b->q_start, b->kv_len, b->page_table, b->n_seqs, b->table_width, int(b->total_rows), c->n_pages};
}
inline int launched(const char *what, hipError_t e) {
  if (e == hipSuccess) e = hipGetLastError();
  if (e == hipSuccess) return CA_OK;
  return fail(CA_ERR_HIP, std::string(what) + ": " + hipGetErrorName(e) + " (" + hipGetErrorString(e) + ")");
}

// Workers of W waves per KV head: as many as are on the chip at a time (NR: 16-row groups of a tile; 8: chunks), eight waves to a CU.  Of tiles of

}  // namespace ca
