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
__device__ __forceinline__ Seq seq_from(const SeqArgs &a, int start, int end, int len) {
  Seq q;
  q.row0 = min(max(start, 0), a.total);
  q.n = min(max(end, q.row0), a.total) - q.row0;
  q.len = min(max(len, 0), a.width * PAGE);
  q.more = 0;
  return q;
}
__device__ __forceinline__ Seq seq_of(const SeqArgs &a, int s) { return seq_from(a, a.q_start[s], a.q_start[s + 1], a.kv_len[s]); }
// What the arrays say of the first 64 groups and sequences, one per lane, all of it in one trip to memory.
struct GroupLanes {
  int start, end, pages;  // of this lane's group
  int row, row_end, len;  // q_start of this lane and of the next, kv_len
  int n;                  // groups
  __device__ __forceinline__ void load(const GroupedSeqs &a) {
    const int lane = threadIdx.x & 63, g = min(lane, max(a.n_groups - 1, 0));
    n = a.n_groups, start = end = pages = 0;
    if (n > 0) start = a.group_start[g], end = a.group_start[g + 1], pages = a.prefix_pages[g];
    row = a.q_start[min(lane, a.n_seqs)], row_end = a.q_start[min(lane + 1, a.n_seqs)], len = a.kv_len[min(lane, a.n_seqs - 1)];
  }
  __device__ __forceinline__ int row_of(const GroupedSeqs &a, int i) const {  // q_start[i], of any lane's own i
    if (a.n_seqs < 64) return __shfl(row, i);
    return a.q_start[i];
  }
  // the pages that sequence s shares (for all lanes of a wave together)
  __device__ __forceinline__ int shared_by(const GroupedSeqs &a, int s) const {
    if (n == 0) return 0;
    int lo = 0, hi = n;  // the last group that begins at s or before
    int first, last, p;
    if (n <= 64) {
      for (int step = 32; step > 0; step >>= 1) {
        if (step >= n) continue;
        const int mid = min(lo + step, n - 1);
        if (__shfl(start, mid) <= s) lo = mid;
      }
      first = __shfl(start, lo), last = __shfl(end, lo), p = __shfl(pages, lo);
    } else {
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.group_start[mid] <= s) lo = mid;
        else hi = mid;
      }
      first = a.group_start[lo], last = a.group_start[lo + 1], p = a.prefix_pages[lo];
    }
    return first <= s && s < last ? min(max(p, 0), a.width) : 0;
  }
};
__device__ __forceinline__ Seq group_as_seq(const GroupedSeqs &a, const GroupLanes &l, int g) {
  int start = l.start, end = l.end, pages = l.pages;
  if (a.n_groups > 64) start = a.group_start[g], end = a.group_start[g + 1], pages = a.prefix_pages[g];
  const int first = min(max(start, 0), a.n_seqs), last = min(max(end, first), a.n_seqs);
  Seq q = seq_from(a, l.row_of(a, first), l.row_of(a, last), 0);
  q.more = first, q.len = min(max(pages, 0), a.width) * PAGE;
  if (q.len == 0 || last == first) q.n = 0;
  return q;
}
__device__ __forceinline__ Seq tail_of(const GroupedSeqs &a, const GroupLanes &l, int s) {
  Seq q = a.n_seqs <= 64 ? seq_from(a, l.row, l.row_end, l.len) : seq_of(a, s);
  const int shared = l.shared_by(a, s);
  if (q.len - q.n >= shared * PAGE) q.more = shared, q.len -= shared * PAGE;
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
  GroupLanes lanes;  // PREFIX and TAIL: loaded before

  template <class A>
  __device__ __forceinline__ Seq entry(const A &a, int i) const {
    if constexpr (P == WHOLE) return seq_of(a, i);
    else if constexpr (P == PREFIX) return group_as_seq(a, lanes, i);
    else return tail_of(a, lanes, i);
  }
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
      mine = entry(a, min(lane, n_seqs - 1));  // (of lanes behind the last one nothing is used)
      upto = wave_prefix(lane < n_seqs ? units(mine) : 0);
      return __builtin_amdgcn_readlane(upto, 63);
    }
    const int stride = (n_seqs + 4) / 4 * 4;
    wave_sums = static_cast<int *>(lds), pre = wave_sums + 16, row0 = pre + stride, n = row0 + stride, len = n + stride, more = len + stride;
    int carry = 0;
    for (int base = 0; base < n_seqs; base += T) {
      const int i = base + int(threadIdx.x);
      int x = 0;
      Seq q;
      if (P != WHOLE) q = entry(a, min(i, n_seqs - 1));  // (by all lanes)
      if (i < n_seqs) {
        if (P == WHOLE) q = entry(a, i);
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
    if constexpr (P != WHOLE) return last_upto(pre, u);
    int lo = 0, hi = n_seqs;  // pre[lo] <= u < pre[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pre[mid] <= u) lo = mid;
      else hi = mid;
    }
    return __builtin_amdgcn_readfirstlane(lo);
  }
  // the last of x[0 .. n_seqs - 1], which do not descend, that is not above v, or -1: two looks at 64 of them
  __device__ __forceinline__ int last_upto(const int *x, int v) const {
    const int lane = threadIdx.x & 63, run = (n_seqs + 63) / 64;
    const int before = max(0, __builtin_popcountll(__ballot(lane * run < n_seqs && x[min(lane * run, n_seqs - 1)] <= v)) - 1) * run;
    return before + __builtin_popcountll(__ballot(lane < run && before + lane < n_seqs && x[min(before + lane, n_seqs - 1)] <= v)) - 1;
  }
  __device__ __forceinline__ int find_row(int row) const {  // the last one that begins at the row or before, or -1
    if (n_seqs <= 64) return __builtin_popcountll(__ballot(int(threadIdx.x & 63) < n_seqs && mine.row0 <= row)) - 1;
    return last_upto(row0, row);
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
}  // namespace ca
