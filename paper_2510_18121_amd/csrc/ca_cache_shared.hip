// Attention over the cache where groups of sequences share their first pages (forks of one prompt): those are attended once for all rows of
// a group, the tokens behind them sequence by sequence, and a row's two results are joined.
//
// Of a row the keys are split into the shared ones (P) and the others (T): with L the log-sum-exp over each,
//   O = (exp(L_P) O_P + exp(L_T) O_T) / (exp(L_P) + exp(L_T)).
// Without sharing the codes of the prefix are read once per sequence, 2 D bytes per (token, KV head) each time, and that is what single tokens cost.
// Here the rows of the whole group make up tiles of 128 rows (or 16, 32 where there are few), to which a page is fetched once: the prefix is
// bound by the matrix products, 4 D flops per (row, head, token), and the tails by reading them.  Both go on side by side, in one launch of
// workgroups of either kind (ca_cache_attend.h); a second one joins the results and the parts of the tiles that were cut.
// Measured, whole calls (of which 9 to 10 us are the second launch and the gap before it), 8 KV heads of 128 unless noted, and ca_cache_attend beside it:
//   64 tokens behind 8192, tails of about 560 tokens, 32 heads      46 to 47 us (104)
//   32 tokens behind 130K, 64 heads                                234 to 242 us (703): 0.58 PFLOP/s, MFMAs 43 % busy (a third of them for P's second operand)
//   24 drafts of 3 to 5 rows behind two prefixes of about 5000       42 us (51)
//   200 tokens behind nine prefixes of up to 4000, 16/16 heads of 64  67 us (145): the tails' 165 MB in 45 of them
//   8 tokens behind 2048                                            17 us (17): fixed times, 6 us from the start to the end of one page, most of it cold code and trips to memory
// It pays from about 16 sequences of 8192 shared tokens, or 64 of 512, on; 2 to 8 sequences behind less than 8192 tokens are 1 to 5 us faster without.
// Sequences that share nothing cost less in no group than as groups of no pages, which count in the average that tiles go by: 64 behind 8192 beside 100 of about 1000
// tokens 86 and 99 us (151 without sharing), 16 behind 32768 beside 100 79 and 96 (163), 2 behind 8192 beside 198 109 and 108 (97).
// Not kept (measured with P of the prefix in one operand): every workgroup with a share of both kinds (47 to 51 us, 190, 52, 76 in the first four: a second start costs what the balance gains); runs by what a
// workgroup has beside it on its CU (46 to 49, 184 to 218); tails with workgroups of four waves (200 behind nine: 88); P of the tails as one operand (level).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <sstream>

#include "ca_cache.h"
#include "ca_cache_attend.h"
#include "ca_device.h"
#include "ca_internal.h"
#include "ca_launch.h"

namespace ca {

struct SharedLaunch {
  SharedArgs a;
  float *parts;
  int groups;                // workgroups per KV head, of both kinds
  float cost[2], tiles[2];   // of PREFIX and of TAIL: what a unit costs a workgroup, and all tiles beside their units
  float by_tiles;            // 1 / the tiles of PREFIX, about
  int one_tile;              // the average sequence's rows are one tile of TAIL: a page of it is read once
};

// A worker is a workgroup where tiles are of 128 rows, otherwise a wave.
constexpr int waves_apart(int NR) { return NR == 8 ? 1 : 4; }
// Tiles of up to CUT_SHARED pages are not cut.  (There is a second launch anyway, and more parts cost little there.)
constexpr int CUT_SHARED = 4;

// How the workgroups are dealt to the two kinds: by what they cost together, from the device's arrays, the same in every workgroup.
struct TwoSplits {
  WorkSplit<PREFIX> prefix;
  WorkSplit<TAIL> tail;
  int groups;  // workgroups of PREFIX, the first ones
  int workers[2];
  float *parts[2];
  // KEEP_BOTH: tables of both (lds has room for them); otherwise of the kind that the workgroup is of.
  template <int D, int NP, int NT, bool KEEP_BOTH>
  __device__ __forceinline__ void make(char *lds, const SharedLaunch &x, int group) {
#pragma clang fp contract(off)  // both launches have to come to the same numbers
    const SharedArgs &a = x.a;
    const bool clash = !KEEP_BOTH && a.s.n_groups > 64;  // both tables lie in LDS
    constexpr int WP = waves_apart(NP), WT = waves_apart(NT);
    tail.tab.lanes.load(a.s);
    prefix.tab.lanes = tail.tab.lanes;
    prefix.count<256>(lds, a, 16 * NP);
    if (clash) __syncthreads();
    tail.count<256>(KEEP_BOTH ? lds + seq_table_bytes(a.s.n_groups, PREFIX) : lds, a, 16 * NT);
    // (a unit of 128 rows to one of 16: 3.4 to 1.5, with P in one operand 2.6.  With 2.6 and with 3.8 to 1.5 64 tokens behind 8192 take 47.2 and 46.1 us, not 46.4, 24 drafts
    // behind two prefixes 45.1 and 42.3, not 42.2, 32 tokens behind 130K 232 and 233, not 236.)
    const float p = x.cost[0] * float(prefix.total) + x.tiles[0], t = x.cost[1] * float(tail.total) + x.tiles[1];
    // Units of a worker of PREFIX, at least: of tiles of 16 rows a page takes a wave about as long as the join takes for 14 parts.
    const int least = NP == 8 ? 2 : max(2, int(__builtin_amdgcn_sqrtf(float(prefix.total) * x.by_tiles * (1.f / 14.f)) + 0.5f));
    const int most = quotient(prefix.total + least * WP - 1, least * WP);
    groups = prefix.total == 0 ? 0 : min(most, max(1, min(x.groups - 1, int(float(x.groups) * p / (p + t) + 0.5f))));
    groups = __builtin_amdgcn_readfirstlane(groups);
    workers[0] = groups * WP, workers[1] = (x.groups - groups) * WT;
    prefix.run = max(__builtin_amdgcn_readfirstlane(least), quotient(prefix.total + max(workers[0], 1) - 1, max(workers[0], 1)));
    tail.run = max(1, quotient(tail.total + workers[1] - 1, workers[1]));
    prefix.cut = tail.cut = CUT_SHARED;
    // Tails that the last cache does not hold until the next call, as in ca_cache_attend.  Not what is fetched by several tiles: the prefix, and tails of more rows (24 sequences
    // of 20 or 32 rows behind a prefix of 6000, 8 heads of 128: tails of 329 MiB 145 us past the cache, 128 through it, 446 MiB 197 and 173, 835 MiB 296 and 286, 890 MiB 336 and 342).
    tail.stream = x.one_tile && float(tail.total) * float(a.hkv * 2 * PAGE * D) > float(384 << 20);
    parts[0] = x.parts, parts[1] = x.parts + size_t(workers[0]) * 2 * a.hkv * (16 * NP * (D + 2));
    if (clash && group < groups) {
      __syncthreads();
      prefix.count<256>(lds, a, 16 * NP);
    }
  }
};

template <int D, int NR>
constexpr int tile_bytes() {
  if constexpr (NR == 8) return ChunkSmem<D>::TOTAL;
  else return 4 * AttendShape<D, NR, 1>::MERGE;
}
template <Part P, int D, int NR, bool TWO, class A>
__device__ __forceinline__ void tile_workgroup(const A &a, char *smem, const WorkSplit<P> &split, int hk, int group, float *parts) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if constexpr (NR == 8) chunk_workgroup<P, D, TWO>(a, smem, split, hk, group, parts);
  else attend_workgroup<P, D, NR, 1>(a, smem + wave * AttendShape<D, NR, 1>::MERGE, split, hk, 4 * group + wave, parts);
}

// NP, NT: 16-row groups of a tile of the prefix and of the tails.
template <int D, int NP, int NT>
__global__ __launch_bounds__(256, 2) void ca_cache_shared_kernel(const SharedLaunch x) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  // P of tiles of 128 rows in two operands where ca_cache_attend has them, by the rows of a sequence and whatever the group: one costs 2.3e-3 of O in place of
  // 1.7e-3, two cost 64 tokens behind 8192 46 us in place of 44, 24 drafts 42 (40), 32 tokens behind 130K 236 (186).
  constexpr bool TWO = NT != 8;
  const int group = blockIdx.y;
  TwoSplits s;
  s.make<D, NP, NT, false>(smem + std::max(tile_bytes<D, NP>(), tile_bytes<D, NT>()), x, group);
  if (group < s.groups) tile_workgroup<PREFIX, D, NP, TWO>(x.a, smem, s.prefix, blockIdx.x, group, s.parts[0]);
  else tile_workgroup<TAIL, D, NT, TWO>(x.a, smem, s.tail, blockIdx.x, group - s.groups, s.parts[1]);
}

// What there is of a row's tile: the parts of the workers that had a run of its pages each, or one sum of the row.
struct RowParts {
  const float *first, *others;
  uint32_t stride;  // from a worker's part to the next one's
  int sums, ml;     // where they are in a part
  int n;
  template <Part P, int D, class A>
  __device__ __forceinline__ void of(const A &a, const WorkSplit<P> &split, const float *parts, int n_workers, int entry, const Seq &q, int row, int h, int hk) {
    const int R = split.R, G = a.G, r = (row - q.row0) * G + h - hk * G, tile = r / R, in_tile = r - tile * R;
    const int per = tile_pages(q.len, R, G, a.window, a.sinks), u0 = split.tab.before(entry) + tile * per;
    // (sequences that overlap, against their description, may have more units than are counted)
    const int w0 = min(quotient(u0, split.run), n_workers - 1), w1 = min(quotient(u0 + per - 1, split.run), n_workers - 1);
    if (per <= split.cut || w0 == w1) {
      n = 1, sums = 0, ml = D, first = others = a.row_sums[P == TAIL] + (size_t(row) * a.hq + h) * row_floats(D);
      return;
    }
    const uint32_t size = R * (D + 2);
    n = w1 - w0 + 1, stride = 2 * a.hkv * size, sums = in_tile * D, ml = R * D + 2 * in_tile;
    first = parts + (size_t(2 * w0 + 1) * a.hkv + hk) * size;  // (the part of a tile that begins in a worker's run is its second)
    others = parts + (size_t(2 * w0 + 2) * a.hkv + hk) * size;
  }
  __device__ __forceinline__ const float *part(int i) const { return i == 0 ? first : others + uint32_t(i - 1) * size_t(stride); }
};

// A wave takes a row and head at a time: D / 4 lanes to a part.
template <int D, int NP, int NT>
__global__ __launch_bounds__(256) void ca_cache_join_kernel(const SharedLaunch x) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  constexpr int LANES = D / 4, AT_A_TIME = 64 / LANES, LOADS = 8;
  const SharedArgs &a = x.a;
  TwoSplits split;
  split.make<D, NP, NT, true>(smem, x, 0);
  const WorkSplit<PREFIX> &prefix = split.prefix;
  const WorkSplit<TAIL> &tail = split.tail;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = lane / LANES, col = 4 * (lane % LANES);
  for (int row = blockIdx.x; row < a.s.total; row += gridDim.x) {
    const int s = tail.tab.find_row(row);
    if (s < 0) continue;
    const Seq q = tail.tab.at(s);
    if (row < q.row0 || row >= q.row0 + q.n) continue;
    int g = -1;
    Seq of_group = {};
    if (q.more > 0) {
      g = prefix.tab.find_row(row);
      of_group = prefix.tab.at(max(g, 0));
      if (row < of_group.row0 || row >= of_group.row0 + of_group.n) g = -1;
    }
    for (int h = 4 * blockIdx.y + wave; h < a.hq; h += 4 * gridDim.y) {
      const int hk = a.token_of(h);  // h / G
      RowParts t, p;
      t.of<TAIL, D>(a, tail, split.parts[1], split.workers[1], s, q, row, h, hk);
      if (q.more == 0 && t.n == 1) continue;  // it is done
      p = t, p.n = 0;
      if (g >= 0) p.of<PREFIX, D>(a, prefix, split.parts[0], split.workers[0], g, of_group, row, h, hk);
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
      float top = NO_MAX, sum = 0.f;
      auto add = [&](float m, float l, const f32x4 &z) __attribute__((always_inline)) {
        const float grown = fmaxf(top, m), old = fast_exp2(top - grown), w = fast_exp2(m - grown);
        top = grown, sum = sum * old + w * l;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = y[e] * old + w * z[e];
      };
      const int n_parts = p.n + t.n;
      for (int base = 0; base < n_parts; base += LOADS * AT_A_TIME) {  // (all of a round's loads before the first sum)
        f32x4 z[LOADS];
        f32x2 ml[LOADS];
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
          const int i = min(base + k * AT_A_TIME + mine, n_parts - 1);
          const bool in_prefix = i < p.n;
          const float *const from = in_prefix ? p.part(i) : t.part(i - p.n);
          z[k] = *reinterpret_cast<const f32x4 *>(from + (in_prefix ? p.sums : t.sums) + col);
          ml[k] = *reinterpret_cast<const f32x2 *>(from + (in_prefix ? p.ml : t.ml));
        }
#pragma unroll
        for (int k = 0; k < LOADS; ++k)
          if (base + k * AT_A_TIME + mine < n_parts) add(ml[k][0], ml[k][1], z[k]);
      }
#pragma unroll
      for (int o = LANES; o < 64; o <<= 1) {
        f32x4 z;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = __shfl_xor(y[e], o);
        add(__shfl_xor(top, o), __shfl_xor(sum, o), z);
      }
      if (mine != 0) continue;
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      *reinterpret_cast<u32x2 *>(a.o + (size_t(row) * a.hq + h) * D + col) =
          u32x2{pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv)};
      if (col == 0 && a.lse) a.lse[size_t(h) * a.s.total + row] = 0.6931471805599453f * (top + fast_log2(sum));
    }
  }
}

// ------------------------------------------------------------------------------------------------ calls
// Workgroups per KV head: two of four waves to a CU.
static int shared_groups(int hkv) { return std::max(2, N_CU * 2 / hkv); }
static size_t round_up(size_t x) { return (x + 255) / 256 * 256; }
struct SharedBytes {
  size_t parts, sums;  // sums: of each kind
  size_t all() const { return parts + 2 * sums; }
};
static SharedBytes shared_bytes(int d, int hkv, int hq, int64_t rows) {
  // (parts: two of 128 rows for each workgroup, which is also room for two of 16 rows for each of its waves)
  return {round_up(size_t(shared_groups(hkv)) * 2 * hkv * (128 * (d + 2)) * 4), round_up(size_t(rows) * hq * row_floats(d) * 4)};
}

template <int D, int NP, int NT>
static int launch_shared(SharedLaunch &x, hipStream_t st) {
  const SharedArgs &a = x.a;
  x.groups = shared_groups(a.hkv);
  const float rows = float(a.s.total) * a.G;
  x.cost[0] = NP == 8 ? (NT == 8 ? 2.6f : 3.4f) : 1.2f, x.cost[1] = NT == 8 ? 2.6f : 1.5f;
  x.one_tile = int64_t(a.s.total) * a.G <= int64_t(16 * NT) * a.s.n_seqs;
  x.by_tiles = 1.f / (rows / (16 * NP) + float(std::max(1, a.s.n_groups)) / 2);
  x.tiles[0] = (rows / (16 * NP) + a.s.n_groups) * (NP == 8 ? 4.f : 1.f), x.tiles[1] = (rows / (16 * NT) + a.s.n_seqs) * (NT == 8 ? 4.f : 1.f);
  const size_t tables[2] = {seq_table_bytes(a.s.n_groups, PREFIX), seq_table_bytes(a.s.n_seqs, TAIL)};
  const size_t bytes = std::max(tile_bytes<D, NP>(), tile_bytes<D, NT>()) + std::max(tables[0], tables[1]);
  auto kern = ca_cache_shared_kernel<D, NP, NT>;
  auto join = ca_cache_join_kernel<D, NP, NT>;
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  static std::atomic<bool> done[2][16];
  if (e == hipSuccess) e = set_smem(kern, int(std::max(tile_bytes<D, NP>(), tile_bytes<D, NT>()) + seq_table_bytes(MAX_SEQS, TAIL)), device, done[0]);
  if (e == hipSuccess) e = set_smem(join, int(seq_table_bytes(MAX_SEQS, PREFIX) + seq_table_bytes(MAX_SEQS, TAIL)), device, done[1]);
  if (e != hipSuccess) return launched("cache attention of groups", e);
  hipLaunchKernelGGL(kern, dim3(unsigned(a.hkv), unsigned(x.groups)), dim3(256), bytes, st, x);
  const int heads = std::min((a.hq + 3) / 4, 1 << 10), rows_at_a_time = std::min(a.s.total, std::max(1, N_CU * 64 / heads));
  hipLaunchKernelGGL(join, dim3(unsigned(rows_at_a_time), unsigned(heads)), dim3(256), tables[0] + tables[1], st, x);
  return launched("cache attention of groups", hipSuccess);
}

// Rows per tile, as in ca_cache_attend, from the average group and the average sequence.  (Tiles of 32 rows, as there, are none here: at head_dim 128 they leave
// room for four waves to a CU, 8 answers to a prompt of 2048 tokens 20.6 us with them and 17.8 without; at 64 200 answers to nine of 4000 72 and 68.  Without them sequences of
// 17 to 32 rows read their tails twice: 24 of 20 rows behind 6000 tokens of one prefix, 8 heads of 128, tails of about 500 tokens 46 us and ca_cache_attend 55, of 2000 63 and 68, of 5000 128 and
// 105, of 16000 286 and 200.  Sequences of more rows, whose prefix is bound by its products, gain nothing: 4 of 500 behind 8192, 32 heads, 366 and 313, at 64 281 and 195.)
template <int D>
static int shared_by_rows(SharedLaunch &x, hipStream_t st) {
  const SharedArgs &a = x.a;
  const int64_t rows = int64_t(a.s.total) * a.G, of_group = rows / std::max(1, a.s.n_groups), of_seq = rows / a.s.n_seqs;
  if (of_seq > 32) return launch_shared<D, 8, 8>(x, st);
  return of_group > 32 ? launch_shared<D, 8, 1>(x, st) : launch_shared<D, 1, 1>(x, st);
}

}  // namespace ca

extern "C" {

int ca_cache_attend_shared_workspace_bytes(const ca_cache *c, int32_t n_q_heads, int64_t total_rows, size_t *bytes) {
  using namespace ca;
  if (const int rc = check_cache(c); rc != CA_OK) return rc;
  if (!bytes) return fail(CA_ERR_INVALID_ARG, "output is null");
  if (n_q_heads < 1 || n_q_heads % c->n_kv_heads != 0) return fail(CA_ERR_UNSUPPORTED, "n_q_heads is not a multiple of n_kv_heads");
  if (total_rows < 0 || total_rows >= (int64_t(1) << 30)) return fail(CA_ERR_INVALID_ARG, "total_rows: not negative, below 2^30");
  *bytes = shared_bytes(c->head_dim, c->n_kv_heads, n_q_heads, total_rows).all();
  return CA_OK;
}

int ca_cache_attend_shared(const ca_cache *c, const ca_cache_batch *b, const ca_cache_groups *groups, int32_t n_q_heads, float softmax_scale,
                           const void *q, void *o, float *lse, void *ws, size_t ws_bytes, void *hip_stream) {
  using namespace ca;
  if (const int rc = check_cache(c); rc != CA_OK) return rc;
  if (const int rc = check_batch(b); rc != CA_OK) return rc;
  if (!groups) return fail(CA_ERR_INVALID_ARG, "groups is null");
  if (groups->n_groups < 0 || groups->n_groups > b->n_seqs) return fail(CA_ERR_INVALID_ARG, "groups: none, or up to as many as there are sequences");
  if (groups->n_groups > 0 && (!groups->group_start || !groups->prefix_pages)) return fail(CA_ERR_INVALID_ARG, "groups: group_start or prefix_pages is null");
  if (n_q_heads < 1 || n_q_heads % c->n_kv_heads != 0) return fail(CA_ERR_UNSUPPORTED, "n_q_heads is not a multiple of n_kv_heads");
  if (b->n_seqs == 0 || b->total_rows == 0) return CA_OK;
  if (!q || !o) return fail(CA_ERR_INVALID_ARG, "q or o is null");
  if (!aligned(q) || !aligned(o)) return fail(CA_ERR_INVALID_ARG, "q or o is not 16-byte aligned");
  const SharedBytes need = shared_bytes(c->head_dim, c->n_kv_heads, n_q_heads, b->total_rows);
  if (!ws || ws_bytes < need.all() || reinterpret_cast<uintptr_t>(ws) % 256 != 0) {
    std::ostringstream os;
    os << "workspace of " << (ws ? ws_bytes : 0) << " bytes given, " << need.all() << " needed, 256-byte aligned";
    return fail(CA_ERR_WORKSPACE, os.str());
  }
  const int64_t g = n_q_heads / c->n_kv_heads;
  if ((b->total_rows * g / 16 + b->n_seqs) * std::max(1, b->table_width) >= int64_t(1) << 30)
    return fail(CA_ERR_UNSUPPORTED, "batch: rows times pages beyond 2^30");
  if ((b->total_rows * g + 128) * g >= int64_t(1) << 32) return fail(CA_ERR_UNSUPPORTED, "batch: rows times the square of the heads per KV head beyond 2^32");
  SharedLaunch x = {};
  SharedArgs &a = x.a;
  static_cast<SeqArgs &>(a.s) = seq_args(c, b);
  a.s.group_start = groups->group_start, a.s.prefix_pages = groups->prefix_pages, a.s.n_groups = groups->n_groups;
  a.k = static_cast<const uint8_t *>(c->k), a.v = static_cast<const uint8_t *>(c->v), a.k_scale = c->k_scale, a.v_scale = c->v_scale;
  a.q = static_cast<const bf16_t *>(q), a.o = static_cast<bf16_t *>(o), a.lse = lse;
  a.hq = n_q_heads, a.hkv = c->n_kv_heads, a.G = int(g), a.by_g = uint32_t(((uint64_t(1) << 32) + uint64_t(g) - 1) / uint64_t(g));
  a.window = 1 << 30, a.sinks = 0;
  a.c = (softmax_scale > 0.f ? softmax_scale : c->head_dim == 128 ? 0.08838834764831845f : 0.125f) * 1.4426950408889634f;
  char *at = static_cast<char *>(ws);
  x.parts = reinterpret_cast<float *>(at), at += need.parts;
  for (int i = 0; i < 2; ++i) {
    a.row_sums[i] = reinterpret_cast<float *>(at), at += need.sums;
  }
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  return c->head_dim == 128 ? shared_by_rows<128>(x, st) : shared_by_rows<64>(x, st);
}

}  // extern "C"
