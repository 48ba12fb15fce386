// The schedule of a windowed plan: attention with a sliding window and sinks over the tasks of a batch (host only).
//
// A row at position p sees [lo, hi] with hi = min(p, kv_len - 1), lo = p - window + 1, and the keys below `sinks` up to hi.  Rows of
// a document are sorted by (hi, lo).  Forward / dQ units are always head-packed: 256 / hp slots x hp heads span few positions, so a
// unit's tiles are little more than the window (with 256 slots of one head a window of 1024 keys takes 21 tiles, with 64 slots of 4
// heads 18).  Part of ca_plan.cpp.
#pragma once
#include <algorithm>
#include <climits>

#include "ca_internal.h"

namespace ca {

// Returns false where there are too many padded rows.
inline bool schedule_window(ca_plan_t *p) {
  constexpr size_t MAX_PARTS = size_t(256) << 20;
  auto up = [](int64_t x, int64_t m) { return (x + m - 1) / m * m; };
  const int hq = p->hq, hkv = p->hkv, g = hq / hkv;
  const int hp = g % 8 == 0 ? 8 : g % 4 == 0 ? 4 : g % 2 == 0 ? 2 : 1;
  const int sub = FWD_BM / hp, align = std::max(sub, BWD_BQ);
  p->heads_packed = hp, p->slot_align = align;
  std::vector<std::vector<int32_t>> by_doc(size_t(p->n_docs));
  int64_t covered_q = 0, covered_kv = 0;
  for (int t = 0; t < p->n_tasks; ++t) by_doc[size_t(p->task_doc[t])].push_back(t), covered_q += p->task_q_len[t];

  struct Row {
    int32_t hi, lo, row;
  };
  struct Tile {
    int64_t cost;
    FwdUnit u;
  };
  std::vector<Tile> ftiles;
  std::vector<WindowUnit> btiles;
  std::vector<Row> rows;
  std::vector<int32_t> block_hi_min, block_hi_max, lo_from, lo_upto;  // per block of 64 slots; lo: the least from there on, the largest so far
  for (int dd = 0; dd < p->n_docs; ++dd) {
    auto &tasks = by_doc[size_t(dd)];
    if (tasks.empty()) continue;
    std::stable_sort(tasks.begin(), tasks.end(), [&](int a, int b) { return p->task_q_pos[a] < p->task_q_pos[b]; });
    rows.clear();
    for (int t : tasks)
      for (int64_t i = 0; i < p->task_q_len[t]; ++i) {
        const int64_t pos = p->task_q_pos[t] + i, hi = std::min(pos, p->task_kv_len[t] - 1);
        // (an empty window begins behind hi, whatever it would begin at)
        rows.push_back({int32_t(hi), int32_t(std::min(std::max<int64_t>(0, pos - p->window + 1), hi + 1)), int32_t(p->task_q_start[t] + i)});
      }
    auto before = [](const Row &a, const Row &b) { return a.hi != b.hi ? a.hi < b.hi : a.lo < b.lo; };
    if (!std::is_sorted(rows.begin(), rows.end(), before)) std::stable_sort(rows.begin(), rows.end(), before);
    const size_t s0 = p->slot_row.size();
    const int32_t kv_row0 = int32_t(p->doc_kv_start[dd]);
    // runs of rows whose windows leave no key between them out, each padded: what a unit's window tiles hold from its first window on is
    // seen by somebody
    for (size_t a = 0, b; a < rows.size(); a = b) {
      for (b = a + 1; b < rows.size() && rows[b].lo <= rows[b - 1].hi + 1; ++b) {
      }
      const size_t n = size_t(up(int64_t(b - a), align)), at = p->slot_row.size();
      if (at + n >= size_t(INT32_MAX) - SLOT_ALIGN) return false;
      for (size_t i = 0; i < n; ++i) {
        const Row &r = rows[std::min(a + i, b - 1)];
        p->slot_row.push_back(a + i < b ? r.row : -1), p->slot_pos.push_back(r.hi), p->slot_lo.push_back(r.lo), p->slot_src.push_back(r.row);
      }
      for (size_t i = a; i < b; i += size_t(sub)) {
        const size_t e = std::min(b, i + size_t(sub));
        int32_t lo = INT32_MAX;
        for (size_t r = i; r < e; ++r)
          if (rows[r].lo <= rows[r].hi) lo = std::min(lo, rows[r].lo);
        const int32_t n_keys = rows[e - 1].hi + 1, key0 = std::min(lo, n_keys - 1) / FWD_BN * FWD_BN;
        const int32_t n_sink = std::min((p->sinks + FWD_BN - 1) / FWD_BN, key0 / FWD_BN);
        ftiles.push_back({n_sink + (n_keys - key0 + FWD_BN - 1) / FWD_BN,
                          {int32_t(at + i - a), kv_row0, n_keys, 0, int32_t(hp), key0, -1 - std::min(lo, n_keys), int32_t(e - i)}});
      }
    }
    // backward tiles: every resident key of the document (those that nobody sees get zeros)
    const size_t s1 = p->slot_row.size(), n_blocks = (s1 - s0) / BWD_BQ;
    block_hi_min.resize(n_blocks), block_hi_max.resize(n_blocks), lo_from.resize(n_blocks), lo_upto.resize(n_blocks);
    for (size_t b = 0; b < n_blocks; ++b) {
      const int32_t *const lo = p->slot_lo.data() + s0 + b * BWD_BQ, *const hi = p->slot_pos.data() + s0 + b * BWD_BQ;
      block_hi_min[b] = hi[0], block_hi_max[b] = hi[BWD_BQ - 1];
      lo_from[b] = *std::min_element(lo, lo + BWD_BQ), lo_upto[b] = *std::max_element(lo, lo + BWD_BQ);
      if (b > 0) lo_upto[b] = std::max(lo_upto[b], lo_upto[b - 1]);
    }
    for (size_t b = n_blocks - 1; b-- > 0;) lo_from[b] = std::min(lo_from[b], lo_from[b + 1]);
    const int32_t doc_len = int32_t(p->doc_kv_len[dd]);
    auto first = [](const std::vector<int32_t> &v, int32_t at_least) { return std::lower_bound(v.begin(), v.end(), at_least) - v.begin(); };
    for (int32_t k0 = 0; k0 < doc_len; k0 += BWD_BN) {
      WindowUnit u{};
      u.kv_row = kv_row0 + k0, u.n_valid = std::min<int32_t>(BWD_BN, doc_len - k0), u.key_pos0 = k0, u.heads = g;
      const int64_t begin = first(block_hi_max, k0);
      int64_t end = k0 < p->sinks ? int64_t(n_blocks) : first(lo_from, k0 + BWD_BN);
      while (end > begin && p->slot_row[s0 + size_t(end - 1) * BWD_BQ] < 0) --end;  // pure padding
      end = std::max(begin, end);
      int64_t full = std::clamp<int64_t>(first(block_hi_min, k0 + BWD_BN - 1), begin, end), edge = std::clamp<int64_t>(first(lo_upto, k0 + 1), begin, end);
      if (full >= edge) full = edge = end;
      auto slot = [&](int64_t b) { return int32_t(s0 + size_t(b) * BWD_BQ); };
      u.slot_begin = slot(begin), u.slot_end = slot(end), u.slot_full = slot(full), u.slot_edge = slot(edge);
      btiles.push_back(u);
    }
    covered_kv += doc_len;
  }

  // longest first; unit index modulo KV heads = KV head (see the plan without a window)
  std::stable_sort(ftiles.begin(), ftiles.end(), [](const Tile &a, const Tile &b) { return a.cost > b.cost; });
  p->fwd_units.reserve(ftiles.size() * size_t(hq / hp));
  for (const Tile &t : ftiles)
    for (int i = 0; i < hq / hp; ++i) {
      FwdUnit u = t.u;
      u.head = (i % hkv) * g + (i / hkv) * hp;
      p->fwd_units.push_back(u);
      p->fwd_steps += t.cost;
    }

  // Backward: a tile with sinks is seen by every later row of its document, and a small batch has few units.  Units longer than what
  // each of the workgroups that run at a time would have, were the launch's work spread evenly, are cut along their query blocks, and
  // those with sinks that are longer than a quarter of that: they have one busy wave of four, and are better off beside others than first
  // (64K tokens, window 1024, 4 sinks, 32/8 heads: 5.68 -> 5.45 ms).  (A dQ half does 3 products per pair of its 128 rows and 64 keys, a
  // dK/dV step 4 of as many pairs.)
  auto steps = [](const BwdUnit &u) { return int64_t(u.slot_end - u.slot_begin) / BWD_BQ * u.heads; };
  for (const WindowUnit &u : btiles) p->bwd_steps += steps(u) * hkv;
  const int64_t slots = (p->d == 64 ? 3 : 2) * N_CU, mean = (p->bwd_steps + 2 * p->fwd_steps * 3 / 4) / slots;
  int64_t piece = std::max<int64_t>(24, mean);
  auto pieces_of = [&](const WindowUnit &u) {
    const int64_t n = steps(u), most = u.key_pos0 < p->sinks ? std::max<int64_t>(24, piece / 4) : piece;
    return n > most ? std::min((n + most - 1) / most, int64_t(u.slot_end - u.slot_begin) / BWD_BQ) : int64_t(1);
  };
  for (;; piece *= 2) {
    int64_t parts = 0;
    for (const WindowUnit &u : btiles)
      if (const int64_t k = pieces_of(u); k > 1) parts += k * hkv;
    if (size_t(parts) * part_bytes(p->d) <= MAX_PARTS) break;
  }
  std::vector<WindowUnit> tiles;
  std::vector<int32_t> parts_per_head;
  for (const WindowUnit &u : btiles) {
    const int64_t k = pieces_of(u), blocks = int64_t(u.slot_end - u.slot_begin) / BWD_BQ;
    for (int64_t i = 0; i < k; ++i) {
      WindowUnit v = u;
      v.slot_begin = int32_t(u.slot_begin + blocks * i / k * BWD_BQ), v.slot_end = int32_t(u.slot_begin + blocks * (i + 1) / k * BWD_BQ);
      v.slot_full = std::clamp(u.slot_full, v.slot_begin, v.slot_end), v.slot_edge = std::clamp(u.slot_edge, v.slot_begin, v.slot_end);
      v.count = 1, v.follow = k > 1 ? -1 - (p->n_bwd_parts + int32_t(i)) : 0;
      tiles.push_back(v);
      parts_per_head.push_back(k > 1 ? int32_t(k) : 0);
    }
    if (k > 1)
      for (int h = 0; h < hkv; ++h, p->n_bwd_parts += int32_t(k)) p->bwd_combine.push_back({p->n_bwd_parts, int32_t(k), u.kv_row, u.n_valid, h, 0});
  }
  // longest first; whole units of a few steps are chained: one workgroup runs tiles [a, b) of the list one after the other
  std::vector<size_t> order(tiles.size());
  for (size_t i = 0; i < order.size(); ++i) order[i] = i;
  std::stable_sort(order.begin(), order.end(), [&](size_t a, size_t b) { return steps(tiles[a]) > steps(tiles[b]); });
  struct Chain {
    size_t a, b;
    int64_t steps;
  };
  constexpr int64_t CHAIN_UNIT = 16, CHAIN_UNITS = 32;
  std::vector<Chain> chains;
  int64_t left = 0;
  for (const WindowUnit &u : tiles)
    if (steps(u) <= CHAIN_UNIT) left += steps(u) * hkv;
  for (size_t a = 0; a < order.size();) {
    int64_t sum = steps(tiles[order[a]]);
    size_t b = a + 1;
    if (sum <= CHAIN_UNIT && parts_per_head[order[a]] == 0) {
      const int64_t target = std::min<int64_t>(64, left / (4 * N_CU));
      while (b < order.size() && parts_per_head[order[b]] == 0 && sum + steps(tiles[order[b]]) <= target && int64_t(b - a) < CHAIN_UNITS) sum += steps(tiles[order[b++]]);
      left -= sum * hkv;
    }
    chains.push_back({a, b, sum});
    a = b;
  }
  std::stable_sort(chains.begin(), chains.end(), [](const Chain &x, const Chain &y) { return x.steps > y.steps; });
  p->bwd_workgroups = int32_t(chains.size() * size_t(hkv));
  p->window_units.resize(size_t(p->bwd_workgroups));
  for (size_t c = 0; c < chains.size(); ++c)
    for (int h = 0; h < hkv; ++h) {
      WindowUnit u = tiles[order[chains[c].a]];
      u.kv_head = h, u.count = int32_t(chains[c].b - chains[c].a);
      if (const int32_t k = parts_per_head[order[chains[c].a]]) u.follow -= h * k;  // the parts of a head are neighbours
      else if (u.count > 1) u.follow = int32_t(p->window_units.size());
      p->window_units[c * size_t(hkv) + size_t(h)] = u;
      for (size_t t = chains[c].a + 1; t < chains[c].b; ++t) {
        WindowUnit f = tiles[order[t]];
        f.kv_head = h, f.count = 0;
        p->window_units.push_back(f);
      }
    }
  // workspace of backward: per (head, slot) -Delta and log2(e) * LSE, both once more in the order of dK/dV's tiles, and the parts
  const size_t per = (p->slot_row.size() * size_t(hq) * sizeof(float) + 255) / 256 * 256;
  p->ws_off_l2 = per, p->ws_off_stats_kv = 2 * per;
  p->ws_bwd = p->ws_off_parts_kv = 4 * per;
  p->ws_bwd += size_t(p->n_bwd_parts) * part_bytes(p->d);
  p->ws_bwd_split = p->ws_bwd;
  p->q_covered = covered_q == p->total_q;
  p->kv_covered = covered_kv == p->total_kv;
  return true;
}

}  // namespace ca
