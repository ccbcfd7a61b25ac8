// How one batch of finch_attend is launched (host only): which problems go to which kernel, how the keys of a tile of rows are
// dealt out to workgroups, and the table that tells a workgroup its piece of work.
#pragma once

#include <algorithm>
#include <cmath>

#include "attend_common.h"
#include "context.h"

namespace finch {

// Most stacked rows of a problem that go to attend_rows: its waves read K and V once for 32 rows, attend_tiles once for 256, but with most of
// its waves idle.  16 requests of 20000 keys, 4 heads on each of 8: 64 rows 279 us there and 328 here, 96 rows 475 and 327; one request of
// 128 rows on 20000 keys 45 and 32.
constexpr int kSomeRows = 64;
constexpr int kLaunchGrid = (1 << 22) - 1;  // workgroups of a launch: fewer than 2^32 threads
constexpr int64_t kMostPieces = int64_t{1} << 30;  // workgroups of a batch: their numbers are 32 bits

// Neighbours in a batch with as many tiles of rows and of keys; where a batch has more such groups than a launch has runs,
// neighbours that are near to it, with the most of either (and what lies between them).
struct AttendGroup {
  int64_t problem, count;
  int64_t levels, keys;  // tiles of rows of a problem, of keys
  int64_t tiles;         // tiles of rows that are there
  bool causal;
};

// The launch of one kernel, and of the join of its splits.
struct AttendLaunch {
  int tile_rows, tile_keys, rows_lo, rows_hi;
  int rows_max = 0;
  // tiles of rows, tiles of keys that these see, most tiles of keys
  int64_t tiles = 0, work = 0, keys_max = 0;
  int groups = 0, runs = 0;
  int64_t span = 1, most_splits = 1, workgroups = 0, slots = 0;
  size_t off_o = 0, off_ml = 0;
  AttendGroup group[kMostRuns];
  AttendRun run[kMostRuns];
  int64_t start[kMostRuns];
  // of the problem that came last: sizes, tiles of rows, of keys, what it adds to `work`
  int32_t n_que = -1, c = 0, m = 0;
  int64_t levels = 0, keys = 0, sees = 0;

  AttendLaunch(int tile_rows_, int tile_keys_, int lo, int hi) : tile_rows(tile_rows_), tile_keys(tile_keys_), rows_lo(lo), rows_hi(hi) {}

  // Fewer groups: neighbours become one where that adds the least idle work, an ever larger share of it until enough have.
  void merge() {
    const auto volume = [](const AttendGroup& g) { return static_cast<double>(g.count) * g.levels * std::max<int64_t>(g.keys, 1); };
    for (double more = 1.25; groups > kMostRuns / 2; more *= 1.5) {
      int n = 0;
      for (int i = 1; i < groups; ++i) {
        const AttendGroup &a = group[n], &b = group[i];
        const AttendGroup both = {a.problem, b.problem + b.count - a.problem, std::max(a.levels, b.levels), std::max(a.keys, b.keys), a.tiles + b.tiles,
                                  a.causal && b.causal};
        if (volume(both) <= more * (volume(a) + volume(b))) {
          group[n] = both;
        } else {
          group[++n] = b;
        }
      }
      groups = n + 1;
    }
  }

  void add(const finch_attention& a, int64_t problem, int64_t rows) {
    AttendGroup* const last = groups > 0 ? &group[groups - 1] : nullptr;
    // (mostly as the one before, another head of the same request)
    const bool again = last && last->problem + last->count == problem && a.n_que == n_que && a.c == c && a.m == m && (a.causal != 0) == last->causal;
    if (!again) {
      const auto tiles_of = [](int64_t n, int tile) { return (n + tile - 1) >> __builtin_ctz(static_cast<unsigned>(tile)); };
      n_que = a.n_que, c = a.c, m = a.m;
      levels = tiles_of(rows, tile_rows);
      keys = tiles_of(c, tile_keys) + tiles_of(m, tile_keys);
      // (causal rows of the chunk itself see half of themselves on average)
      sees = levels * (keys - (a.causal ? std::min(n_que, m) / 2 >> __builtin_ctz(static_cast<unsigned>(tile_keys)) : 0));
      keys_max = std::max(keys_max, keys);
      rows_max = std::max(rows_max, static_cast<int>(rows));
    }
    tiles += levels;
    work += sees;
    if (again || (last && last->problem + last->count == problem && last->levels == levels && last->keys == keys && last->causal == (a.causal != 0))) {
      ++last->count;
      last->tiles += levels;
      return;
    }
    if (groups == kMostRuns) merge();
    group[groups++] = AttendGroup{problem, 1, levels, keys, levels, a.causal != 0};
  }

  // Tiles of keys that a split has at most.  Where tiles of rows are too few for the chip, the keys each sees are dealt out to several
  // workgroups, so that there are about as many as the chip takes.
  void choose_span(bool many, int64_t cu) {
    // (a join takes its time with the number of splits, so that it is shortest with the square root of all tiles)
    const int64_t least = std::max<int64_t>(many ? 8 : 4, static_cast<int64_t>(std::sqrt(0.5 * static_cast<double>(keys_max))));
    // Few rows: two workgroups a compute unit are on the chip at once, and as many are enough where they are alike or few (one request,
    // 131000 keys in 8 bits: 60 us, 73 with twice as many; 512 problems of 2000 keys 92 and 108 us); problems of different
    // length level out with twice as many (512 of 64 to 8192 keys 224 us, 236 with half).
    // Many rows: one workgroup a compute unit, whose eight waves fill it (256 rows of 4 heads on 8 heads' 20000 keys 95 us, 112 with
    // twice as many).
    const bool alike = 4 * keys_max * tiles <= 5 * work || tiles < cu;
    const int64_t at_once = many ? cu : (alike ? 2 : 4) * cu;
    span = std::max((work + at_once - 1) / at_once, least);
    if (!many || tiles < cu) return;
    // Where there is a tile of rows for each compute unit, what most of them see is not split: partial results cost more than an uneven
    // end.  Problems with more keys than that and than a compute unit's share of all work would be the end alone, and are.
    const AttendGroup* bulk = &group[0];
    for (int i = 1; i < groups; ++i)
      if (group[i].tiles > bulk->tiles || (group[i].tiles == bulk->tiles && group[i].keys < bulk->keys)) bulk = &group[i];
    span = std::max(span, bulk->keys);
  }

  int64_t splits_of(const AttendGroup& g) const { return std::max<int64_t>(1, (g.keys + span - 1) / span); }

  finch_status deal(bool many, int64_t cu, int head_dim, int heads, size_t& off) {
    if (tiles == 0) return FINCH_OK;
    if (tiles > kMostPieces) return FINCH_ERR_CAPACITY;
    choose_span(many, cu);
    // partial results of at most 64 MiB, and a counter for each
    const int64_t bytes = int64_t{tile_rows} * (head_dim + 2) * 4, most = std::min<int64_t>((int64_t{64} << 20) / bytes, kAttendMeetWords);
    for (;;) {
      slots = 0;
      for (int i = 0; i < groups; ++i)
        if (splits_of(group[i]) > 1) slots += group[i].count * group[i].levels * splits_of(group[i]);
      if (slots <= most) break;
      span = std::min(keys_max, std::max(span + 1, span * slots / most));
    }
    // One run for all, in the batch's order, where that has no more workgroups than are on the chip at once, or none that has nothing to
    // do: looking up the run takes time at a kernel's start (20 problems of 3 rows on 3751 to 7414 keys 18.2 us, 19.1 with four runs).
    AttendGroup all = group[0];
    int64_t real = 0;
    for (int i = 0; i < groups; ++i) {
      const AttendGroup& g = group[i];
      all = AttendGroup{all.problem, g.problem + g.count - all.problem, std::max(all.levels, g.levels), std::max(all.keys, g.keys), tiles, all.causal && g.causal};
      real += g.count * g.levels * splits_of(g);
    }
    const int64_t whole = all.count * all.levels * splits_of(all);
    if ((whole <= (many ? cu : 2 * cu) || whole == real) && (splits_of(all) == 1 || whole <= most)) {
      groups = 1;
      group[0] = all;
      slots = splits_of(all) > 1 ? whole : 0;
    }
    // Runs.  Those whose workgroups have the most to do start first; with tiles of rows that see more or less (many rows, causal) a group is
    // cut into three (packed prompts of 58 to 2048 rows: 109.4 us, 113.9 uncut, 111.4 in six: then neighbours in time share fewer keys).
    const int cuts = many ? std::min(3, kMostRuns / groups) : 1;
    int64_t length[kMostRuns], slot = 0;
    for (int i = 0; i < groups; ++i) {
      const AttendGroup& g = group[i];
      const int64_t splits = splits_of(g), n = splits > 1 || groups == 1 ? 1 : std::min<int64_t>(g.levels, cuts);
      for (int64_t c = 0; c < n; ++c) {
        const int64_t top = g.levels - g.levels * c / n - 1, levels = top + 1 - (g.levels - g.levels * (c + 1) / n);
        const int64_t less = g.causal ? (g.levels - 1 - top) * tile_rows / (int64_t{heads} * tile_keys) : 0;
        const int64_t has = std::max<int64_t>(1, (g.keys - less + splits - 1) / splits);
        int at = runs++;
        for (; at > 0 && length[at - 1] < has; --at) {
          length[at] = length[at - 1];
          run[at] = run[at - 1];
        }
        length[at] = has;
        run[at] = AttendRun{static_cast<int32_t>(g.problem), static_cast<int32_t>(g.count), static_cast<int32_t>(top), static_cast<int32_t>(levels),
                            static_cast<int32_t>(splits), static_cast<int32_t>(slot)};
      }
      if (splits > 1) slot += g.count * g.levels * splits;
      most_splits = std::max(most_splits, splits);
    }
    for (int r = 0; r < runs; ++r) {
      start[r] = workgroups;
      workgroups += int64_t{run[r].count} * run[r].levels * run[r].splits;
    }
    if (workgroups > kMostPieces) return FINCH_ERR_CAPACITY;
    if (slots > 0) {
      off_o = off = std::max<size_t>(off, 256);  // (behind the status word that other calls keep there)
      off = align_up(off + static_cast<size_t>(slots) * tile_rows * head_dim * 4, 256);
      off_ml = off;
      off = align_up(off + static_cast<size_t>(slots) * tile_rows * 8, 256);
    }
    return FINCH_OK;
  }

  // The table for the kernel's workgroups.
  void table(AttendParams& p) const {
    p.rows_lo = rows_lo;
    p.rows_hi = rows_hi;
    p.most_splits = static_cast<int32_t>(most_splits);
    p.span = static_cast<int32_t>(span);
    p.base = 0;
    p.runs = runs;
    p.one = run[0];
    for (int r = 0; r < runs; ++r) {
      p.start[r] = static_cast<int32_t>(start[r]);
      p.run[r] = run[r];
    }
  }
  // That of the join: runs with splits, numbered by tiles of rows.  Returns how many tiles there are; problems: theirs.
  int join_table(AttendParams& p, int& problems) const {
    int64_t at = 0;
    p.runs = problems = 0;
    for (int r = 0; r < runs; ++r) {
      if (run[r].splits == 1) continue;
      if (p.runs == 0) p.one = run[r];
      p.start[p.runs] = static_cast<int32_t>(at);
      p.run[p.runs++] = run[r];
      problems += run[r].count;
      at += int64_t{run[r].count} * run[r].levels;
    }
    return static_cast<int>(at);
  }
};

// Problems of few rows, of some and of many go to kernels of their own; fp32 ones all to one (`some`).
struct AttendPlan {
  AttendLaunch few, some, many;
  bool eight = false;
  size_t bytes = 0;
  explicit AttendPlan(bool bf16)
      : few(kRows16, kRowsKeys, 1, kRows16),
        some(bf16 ? AttendLaunch(kRowsTile, kRowsKeys, kRows16 + 1, kSomeRows) : AttendLaunch(kF32Tile, kF32Keys, 1, INT32_MAX)),
        many(kTilesRows, kTilesKeys, kSomeRows + 1, INT32_MAX) {}
};

}  // namespace finch
