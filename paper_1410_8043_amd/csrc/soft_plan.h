// What a call of ps_soft.hip takes of its handle's workspace, and how it cuts its work into pieces: host code without a
// device call, so that it is also built and checked by the host's compiler.
#pragma once

#include <algorithm>
#include <cstdint>

#include "../../include/ps_soft.h"

namespace pssoft {

constexpr int kMaxK = 512, kMaxTop = 256;
constexpr int64_t kMaxRows = 1LL << 26;  // a record holds 32 row + item mod 32 in 32 bits
constexpr int64_t kMaxItems = (1LL << 31) - 65, kMaxEntries = (1LL << 31) - 65;

constexpr int kTile = 32;        // rows of a packed tile, and of a matrix instruction
constexpr int kFrag = 512;       // halves of one fragment: 64 lanes x 8
constexpr int kParts = 256;      // workgroups, and partial maxima, of each table's scan
constexpr int kRowParts = 4096;  // most workgroups, and partial maxima, of the row scan
constexpr int kScalBytes = 16;   // scalars that the kernels share
constexpr int kWaves = 4;        // wavefronts of a pass's workgroup: 128 own rows
constexpr int kBins = 1024, kSortTile = 4096;  // digits of a sorting pass, records of a workgroup
constexpr int kTopGroup = 64;    // items of a group
constexpr int kScoreTiles = 2;   // tiles of 32 items that a step of the search stages
constexpr int kCandidates = 1024;

// A handle's table and options
struct Shape {
  int64_t items = 0;
  int32_t K = 0, type = 0;
  int32_t splits = 0, search = -1;
};

// Offsets into the workspace, taken in order
struct Arena {
  int64_t at = 0;
  int64_t take(int64_t bytes) {
    const int64_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  }
};

inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Sizes and places of one call's intermediate values
struct Plan {
  int32_t np, k16, kd;
  int64_t n, entries, xt, wt;  // rows, entries, tiles of each table
  bool few;                    // the loss alone of few rows: k_few instead of the packed tables and the pass
  int64_t few_items;           // of a piece
  bool want_dx, want_dw;
  int64_t x_stride, w_stride;  // halves per tile
  int32_t rsplits, csplits;
  int64_t rper, cper;          // tiles per split
  int32_t sort_blocks, passes, bits;  // of the sort: bits of a pass
  int64_t key[2], pay[2], act, total, extra, share, gw, logz, row_part, part, scal, px, pw, m, l, o, rowvec, hist, bins, first;
  int64_t bytes;
};

// Chunks of 16 numbers that rows are padded to: the passes are built for these
inline int32_t padded_chunks(int32_t K) {
  for (int32_t c : {2, 4, 6, 8, 12, 16})
    if (K <= 16 * c) return c;
  return 32;
}

// Pieces of the reduced axis, each its own workgroups: enough of them for 256 CUs three times over, and a multiple
// of 8 where the axis is long: workgroup b runs on XCD b mod 8 and takes piece b mod pieces, so the
// part of the stream that an XCD's L2 sees is an eighth of it.  No piece shorter than 8 tiles, or than 2 where 8 would
// leave CUs idle (a tile takes about 1 us, a piece's start and its part of the join about 2).
inline int32_t pieces(int64_t own_tiles, int64_t tiles, int32_t forced) {
  const int64_t groups = up(own_tiles, kWaves);
  if (forced > 0) return static_cast<int32_t>(std::max<int64_t>(1, std::min({static_cast<int64_t>(forced), tiles, (static_cast<int64_t>(1) << 30) / groups})));
  // 512 workgroups run at once.  Up to two rounds of them 4 pieces fill the last round (550 workgroups of K = 128 fp32, 8192 streamed
  // rows: 1 piece 917 us with the join, 2 801, 4 765, 8 824; 782: 1218, 1133, 1108, 1156); from there on the rounds are
  // many and a piece more only costs its part of the join (1000, K = 128 bf16, 4096 rows: 391, 406, 445, 530; 2200: 889, 921,
  // 997, 1208; 4500: 1771, 1843, 2030, 2418).  Longer streams differ less (1000, 32,768 rows: 2942, 2929, 2949, 3025)
  if (groups >= 512) return static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(tiles / 8, groups >= 1000 ? 1 : 4)));
  const int64_t most = std::max<int64_t>(1, groups * (tiles / 8) < 256 ? std::min(up(256, groups), tiles / 2) : tiles / 8);
  int64_t want = up(768, groups);
  if (most >= 8) want = up(want, 8) * 8;
  return static_cast<int32_t>(std::min({want, most, static_cast<int64_t>(256)}));
}

constexpr int64_t kFewRows = 4096;
inline int64_t few_rows(int64_t n) { return n >= 8 ? 8 : n >= 3 ? 4 : 1; }  // that share a read of W

// room: enough for calls of fewer rows too, whose pieces may be more (ps_soft_reserve)
inline Plan plan(const Shape *h, int64_t n, int64_t entries, bool dx, bool dw, bool room = false) {
  Plan p{};
  p.np = h->type == PS_SOFT_F32 ? 2 : 1;
  p.k16 = padded_chunks(h->K);
  p.kd = p.k16 / 2;
  p.n = n;
  p.entries = entries;
  p.xt = std::max<int64_t>(1, up(n, kTile));  // no row: the plan of one, of which nothing is launched
  p.wt = up(h->items, kTile);
  p.want_dx = dx;
  p.want_dw = dw;
  p.x_stride = static_cast<int64_t>(p.np) * kFrag * (p.k16 + (dw ? 2 * p.kd : 0));
  p.w_stride = static_cast<int64_t>(p.np) * kFrag * (p.k16 + (dx ? 2 * p.kd : 0));
  p.rsplits = pieces(p.xt, p.wt, h->splits);
  p.rper = up(p.wt, p.rsplits);
  p.rsplits = static_cast<int32_t>(up(p.wt, p.rper));
  // in us: packing and the pass take about 12 and the packing's bytes.  One user, 17,770 items, K = 128: 32 -> 22
  const double scores = static_cast<double>(n) * static_cast<double>(h->items);
  p.few = !dx && !dw && h->splits == 0 && n <= kFewRows && scores * (5 + 0.065 * h->K) * 1e-6 < 12 + h->items * 4e-6 * h->K;
  if (p.few) {
    const int64_t rows = up(std::max<int64_t>(n, 1), few_rows(n)), most = up(h->items, kTopGroup);
    p.few_items = up(h->items, std::min<int64_t>(most, up(1024, rows)));
    p.few_items = up(p.few_items, 32) * 32;
    p.rsplits = static_cast<int32_t>(up(h->items, p.few_items));
  }
  p.csplits = 0;
  p.cper = 1;
  if (dw) {
    p.csplits = pieces(p.wt, p.xt, h->splits);
    p.cper = up(p.xt, p.csplits);
    p.csplits = static_cast<int32_t>(up(p.xt, p.cper));
  }
  p.sort_blocks = static_cast<int32_t>(up(entries, kSortTile));
  int32_t bits = 0;
  for (int64_t v = p.wt; v > 0; v >>= 1) ++bits;  // keys 0 .. tiles
  p.passes = (bits + 9) / 10;
  p.bits = (bits + p.passes - 1) / p.passes;
  Arena a;
  for (int q = 0; q < 2; ++q) {
    p.key[q] = a.take(dw ? entries * 4 : 0);
    p.pay[q] = a.take(dw ? entries * 8 : 0);
  }
  p.act = a.take(n * 4);
  p.total = a.take(n * 4);
  p.extra = a.take(n * 4);
  p.share = a.take(n * 4);
  p.gw = a.take(n * 4);
  p.logz = a.take(n * 8);
  p.row_part = a.take(kRowParts * 4);
  p.part = a.take(2 * kParts * 4);
  p.scal = a.take(kScalBytes);
  p.px = a.take(p.few ? 0 : p.xt * p.x_stride * 2);
  p.pw = a.take(p.few ? 0 : p.wt * p.w_stride * 2);
  int64_t rpad = p.rsplits * p.xt * kTile, cpad = p.csplits * p.wt * kTile;
  if (room) {
    // g workgroups of own tiles take at most max(768 / g + 8, 256 / g + 1, 4) pieces (pieces(), or the forced number), and
    // one row in a piece of k_few's at most 1024 + 32 blocks' pieces of 32 padded rows
    const int64_t gx = up(p.xt, kWaves), gw = up(p.wt, kWaves), force = h->splits;
    rpad = std::max<int64_t>(kWaves * kTile * (force > 0 ? force * gx : 768 + 9 * gx), 1056 * kTile + 2 * kFewRows);
    cpad = kWaves * kTile * (force > 0 ? force * gw : 768 + 9 * gw);
  }
  p.m = a.take(std::max(rpad, cpad) * 4);
  p.l = a.take(rpad * 4);
  p.o = a.take(std::max(dx ? rpad : 0, cpad) * p.kd * 32 * 4);
  p.rowvec = a.take(dw ? p.xt * 64 * 4 : 0);
  p.hist = a.take(dw ? static_cast<int64_t>(p.sort_blocks) * kBins * 4 : 0);
  p.bins = a.take(kBins * 4);
  p.first = a.take(dw ? (p.wt + 1) * 8 : 0);
  p.bytes = a.at;
  return p;
}

// Chunks of 16 numbers, the bound's among them, that the search's passes are built for
inline int32_t score_chunks(int32_t K) {
  for (int32_t c : {2, 3, 5, 7, 9, 13, 17, 25})
    if (K + 1 <= 16 * c) return c;
  return 33;
}

struct TopPlan {
  bool filter;
  int64_t rows;  // rows of one launch: what they need stays near a gigabyte
  int32_t words, kc, groups;
  int64_t xt, wt, steps, per_split, per_row;
  int32_t splits;
  int64_t bits, key, maxima, part, px, pw, most, least, found, count, bytes;
};

// The form estimated faster, in us.  Measured (all scores / candidates): 64 rows x 17,770 items K = 64 30 / 77, 256 rows
// 66 / 79, 1024 rows 180 / 89; 256 rows x 100,000 items K = 16 160 / 75; 8 rows x 100,000 K = 256 43 / 135
inline bool top_by_candidates(int64_t n, int64_t items, int32_t K) {
  const double scores = static_cast<double>(n) * static_cast<double>(items);
  const double all = 17.0 + scores * (5.0 + 0.065 * K) * 1e-6;
  const double candidates = 60.0 + 0.2 * K + 0.01 * n + items * 1e-6 * K + scores * 0.006e-6 * K;
  return all > candidates;
}

inline TopPlan top_plan(const Shape *h, int64_t n, int32_t k, bool exclude, int32_t search) {
  TopPlan p{};
  const int64_t all = std::max<int64_t>(n, 1);
  p.words = static_cast<int32_t>(up(h->items, 32));
  // a threshold needs more groups of 16 items than k: 64 k items leave about k / 8 candidates more than k
  p.filter = h->items >= 64LL * k && top_by_candidates(all, h->items, h->K);
  if (search >= 0) p.filter = search == 1;
  p.filter = p.filter && h->items < 1 << 30;  // counts of candidates
  Arena a;
  if (p.filter) {
    p.kc = score_chunks(h->K);
    p.wt = up(h->items, kTile);
    p.steps = up(p.wt, kScoreTiles);
    const int64_t per_row = (exclude ? p.words * 4LL : 0) + p.steps * 16 + 32 + kCandidates * 4 + (p.kc + 1) * 32;
    p.rows = std::min(all, std::max<int64_t>(256, (1LL << 30) / per_row / 256 * 256));
    p.xt = up(p.rows, kTile);
    // two workgroups a CU at once: 512, as multiples of 8 pieces (one XCD's L2 sees its eighth of the items)
    const int64_t groups = up(p.xt, 2 * kWaves), want = std::max<int64_t>(1, 512 / groups);
    p.splits = static_cast<int32_t>(std::min<int64_t>(p.steps, h->splits > 0 ? h->splits : want >= 8 ? want / 8 * 8 : want));
    p.per_split = up(up(p.steps, p.splits), 2) * 2;
    p.splits = static_cast<int32_t>(up(p.steps, p.per_split));
    p.per_row = up(p.steps, 2) * 8;
    p.part = a.take(2 * kParts * 4);
    p.px = a.take(p.xt * (p.kc + 1) * kFrag * 2);
    p.pw = a.take(p.wt * p.kc * kFrag * 2);
    p.most = a.take(p.rows * p.per_row * 4);
    p.least = a.take(p.rows * 4);
    p.found = a.take(p.rows * kCandidates * 4);
    p.count = a.take(p.rows * 4);
    p.bits = a.take(exclude ? p.rows * p.words * 4 : 0);
  } else {
    p.groups = static_cast<int32_t>(up(h->items, kTopGroup));
    p.rows = std::min(all, std::max<int64_t>(1, (1LL << 30) / (8LL * p.groups * (kTopGroup + 1))));
    p.rows = std::min<int64_t>(p.rows, 32768);  // rows are the launch's second dimension
    p.key = a.take(p.rows * p.groups * kTopGroup * 8);
    p.maxima = a.take(p.rows * p.groups * 8);
  }
  p.bytes = a.at;
  return p;
}

// What any call of at most n rows, `entries` targets or exclusions and `top` items per row takes
inline int64_t reserved_bytes(const Shape *h, int64_t n, int64_t entries, int32_t top) {
  int64_t bytes = plan(h, n, entries, true, true, true).bytes;
  if (top > 0) {
    // what either form takes; the first's rows end where the second is faster, unless `top` rules that out
    int64_t all = n;
    if (h->search < 0 && h->items >= 64LL * top && top_by_candidates(n, h->items, h->K)) {
      int64_t lo = 0;
      while (lo < all) {
        const int64_t mid = (lo + all) / 2;
        if (top_by_candidates(mid, h->items, h->K)) all = mid; else lo = mid + 1;
      }
    }
    // without exclusions more rows share a launch, which can take more room
    for (bool exclude : {false, true})
      bytes = std::max({bytes, top_plan(h, all, top, exclude, 0).bytes, top_plan(h, n, top, exclude, 1).bytes});
  }
  return bytes;
}

}  // namespace pssoft
