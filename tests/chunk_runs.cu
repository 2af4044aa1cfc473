// The way the attention kernels for chunks share out their work, on the host: the sums, borders and steps are the kernels' own, from paged_chunk.cuh; only the
// searches, which the kernels do 32 places at a time, are done one by one here.  Built and called by test_chunk_runs.py.
#include "paged_chunk.cuh"

namespace {

using paged::ChunkParams;
using paged::ChunkWalk;

// Where the runs of `grid` CTAs begin, and behind them where the last one ends: (sequence, head, tile, unit) each.  The sum of costs, or -1 where one is below 0 or the
// sum leaves 32 bits.
template <int R, int KEYS, int ITEM_COST, int SNAP, int MIN_RUN>
int64_t play(ChunkParams p, int64_t tiles, int grid, int32_t *begins) {
  typedef paged::ChunkRuns<R, KEYS, ITEM_COST, SNAP, MIN_RUN> Share;
  Share::set(p, grid, tiles);
  const Share runs(p);
  int64_t total = 0;
  for (int i = 0; i < p.n; ++i) {
    ChunkWalk w{i};
    runs.enter(w);
    if (runs.wrong(w)) return -1;
    const int of_head = runs.upto(w, w.tiles);
    if (of_head < 0 || (int64_t)of_head * p.Hkv > INT32_MAX) return -1;
    total += (int64_t)of_head * p.Hkv;
  }
  if (total > INT32_MAX) return -1;
  const int run = max(((MIN_RUN * KEYS * p.group) >> p.shift) + 1, p.grid_of.quot((int)total) + 1);
  for (int c = 0; c <= grid; ++c) {
    int64_t x = min((int64_t)run * c, total);
    ChunkWalk w{p.n};
    if (x < total) {
      int64_t at = 0;
      for (int i = 0; i < p.n; ++i) {                              // the last that begins at or in front of it
        ChunkWalk y{i};
        runs.enter(y);
        const int64_t of = (int64_t)runs.upto(y, y.tiles) * p.Hkv;
        if (at > x) break;
        w = y;
        if (at + of > x) break;
        at += of;
      }
      x -= at;
      const int each = runs.upto(w, w.tiles);
      w.head = (int)(x / each);
      x -= (int64_t)w.head * each;
      int lo = 0, hi = w.tiles;                                    // the last tile that begins at or in front of it
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (runs.upto(w, mid) <= x ? lo : hi) = mid;
      }
      w.rt = lo;
      x -= runs.upto(w, lo);
      w.units = runs.units_of(w, lo);
      const int unit = p.unit_of.quot((int)(x << p.shift)) - ITEM_COST;
      w.unit = unit <= p.snap ? 0 : unit;
      if (w.unit > 0 && w.units - unit <= p.snap) runs.next_item(w);
    }
    const int32_t to[4] = {w.s, w.head, w.rt, w.unit};
    for (int k = 0; k < 4; ++k) begins[4 * c + k] = to[k];
  }
  return total;
}

}  // namespace

// tc: the tcgen05 kernel; costs and borders as the kernels' sources have them.  tiles: what the call's checks make of the sizes.
extern "C" int64_t chunk_runs(int tc, const int32_t *lens, const int32_t *starts, int n, int rows, int Hkv, int group, int cap, int64_t tiles, int grid, int32_t *begins) {
  ChunkParams p{};
  p.lens = lens; p.starts = starts;
  p.n = n; p.rows = rows; p.Hkv = Hkv; p.group = group; p.H = Hkv * group; p.cap = cap; p.max_seqs = n; p.max_pages = 1;
  p.group_of.set(group);
  if (tc) return play<paged::CHUNK_TC_ROWS, 64, TC_ITEM_COST, TC_SNAP, TC_MIN_RUN>(p, tiles, grid, begins);
  return play<paged::CHUNK_ROWS, 64, ROW_ITEM_COST, ROW_SNAP, ROW_MIN_RUN>(p, tiles, grid, begins);
}
