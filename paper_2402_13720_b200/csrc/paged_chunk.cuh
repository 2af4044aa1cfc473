// How the attention kernels for chunks of new tokens share out their work.
//
// A sequence has m new tokens, the newest of its len; they and the query heads of a kv head's group are its m * group query rows, token by token.  An
// item is a sequence's kv head and a tile of R rows; KEYS keys of an item are a unit, and an item has as many as its last row sees.  Items in order
// (sequence, head, tile) are dealt out to the CTAs in runs of equal cost; a run begins within an item unless that is within SNAP units of the item's
// border.  Every CTA works this out for itself from the lengths, so that there is no planning call; what is cut leaves pieces (maximum, sum, unnormalised
// output, in 32 bits), and a second kernel adds them up in ascending order: the same call gives the same bits.
// An item's cost is that of its keys, group times their number, and ITEM_COST units for filling and draining the chain.  It grows by R from one tile to
// the next of a sequence, so that the cost of the first k tiles is a polynomial of k and a run's beginning is found without a walk over the tiles: this is the
// first that a CTA does, a chain of dependent instructions that nothing hides.
#pragma once

#include "paged_runs.cuh"

namespace paged {

struct ChunkParams {
  const uint8_t *k, *v;                             // of the layer
  const int32_t *table, *lens, *seqs, *starts;
  const void *q;
  void *out;
  float *lse;
  int *status;
  int4 *begins;                                     // [CTA] where its run begins: sequence (-1: it has none), head, tile, unit
  float *pieces;                                    // [CTA][2][R][D], then [CTA][2][R][2]
  int64_t page_bytes, slot_bytes, head_bytes, q_stride;
  int n, rows, H, Hkv, group;                       // rows: of q (tokens)
  int n_pages, max_pages, max_seqs, cap, layer, head_dim;
  Div page, group_of, unit_of, grid_of;             // unit_of: KEYS * group
  int shift, snap;                                  // costs are counted in 2^shift; units from an item's border that are not cut off
  float scale_log2;
  uint32_t wait_limit;
  bool wide_out;                                    // out is a multiple of 32 bytes
};

// The tcgen05 kernel (paged_chunk_tc.cu); cost, tiles: units and row tiles of the call at most; 0: does not take the call.  And the join of its pieces (paged_chunk.cu).
int chunk_tc(const ouro_paged_cache *c, const ChunkParams &p, int64_t cost, int64_t tiles, cudaStream_t s, int *status);
int chunk_tc_join(const ChunkParams &p, int grid, cudaStream_t s);

// A place in the list of units.
struct ChunkWalk {
  int s, head, rt, unit, units;                     // units of the item
  int len, m, tiles, start;                         // of the sequence: tokens, new ones, row tiles, first row of q
  const int32_t *row;                               // of the table
};
__device__ __forceinline__ bool same(const ChunkWalk &a, const ChunkWalk &b) { return a.unit == b.unit && a.rt == b.rt && a.head == b.head && a.s == b.s; }

template <int R, int KEYS, int ITEM_COST, int SNAP, int MIN_RUN>
struct ChunkRuns {
  const ChunkParams &p;

  // Whether items of so many keys are worth cuts, and with them a second launch.
  static bool may_cut(int keys) { return (keys + KEYS - 1) / KEYS >= (SNAP > 1 ? 2 * SNAP + 2 : 4); }
  __host__ __device__ __forceinline__ explicit ChunkRuns(const ChunkParams &params) : p(params) {}
  // What is known of a sequence; no tokens outside the table.
  __host__ __device__ __forceinline__ int enter(ChunkWalk &w) const {       // (its row of the table)
    int sid = p.seqs ? p.seqs[w.s] : w.s;
    const bool known = sid >= 0 && sid < p.max_seqs;
    if (!known) sid = 0;
    w.len = known ? min(max(p.lens[sid], 0), p.cap) : 0;
    w.row = p.table + (int64_t)sid * p.max_pages;
    w.start = p.starts[w.s];
    w.m = p.starts[w.s + 1] - w.start;
    w.tiles = (w.m * p.group + R - 1) / R;
    return sid;
  }
  // Brings what every CTA reads of the parameters near, before it waits for the kernel in front.
  __device__ __forceinline__ void touch() const {
    asm volatile("" ::"l"(p.table), "l"(p.lens), "l"(p.seqs), "l"(p.starts), "l"(p.q), "r"(p.n), "r"(p.group), "r"(p.cap), "r"(p.unit_of.mul), "r"(p.shift), "r"(p.wait_limit));
  }
  __host__ __device__ __forceinline__ bool wrong(const ChunkWalk &w) const { return w.start < 0 || w.m < 0 || w.start > p.rows - w.m; }
  // Keys that row r (of the sequence's m * group) sees; below 1: none.
  __host__ __device__ __forceinline__ int sees(const ChunkWalk &w, int r) const { return w.len - w.m + 1 + p.group_of.quot(r); }
  __host__ __device__ __forceinline__ int units_of(const ChunkWalk &w, int rt) const {
    const int last = min(w.m * p.group - 1, rt * R + R - 1);
    return max(1, (sees(w, last) + KEYS - 1) / KEYS);
  }
  // Cost of the first k tiles of a head.  It grows from the first tile on that sees a key: what a sequence has of new tokens beyond its length may be far more than a row
  // of the table holds, and what it costs must not grow with their square.  Whatever has a tile costs something, or the first run would begin behind it.
  __host__ __device__ __forceinline__ int upto(const ChunkWalk &w, int k) const {
    const uint32_t first = p.group * (max(w.len - w.m, 0) + ITEM_COST * KEYS) + R;
    const uint32_t seeing = max(k - (int)((uint32_t)max(w.m - w.len, 0) * p.group / R), 0);
    return max((int)(((uint64_t)(uint32_t)k * first + (uint64_t)seeing * (seeing - 1) * (R / 2)) >> p.shift), min(k, 1));
  }
  // What the host sets for a launch; tiles: of all sequences at most.
  // tiles * Hkv is at most MAX_ITEMS, so that the sum of costs, each up to 1 more than its part of `most`, stays below 2^31.
  static constexpr int64_t MAX_ITEMS = (int64_t)1 << 30;
  static void set(ChunkParams &p, int grid, int64_t tiles) {
    p.unit_of.set(KEYS * p.group);
    p.grid_of.set(grid);
    p.snap = may_cut(p.cap) ? SNAP : INT32_MAX;
    // (a tile sees cap keys at most: its first + seeing * R is group * (len + ITEM_COST * KEYS) + 2 R or less)
    const int64_t most = tiles * p.Hkv * ((int64_t)p.group * (p.cap + ITEM_COST * KEYS) + 2 * R);
    for (p.shift = 0; most >> p.shift >= (int64_t)1 << 30;) ++p.shift;
  }
  // The beginning of the next item that there is, or the end.
  __host__ __device__ __forceinline__ void next_item(ChunkWalk &w) const {
    w.unit = 0;
    if (++w.rt < w.tiles) {
      w.units = units_of(w, w.rt);
      return;
    }
    w.rt = 0;
    if (w.tiles > 0 && ++w.head < p.Hkv) {
      w.units = units_of(w, 0);
      return;
    }
    w.head = 0;
    while (++w.s < p.n) {
      enter(w);
      if (w.tiles == 0) continue;
      w.units = units_of(w, 0);
      return;
    }
  }
  __host__ __device__ __forceinline__ void next(ChunkWalk &w) const {
    if (++w.unit >= w.units) next_item(w);
  }
  // All threads of the CTA: where its run begins and ends (places[2]), by a warp each.  cost, known: [n].  Lists that are wrong leave nothing to do, and the
  // cache's status.
  struct Known {
    int sid, len, start, m;
  };
  __device__ __forceinline__ void plan(int *cost, Known *known, ChunkWalk *places, int threads) const {
    const int tid = threadIdx.x, lane = tid & 31;
    bool bad = false;
    for (int i = tid; i < p.n; i += threads) {
      ChunkWalk w{i};
      const int sid = enter(w);
      bad |= wrong(w);
      cost[i] = upto(w, w.tiles) * p.Hkv;
      known[i] = Known{sid, w.len, w.start, w.m};
    }
    bad = __syncthreads_or(bad);
    if (tid < 64) {
      // the sums, each lane those of its part of the list
      auto scan = [&](int x) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int up = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += up;
        }
        return x;
      };
      const int per = (p.n + 31) / 32, i0 = lane * per;
      int sum = 0;
      for (int i = i0; i < min(i0 + per, p.n); ++i) sum += cost[i];
      const int upto_here = scan(sum), total = bad ? 0 : __shfl_sync(0xffffffffu, upto_here, 31);
      const int run = max(((MIN_RUN * KEYS * p.group) >> p.shift) + 1, p.grid_of.quot(total) + 1);
      int x = (int)min((int64_t)run * (blockIdx.x + (tid >> 5)), (int64_t)total);
      ChunkWalk w{p.n};
      if (x < total) {
        // the last of what begins at or in front of it
        const int part = __popc(__ballot_sync(0xffffffffu, i0 < p.n && upto_here - sum <= x)) - 1;
        x -= __shfl_sync(0xffffffffu, upto_here - sum, part);
        w.s = part * per;
        if (per > 1) {
          const int mine = lane < per && w.s + lane < p.n ? cost[w.s + lane] : 0, to = scan(mine);
          const int k = __popc(__ballot_sync(0xffffffffu, lane < per && w.s + lane < p.n && to - mine <= x)) - 1;
          x -= __shfl_sync(0xffffffffu, to - mine, k);
          w.s += k;
        }
        const Known seq = known[w.s];
        w.row = p.table + (int64_t)seq.sid * p.max_pages;
        w.len = seq.len;
        w.start = seq.start;
        w.m = seq.m;
        w.tiles = (w.m * p.group + R - 1) / R;
        const int each = upto(w, w.tiles);
        w.head = (uint32_t)x / (uint32_t)each;
        x -= w.head * each;
        int n = w.tiles;
        while (n > 1) {                                            // 32 places at a time
          const int step = (n + 31) / 32, i = lane * step;
          const int k = __popc(__ballot_sync(0xffffffffu, i < n && upto(w, w.rt + i) <= x)) - 1;
          w.rt += k * step;
          n = min(step, n - k * step);
        }
        x -= upto(w, w.rt);
        w.units = units_of(w, w.rt);
        const int unit = p.unit_of.quot(x << p.shift) - ITEM_COST;
        w.unit = unit <= p.snap ? 0 : unit;
        if (w.unit > 0 && w.units - unit <= p.snap) next_item(w);
      }
      if (lane == 0) places[tid >> 5] = w;
      if (bad && blockIdx.x == 0 && tid == 0) atomicCAS(p.status, OURO_OK, OURO_EINVAL);
    }
    __syncthreads();
  }
};

}  // namespace paged
