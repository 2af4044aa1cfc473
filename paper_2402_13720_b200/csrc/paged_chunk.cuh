// How the attention kernels for chunks of new tokens share out their work.
//
// A sequence has m new tokens, the newest of its len; they and the query heads of a kv head's group are its m * group query rows, token by token.  An
// item is a sequence's kv head and a tile of R rows; KEYS keys of an item are a unit, and an item has as many as its last row sees.  Items in order
// (sequence, head, tile) are dealt out to the CTAs in runs of equal cost; a run begins within an item unless that is within SNAP units of the item's
// border.  Every CTA works this out for itself from the lengths, so that there is no planning call; what is cut leaves pieces (maximum, sum, unnormalised
// output, in 32 bits), and a second kernel adds them up in ascending order: the same call gives the same bits.
// An item's cost is that of its keys, group times their number, and ITEM_COST units for filling and draining the chain.  It grows by R from one tile to
// the next of a sequence, so that the cost of the first k tiles is a polynomial of k and a run's beginning is found without a walk over the tiles: this is the
// first that a CTA does, with cold caches, and every instruction counts (walking took 4900 cycles before the first copy, this 2500).
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
  Div page, group_of, unit_of;                      // unit_of: KEYS * group
  double inv_grid;
  float scale_log2;
  uint32_t wait_limit;
  bool wide_out;                                    // out is a multiple of 32 bytes
};

// The tcgen05 kernel (paged_chunk_tc.cu); cost: the call's at most; 0: does not take the call.  And the join of its pieces (paged_chunk.cu).
int chunk_tc(const ouro_paged_cache *c, const ChunkParams &p, int64_t cost, cudaStream_t s, int *status);
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

  // Whether an item of so many keys has units for a cut.
  static bool may_cut(int keys) { return (keys + KEYS - 1) / KEYS >= 2 * SNAP + 2; }
  __device__ __forceinline__ explicit ChunkRuns(const ChunkParams &params) : p(params) {}
  // What is known of a sequence; no tokens outside the table.
  __device__ __forceinline__ void enter(ChunkWalk &w) const {
    const int sid = p.seqs ? p.seqs[w.s] : w.s;
    const bool known = sid >= 0 && sid < p.max_seqs;
    w.len = known ? min(max(p.lens[sid], 0), p.cap) : 0;
    w.row = p.table + (int64_t)(known ? sid : 0) * p.max_pages;
    w.start = p.starts[w.s];
    w.m = p.starts[w.s + 1] - w.start;
    w.tiles = (w.m * p.group + R - 1) / R;
  }
  __device__ __forceinline__ bool wrong(const ChunkWalk &w) const { return w.start < 0 || w.m < 0 || w.start > p.rows - w.m; }
  // Keys that row r (of the sequence's m * group) sees; below 1: none.
  __device__ __forceinline__ int sees(const ChunkWalk &w, int r) const { return w.len - w.m + 1 + p.group_of.quot(r); }
  __device__ __forceinline__ int units_of(const ChunkWalk &w, int rt) const {
    const int last = min(w.m * p.group - 1, rt * R + R - 1);
    return max(1, (sees(w, last) + KEYS - 1) / KEYS);
  }
  // Cost of the first k tiles of a head.
  __device__ __forceinline__ int64_t upto(const ChunkWalk &w, int k) const {
    return (int64_t)k * (p.group * (max(w.len - w.m, 0) + ITEM_COST * KEYS) + R) + (int64_t)R * k * (k - 1) / 2;
  }
  // The beginning of the next item that there is, or the end.
  __device__ __forceinline__ void next_item(ChunkWalk &w) const {
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
  __device__ __forceinline__ void next(ChunkWalk &w) const {
    if (++w.unit >= w.units) next_item(w);
  }
  // The last k of 0 .. n - 1 with cost(k) <= x, which does not descend; cost(0) <= x.  A warp together.
  template <typename F>
  __device__ __forceinline__ int last_within(int n, int64_t x, const F &cost) const {
    int lo = 0;
    while (n > 1) {
      const int step = (n + 31) / 32, i = (threadIdx.x & 31) * step;
      const int k = __popc(__ballot_sync(0xffffffffu, i < n && cost(lo + min(i, n - 1)) <= x)) - 1;
      lo += k * step;
      n = min(step, n - k * step);
    }
    return lo;
  }
  // All threads of the CTA: where its run begins and ends (places[2]).  cum: [n + 1].  Lists that are wrong leave nothing to do, and the cache's status.
  __device__ __forceinline__ void plan(int64_t *cum, ChunkWalk *places, int threads) const {
    const int tid = threadIdx.x, lane = tid & 31;
    bool bad = false;
    for (int i = tid; i < p.n; i += threads) {
      ChunkWalk w{i};
      enter(w);
      bad |= wrong(w);
      cum[i + 1] = upto(w, w.tiles) * p.Hkv;
    }
    bad = __syncthreads_or(bad);
    if (tid < 32) {
      // the sums, each lane those of its part of the list
      const int per = (p.n + 31) / 32, i0 = min(lane * per, p.n), i1 = min(i0 + per, p.n);
      int64_t sum = 0;
      for (int i = i0; i < i1; ++i) sum += cum[i + 1];
      int64_t at = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t up = __shfl_up_sync(0xffffffffu, at, o);
        if (lane >= o) at += up;
      }
      const int64_t total = bad ? 0 : __shfl_sync(0xffffffffu, at, 31);
      at -= sum;
      if (lane == 0) cum[0] = 0;
      for (int i = i0; i < i1; ++i) cum[i + 1] = at += cum[i + 1];
      __syncwarp();
      const int64_t run = max((int64_t)MIN_RUN * KEYS * p.group, (int64_t)((double)total * p.inv_grid) + 1);
#pragma unroll 1
      for (int e = 0; e < 2; ++e) {
        int64_t x = run * (blockIdx.x + e);
        ChunkWalk w{p.n};
        if (x < total) {
          w.s = last_within(p.n, x, [&](int i) { return cum[i]; });
          enter(w);
          x -= cum[w.s];
          const int64_t each = upto(w, w.tiles);
          w.head = last_within(p.Hkv, x, [&](int i) { return i * each; });
          x -= w.head * each;
          w.rt = last_within(w.tiles, x, [&](int i) { return upto(w, i); });
          x -= upto(w, w.rt);
          w.units = units_of(w, w.rt);
          const int unit = p.unit_of.quot((int)x) - ITEM_COST;
          w.unit = unit <= SNAP ? 0 : unit;
          if (w.unit > 0 && w.units - unit <= SNAP) next_item(w);
        }
        if (lane == 0) places[e] = w;
      }
      if (bad && blockIdx.x == 0 && lane == 0) atomicCAS(p.status, OURO_OK, OURO_EINVAL);
    }
    __syncthreads();
  }
};

}  // namespace paged
