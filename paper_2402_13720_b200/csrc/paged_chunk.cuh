// How the attention kernels for chunks of new tokens share out their work.
//
// A sequence has m new tokens, the newest of its len; they and the query heads of a kv head's group are its m * group query rows, token by token.  An
// item is a sequence's kv head and a tile of R rows; KEYS keys of an item are a unit, and an item has as many as its last row sees.  Items in order
// (sequence, head, tile) are dealt out to G CTAs in runs of equal cost (units, and ITEM_COST for each item); a run begins within an item unless that is
// within SNAP units of the item's border.  Every CTA works this out for itself from the lengths, so that there is no planning call; what is cut leaves
// pieces (maximum, sum, unnormalised output, in 32 bits), and a second kernel adds them up in ascending order: the same call gives the same bits.
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
  Div page, group_of;
  float scale_log2;
  uint32_t wait_limit;
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
  const int *s_cum;                                 // [n + 1] cost of a head of the sequences before
  int cost, G, each_run, rest;                      // cost = G * each_run + rest (below 2^31: the host checks what it may be); G = 0: the lists are wrong

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
  // All threads of the CTA; grid: CTAs at most; scratch: [n + 1] for the costs, which have to last until the last place(), and a word for every warp.
  __device__ __forceinline__ ChunkRuns(const ChunkParams &params, int grid, int *cum, int *s_sums, int threads) : p(params), s_cum(cum) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = threads / 32;
    bool bad = false;
    if (p.n <= warps) {                             // a warp for a sequence, a lane for a tile
      if (warp < p.n) {
        ChunkWalk w{warp};
        enter(w);
        bad = wrong(w);
        int sum = 0;
        if (!bad)
          for (int rt = lane; rt < w.tiles; rt += 32) sum += units_of(w, rt) + ITEM_COST;
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) cum[warp + 1] = sum;
      }
    } else {
      for (int i = tid; i < p.n; i += threads) {
        ChunkWalk w{i};
        enter(w);
        const bool refused = wrong(w);
        bad |= refused;
        int sum = 0;
        if (!refused)
          for (int rt = 0; rt < w.tiles; ++rt) sum += units_of(w, rt) + ITEM_COST;
        cum[i + 1] = sum;
      }
    }
    bad = __syncthreads_or(bad);
    // their sums in order, by the first warp
    if (warp == 0) {
      int at = 0;
      for (int i0 = 0; i0 < p.n; i0 += 32) {
        int x = i0 + lane < p.n ? cum[i0 + lane + 1] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int up = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += up;
        }
        if (i0 + lane < p.n) cum[i0 + lane + 1] = at + x;
        at += __shfl_sync(0xffffffffu, x, 31);
      }
      if (lane == 0) cum[0] = 0;
    }
    __syncthreads();
    cost = cum[p.n] * p.Hkv;
    G = bad || cost == 0 ? 0 : min(grid, max(1, cost / MIN_RUN));
    each_run = G ? (int)((uint32_t)cost / (uint32_t)G) : 0;
    rest = cost - each_run * G;
    if (bad && blockIdx.x == 0 && tid == 0) atomicCAS(p.status, OURO_OK, OURO_EINVAL);
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
  // Where the c-th run begins, c <= G; a warp looks for it together.
  __device__ __forceinline__ ChunkWalk place(int c) const {
    ChunkWalk w{p.n};
    if (G == 0) return w;
    const int at = each_run * c + (int)((uint32_t)(rest * c) / (uint32_t)G);    // cost * c / G
    if (at >= cost) return w;
    const int lane = threadIdx.x & 31;
    // the last sequence that begins at or in front of it and has something (sequences without tokens cost nothing)
    int lo = 0, hi = p.n;                                           // (all before lo begin in front; all from hi on behind)
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, i = lo + lane * step;
      const int k = __popc(__ballot_sync(0xffffffffu, i < hi && s_cum[min(i, p.n)] * p.Hkv <= at));
      const int new_lo = lo + (k - 1) * step;
      hi = min(hi, new_lo + step);
      lo = new_lo;
    }
    w.s = lo;
    enter(w);
    const int each = s_cum[lo + 1] - s_cum[lo];
    int in = at - s_cum[lo] * p.Hkv;
    w.head = in / each;
    in -= w.head * each;
    for (int t0 = 0; t0 < w.tiles; t0 += 32) {
      const int mine = t0 + lane < w.tiles ? units_of(w, t0 + lane) + ITEM_COST : 0;
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += up;
      }
      const uint32_t behind = __ballot_sync(0xffffffffu, in < upto);
      if (behind) {
        const int k = __ffs(behind) - 1;
        w.rt = t0 + k;
        w.units = __shfl_sync(0xffffffffu, mine, k) - ITEM_COST;
        in -= __shfl_sync(0xffffffffu, upto - mine, k);
        break;
      }
      in -= __shfl_sync(0xffffffffu, upto, 31);
    }
    const int unit = in - ITEM_COST;
    w.unit = unit <= SNAP ? 0 : unit;
    if (w.unit > 0 && w.units - unit <= SNAP) next_item(w);
    return w;
  }
};

}  // namespace paged
