// How the attention kernels of the paged cache share out their work.
//
// An item is a sequence's kv head and a tile of its query rows; TILE keys of an item are a unit, and an item costs its units and ITEM_COST
// more.  The items of a call in order (sequence, head, row tile) are dealt out to G CTAs in runs of equal cost; a run begins within an item unless
// that is within SNAP units of the item's border.  Every CTA works this out for itself from the lengths.
#pragma once

#include <cuda.h>

#include "paged.h"

namespace paged {

// Division of 0 .. 2^31 - 1 by a number that a call does not change: three instructions instead of some thirty, and it is done for every unit.
struct Div {
  uint32_t d, mul, shift;
  void set(uint32_t x) {
    d = x;
    uint32_t bits = 0;
    while (bits < 31 && (1u << bits) < x) ++bits;
    // ceil(2^(31 + bits) / x) < 2^32, and its excess over the quotient is below 2^-31 of it
    mul = x == 1 ? 0 : (uint32_t)((((uint64_t)1 << (31 + bits)) + x - 1) / x);
    shift = bits ? bits - 1 : 0;
  }
  __device__ __forceinline__ int quot(int n) const { return mul ? (int)(__umulhi((uint32_t)n, mul) >> shift) : n; }
};

struct AttnParams {
  const uint8_t *k, *v;                             // of the layer
  const int32_t *table, *lens, *seqs;
  const void *q;
  void *out;
  float *lse;
  int *counters, *status;
  float *pieces;                                    // [CTA][2][rows of a tile][D], then [CTA][2][rows of a tile][2]
  int64_t page_bytes, slot_bytes, head_bytes, q_stride;
  int n, n_new, H, Hkv, group, rows, row_tiles;     // rows = n_new * group
  int n_pages, max_pages, max_seqs, cap, layer;
  Div page, group_of;
  float scale_log2;
  uint32_t wait_limit;                              // polls of a wait (ouro_paged_debug_set_wait_limit)
};

// The pool of a cache's keys or values as (dim, head, row, page, layer), boxes of 64 dims x rows in 128-byte swizzle (paged_attention.cu).
bool make_map(CUtensorMap *m, const ouro_paged_cache *c, const void *base, int box_rows);
// The kernel for many query rows (paged_attention_tc.cu); 0: it does not take the call.
int attention_tc(const ouro_paged_cache *c, const AttnParams &p, cudaStream_t s, int *status);

// A place in the list of units: sequence, head, row tile, unit of the item; and what is known of the sequence.
struct Walk {
  int s, head, rt, tile, tiles, len;
  const int32_t *row;
};

template <int TILE, int ITEM_COST, int SNAP, int MIN_RUN>
struct Runs {
  const AttnParams &p;
  int *s_len, *s_cum;                               // [n] lengths, [n + 1] cost of a head and row tile
  int64_t cost, G, each_run, rest;                  // cost = G * each_run + rest

  // All threads of the CTA; grid: CTAs at most; s_sums: a word for every warp.
  __device__ __forceinline__ Runs(const AttnParams &params, int grid, int *len, int *cum, int *s_sums, int threads) : p(params), s_len(len), s_cum(cum) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, per = (p.n + threads - 1) / threads;
    int sum = 0;
    for (int i = tid * per; i < min(p.n, (tid + 1) * per); ++i) {
      const int sid = p.seqs ? p.seqs[i] : i;
      const bool known = sid >= 0 && sid < p.max_seqs;              // (addresses are valid whether or not the value is wanted)
      const int n = known ? min(max(p.lens[known ? sid : 0], 0), p.cap) : 0;
      s_len[i] = n;
      sum += max(1, (n + TILE - 1) / TILE) + ITEM_COST;
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    if (lane == 31) s_sums[warp] = inc;
    __syncthreads();
    int at = inc - sum;
    for (int w = 0; w < warp; ++w) at += s_sums[w];
    for (int i = tid * per; i < min(p.n, (tid + 1) * per); ++i) {
      s_cum[i] = at;
      at += max(1, (s_len[i] + TILE - 1) / TILE) + ITEM_COST;
    }
    if (tid == threads - 1) s_cum[p.n] = at;
    __syncthreads();
    cost = (int64_t)s_cum[p.n] * (p.Hkv * p.row_tiles);
    G = min((int64_t)grid, max((int64_t)1, cost / MIN_RUN));
    each_run = cost <= INT32_MAX ? (int64_t)((uint32_t)cost / (uint32_t)G) : cost / G;
    rest = cost - each_run * G;
  }
  __device__ __forceinline__ void enter(Walk &w) const {
    w.len = s_len[w.s];
    w.tiles = s_cum[w.s + 1] - s_cum[w.s] - ITEM_COST;
    const int sid = p.seqs ? p.seqs[w.s] : w.s;
    w.row = p.table + (int64_t)(w.len > 0 ? sid : 0) * p.max_pages;
  }
  __device__ __forceinline__ void next(Walk &w) const {
    if (++w.tile < w.tiles) return;
    w.tile = 0;
    if (++w.rt < p.row_tiles) return;
    w.rt = 0;
    if (++w.head < p.Hkv) return;
    w.head = 0;
    if (++w.s < p.n) enter(w);
  }
  // Where the c-th run begins.  A warp looks for the sequence together: one step for 32 sequences, two for all there can be.
  __device__ __forceinline__ Walk place(int64_t c) const {
    const int64_t at = each_run * c + (uint32_t)(rest * c) / (uint32_t)G, F = p.Hkv * p.row_tiles;   // cost * c / G
    Walk w{p.n, 0, 0, 0, 0, 0, nullptr};
    if (at >= cost) return w;
    const int lane = threadIdx.x & 31;
    int lo = 0;
    if (p.n > 32) lo = 32 * (__popc(__ballot_sync(0xffffffffu, 32 * lane < p.n && s_cum[min(32 * lane, p.n)] * F <= at)) - 1);
    if (p.n > 1) lo += __popc(__ballot_sync(0xffffffffu, lo + lane < p.n && s_cum[min(lo + lane, p.n)] * F <= at)) - 1;
    w.s = lo;
    enter(w);
    const int in = (int)(at - s_cum[lo] * F), each = w.tiles + ITEM_COST;   // fits: a sequence's cost is checked on the host
    const int hr = in / each, tile = in - hr * each - ITEM_COST;
    w.head = hr / p.row_tiles;
    w.rt = hr - w.head * p.row_tiles;
    w.tile = tile <= SNAP ? 0 : tile;
    if (w.tile > 0 && w.tiles - tile <= SNAP) {
      w.tile = w.tiles - 1;
      next(w);
    }
    return w;
  }
  // The CTAs that have the beginning and the end of an item that is cut: its cuts are the borders of runs that place() leaves within it.
  __device__ __forceinline__ void owners(const Walk &w, int &c0, int &c1) const {
    const int64_t item0 = (int64_t)s_cum[w.s] * (p.Hkv * p.row_tiles) + (int64_t)(w.head * p.row_tiles + w.rt) * (w.tiles + ITEM_COST) + ITEM_COST;
    const int64_t lo = item0 + SNAP + 1, hi = item0 + w.tiles - SNAP - 1;
    c0 = (int)((lo * G + cost - 1) / cost) - 1;
    c1 = (int)(((hi + 1) * G + cost - 1) / cost) - 1;
  }
};
__device__ __forceinline__ bool same(const Walk &a, const Walk &b) { return a.tile == b.tile && a.rt == b.rt && a.head == b.head && a.s == b.s; }

}  // namespace paged
