// Pages of a cache that several continuations share: forking, extending (with copies of shared unfinished pages), truncating, compacting;
// and the step that rotates new queries and keys and writes keys and values to their pages.
//
// The table, the lengths and the counts are the whole state (no list of free pages besides): a page is free when its count is 0, and pages
// are given out lowest id first, so that the same calls give the same state.  Counts are only ever changed by integer additions.
//  - fork and truncate are one kernel, one cluster: entries to come are read before any is written, with the cluster's barrier between.
//  - extend and compact plan in one CTA (who needs how many pages, the lowest free ones by ballots and a scan over the counts) and leave
//    a list of pages to copy; a second kernel over all SMs copies, bound by HBM, and does what is left (slots; new ids in the table).
// A call whose lists are wrong changes nothing but the status.
#include "paged.h"
#include "row_ops.cuh"

namespace {

constexpr int MAX_LIST = OURO_MAX_LIST;
constexpr int PLAN_THREADS = 1024;
constexpr int ROUND = 16;                          // counts a thread looks at in one round of a scan

struct CacheDev {
  int32_t *table, *lens, *refs, *status;
  int n_pages, page, max_seqs, max_pages, cap;
};
CacheDev dev_of(const ouro_paged_cache *c) {
  return {c->table, c->lens, c->refs, c->status, c->n_pages, c->page_size, c->max_seqs, c->max_pages, c->max_pages * c->page_size};
}
__device__ __forceinline__ int pages_of(int len, int page) { return len / page + (len % page != 0); }
__device__ __forceinline__ bool page_ok(const CacheDev &c, int id) { return id >= 0 && id < c.n_pages; }
__device__ __forceinline__ int len_of(const CacheDev &c, int seq) { return min(max(c.lens[seq], 0), c.cap); }

// Lists of the planning kernels in the workspace.
struct Lists {
  int *head;                                       // [0] pages to copy, [1] the call was refused, [2] pages in use
  int *src, *dst;                                  // pages to copy and where to
  int *aux;                                        // extend: rows of each copy; compact: new ids [n_pages]
  int *free;                                       // extend: the pages given out
};
Lists lists_of(const ouro_paged_cache *c, const paged::Layout &l) {
  int *at = (int *)((char *)c->workspace + l.lists);
  const int n = c->n_pages > MAX_LIST ? c->n_pages : MAX_LIST;
  return {at, at + 64, at + 64 + n, at + 64 + 2 * n, at + 64 + 3 * n};
}

__global__ void __launch_bounds__(256) reset_kernel(CacheDev c, int *counters) {
  pdl_wait();
  pdl_trigger();
  const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = at; i < (int64_t)c.max_seqs * c.max_pages; i += step) c.table[i] = -1;
  for (int64_t i = at; i < c.max_seqs; i += step) c.lens[i] = 0;
  for (int64_t i = at; i < c.n_pages; i += step) c.refs[i] = 0;
  for (int64_t i = at; i < paged::MAX_CTAS; i += step) counters[i] = 0;
  if (at == 0) *c.status = OURO_OK;
}

// ---------------------------------------------------------------------------- fork, truncate
constexpr int RETABLE_THREADS = 512;
constexpr int BLOCK_COLS = 128;                    // entries a warp takes at a time, four a lane
constexpr int SAME = -2;                           // staged: the entry stays

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Row dst[i] becomes the first keep[i] tokens (NULL: all) of what row src[i] was.
__global__ void __launch_bounds__(RETABLE_THREADS) retable_kernel(CacheDev c, const int32_t *src, const int32_t *dst, const int32_t *keep, int n,
                                                                  int *staged) {
  __shared__ int s_src[MAX_LIST], s_dst[MAX_LIST], s_new[MAX_LIST], s_old[MAX_LIST];
  __shared__ uint32_t s_seen[OURO_MAX_SEQS / 32];
  __shared__ int s_cols, s_bad;
  const int tid = threadIdx.x, lane = tid & 31;
  if (tid == 0) s_cols = 0, s_bad = 0;
  for (int i = tid; i < (c.max_seqs + 31) / 32; i += RETABLE_THREADS) s_seen[i] = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();
  int cols = 0;
  for (int i = tid; i < n; i += RETABLE_THREADS) {
    const int a = src[i], b = dst[i], k = keep ? keep[i] : INT32_MAX;
    bool bad = a < 0 || a >= c.max_seqs || b < 0 || b >= c.max_seqs || k < 0;
    if (!bad) {
      bad = atomicOr(&s_seen[b >> 5], 1u << (b & 31)) >> (b & 31) & 1;
      s_src[i] = a;
      s_dst[i] = b;
      s_new[i] = min(len_of(c, a), k);
      s_old[i] = pages_of(len_of(c, b), c.page);
      cols = max(cols, max(s_old[i], pages_of(s_new[i], c.page)));
    }
    if (bad) s_bad = 1;
  }
  if (cols) atomicMax(&s_cols, cols);
  __syncthreads();
  if (s_bad) {                                     // (every CTA of the cluster sees the same lists)
    if (blockIdx.x == 0 && tid == 0) atomicCAS(c.status, OURO_OK, OURO_EINVAL);
    return;
  }
  const int blocks = (s_cols + BLOCK_COLS - 1) / BLOCK_COLS;
  const int w0 = blockIdx.x * (RETABLE_THREADS / 32) + (tid >> 5), W = gridDim.x * (RETABLE_THREADS / 32);
  for (int it = w0; it < n * blocks; it += W) {
    const int i = it / blocks, col0 = (it - i * blocks) * BLOCK_COLS + lane;
    const int pn = pages_of(s_new[i], c.page), po = s_old[i];
    const int32_t *from = c.table + (int64_t)s_src[i] * c.max_pages, *to = c.table + (int64_t)s_dst[i] * c.max_pages;
    int was[4], is[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = col0 + 32 * j;
      was[j] = col < po ? to[col] : -1;
      is[j] = col < pn ? from[col] : -1;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = col0 + 32 * j;
      if (col >= max(pn, po)) continue;
      if (was[j] != is[j]) {
        if (page_ok(c, was[j])) atomicSub(c.refs + was[j], 1);
        if (page_ok(c, is[j])) atomicAdd(c.refs + is[j], 1);
      }
      staged[(int64_t)i * c.max_pages + col] = was[j] == is[j] ? SAME : is[j];
    }
  }
  cluster_barrier();                               // everything has been read
  for (int it = w0; it < n * blocks; it += W) {    // (a thread finds what it staged itself)
    const int i = it / blocks, col0 = (it - i * blocks) * BLOCK_COLS + lane;
    const int top = max(pages_of(s_new[i], c.page), s_old[i]);
    int32_t *to = c.table + (int64_t)s_dst[i] * c.max_pages;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = col0 + 32 * j;
      if (col >= top) continue;
      const int id = staged[(int64_t)i * c.max_pages + col];
      if (id != SAME) to[col] = id;
    }
  }
  if (blockIdx.x == 0)
    for (int i = tid; i < n; i += RETABLE_THREADS) c.lens[s_dst[i]] = s_new[i];
}

// ---------------------------------------------------------------------------- planning
// (What an extend asks for may be more than 31 bits hold; more than there are pages is refused, so it may stop there.)
__device__ __forceinline__ int add_up(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)INT32_MAX); }
// Sum of numbers not below 0 over the CTA's threads in front of this one; total: of all, at most INT32_MAX, and then the sums mean nothing.
__device__ __forceinline__ int scan(int v, int *s_sums, int *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc = add_up(inc, up);
  }
  __syncthreads();                                 // (the sums of an earlier call have been read)
  if (lane == 31) s_sums[warp] = inc;
  __syncthreads();
  int w = lane < PLAN_THREADS / 32 ? s_sums[lane] : 0;
  const int mine = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w = add_up(w, up);
  }
  *total = __shfl_sync(0xffffffffu, w, 31);
  return (int)((uint32_t)(inc - v) + (uint32_t)__shfl_sync(0xffffffffu, w - mine, warp));
}

// One round over the counts of ids base .. base + ROUND * PLAN_THREADS - 1: for every chosen one, in ascending order, put(rank, id).
// choose(id, count) -> 0: no, 1: of the first kind, 2: of the second; ranks are counted per kind from *first, *second, which move on.
template <typename Choose, typename Put>
__device__ __forceinline__ void round_of(const CacheDev &c, int base, int *s_counts, int *s_sums, int *first, int *second, Choose choose, Put put) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int kind[ROUND];
#pragma unroll
  for (int j = 0; j < ROUND; ++j) {
    const int id = base + j * PLAN_THREADS + tid;
    kind[j] = c.refs[min(id, c.n_pages - 1)];
  }
#pragma unroll
  for (int j = 0; j < ROUND; ++j) {
    const int id = base + j * PLAN_THREADS + tid;
    kind[j] = id < c.n_pages ? choose(id, kind[j]) : 0;
    const uint32_t a = __ballot_sync(0xffffffffu, kind[j] == 1), b = __ballot_sync(0xffffffffu, kind[j] == 2);
    if (lane == 0) s_counts[j * (PLAN_THREADS / 32) + warp] = __popc(a) | __popc(b) << 16;
  }
  __syncthreads();
  // at most ROUND * PLAN_THREADS of either kind: the two halves of a word do not meet
  static_assert(ROUND * PLAN_THREADS < 65536 && ROUND * PLAN_THREADS / 32 <= PLAN_THREADS, "");
  int total;
  const int mine = tid < ROUND * PLAN_THREADS / 32 ? s_counts[tid] : 0;
  const int before = scan(mine, s_sums, &total);
  __syncthreads();
  if (tid < ROUND * PLAN_THREADS / 32) s_counts[tid] = before;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < ROUND; ++j) {
    const uint32_t a = __ballot_sync(0xffffffffu, kind[j] == 1), b = __ballot_sync(0xffffffffu, kind[j] == 2);
    const int at = s_counts[j * (PLAN_THREADS / 32) + warp], id = base + j * PLAN_THREADS + tid;
    const uint32_t below = (1u << lane) - 1;
    if (kind[j] == 1) put(1, *first + (at & 0xffff) + __popc(a & below), id);
    if (kind[j] == 2) put(2, *second + (at >> 16) + __popc(b & below), id);
  }
  *first += total & 0xffff;
  *second += total >> 16;
  __syncthreads();
}

__global__ void __launch_bounds__(PLAN_THREADS) extend_plan_kernel(CacheDev c, const int32_t *seqs, const int32_t *add, int n, int width, Lists out) {
  __shared__ int s_seq[MAX_LIST], s_len[MAX_LIST], s_from[MAX_LIST + 1], s_last[MAX_LIST];
  __shared__ union { uint32_t seen[OURO_MAX_SEQS / 32]; struct { int key[2 * MAX_LIST], count[2 * MAX_LIST], latest[2 * MAX_LIST]; } share; } u;
  __shared__ int s_counts[ROUND * PLAN_THREADS / 32], s_sums[32], s_bad, s_copies;
  const int tid = threadIdx.x;
  if (tid == 0) s_bad = INT32_MAX, s_copies = 0;
  for (int i = tid; i < (c.max_seqs + 31) / 32; i += PLAN_THREADS) u.seen[i] = 0;
  pdl_wait();
  pdl_trigger();
  __syncthreads();

  // ---- the list, one sequence a thread
  int seq = -1, more = 0, len = 0;
  if (tid < n) {
    seq = seqs[tid];
    more = add[tid];
    int bad = OURO_OK;
    if (seq < 0 || seq >= c.max_seqs || more < 0 || more > width || (atomicOr(&u.seen[seq >> 5], 1u << (seq & 31)) >> (seq & 31) & 1)) {
      bad = OURO_EINVAL;
    } else {
      len = len_of(c, seq);
      if (more > c.cap - len) bad = OURO_ECAPACITY;
    }
    if (bad) atomicMin(&s_bad, bad);
  }
  __syncthreads();
  const int listed = s_bad;
  for (int i = tid; i < 2 * MAX_LIST; i += PLAN_THREADS) u.share.key[i] = -1, u.share.count[i] = 0, u.share.latest[i] = -1;
  __syncthreads();
  if (listed != INT32_MAX) {
    if (tid == 0) {
      atomicCAS(c.status, OURO_OK, listed);
      out.head[0] = 0;
      out.head[1] = 1;
    }
    return;
  }

  // ---- who needs a page of its own for an unfinished one: all that share it but, if all who do are here, the last
  int last = -1, refs = 0, place = 0;
  if (tid < n && more > 0 && len % c.page) {
    last = c.table[(int64_t)seq * c.max_pages + len / c.page];
    if (page_ok(c, last)) refs = c.refs[last];
  }
  if (refs > 1) {
    place = (uint32_t)last * 2654435761u >> 21;    // (2 * MAX_LIST places for at most MAX_LIST pages)
    for (;;) {
      const int was = atomicCAS(&u.share.key[place], -1, last);
      if (was == -1 || was == last) break;
      place = (place + 1) & (2 * MAX_LIST - 1);
    }
    atomicAdd(&u.share.count[place], 1);
    atomicMax(&u.share.latest[place], tid);
  }
  __syncthreads();
  const int copy = refs > 1 && !(u.share.count[place] == refs && u.share.latest[place] == tid);
  const int need = tid < n ? pages_of(len + more, c.page) - pages_of(len, c.page) + copy : 0;
  int total;
  const int from = scan(need, s_sums, &total);
  if (tid < n) {
    s_seq[tid] = seq;
    s_len[tid] = len;
    s_from[tid] = from;
    s_last[tid] = copy ? last : -1;
  }
  if (tid == 0) s_from[n] = total;

  // ---- the lowest free pages, one for every rank below total
  int found = 0, none = 0;
  for (int base = 0; base < c.n_pages && found < total; base += ROUND * PLAN_THREADS)
    round_of(c, base, s_counts, s_sums, &found, &none, [](int, int count) { return count == 0 ? 1 : 0; },
             [&](int, int rank, int id) { if (rank < total) out.free[rank] = id; });
  if (found < total) {
    if (tid == 0) {
      atomicCAS(c.status, OURO_OK, OURO_ECAPACITY);
      out.head[0] = 0;
      out.head[1] = 1;
    }
    return;
  }
  __syncthreads();                                 // (out.free, s_from)

  // ---- to the sequences
  for (int k = tid; k < total; k += PLAN_THREADS) {
    const int id = out.free[k];
    int lo = 0, hi = n - 1;                        // the last sequence that begins at or before k: the one that needs it
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (s_from[mid] <= k) lo = mid; else hi = mid - 1;
    }
    const int own = s_last[lo] >= 0, j = k - s_from[lo], l0 = s_len[lo];
    const int col = own && j == 0 ? l0 / c.page : pages_of(l0, c.page) + j - own;
    c.table[(int64_t)s_seq[lo] * c.max_pages + col] = id;
    c.refs[id] = 1;
    if (own && j == 0) {
      atomicSub(c.refs + s_last[lo], 1);
      const int at = atomicAdd(&s_copies, 1);
      out.src[at] = s_last[lo];
      out.dst[at] = id;
      out.aux[at] = l0 % c.page;
    }
  }
  if (tid < n) c.lens[seq] = len + more;
  __syncthreads();
  if (tid == 0) {
    out.head[0] = s_copies;
    out.head[1] = 0;
  }
}

__global__ void __launch_bounds__(PLAN_THREADS) compact_plan_kernel(CacheDev c, Lists out, int32_t *live_out) {
  __shared__ int s_counts[ROUND * PLAN_THREADS / 32], s_sums[32];
  const int tid = threadIdx.x;
  pdl_wait();
  pdl_trigger();
  int live = 0;
  for (int i = tid; i < c.n_pages; i += PLAN_THREADS) live += c.refs[i] > 0;
  int total;
  scan(live, s_sums, &total);
  int holes = 0, moves = 0;
  for (int base = 0; base < c.n_pages; base += ROUND * PLAN_THREADS)
    round_of(c, base, s_counts, s_sums, &holes, &moves, [&](int id, int count) { return count > 0 ? (id >= total ? 2 : 0) : (id < total ? 1 : 0); },
             [&](int kind, int rank, int id) { (kind == 1 ? out.dst : out.src)[rank] = id; });
  __syncthreads();
  for (int i = tid; i < moves; i += PLAN_THREADS) {
    const int a = out.src[i], b = out.dst[i];
    c.refs[b] = c.refs[a];
    c.refs[a] = 0;
    out.aux[a] = b;
  }
  if (tid == 0) {
    out.head[0] = moves;
    out.head[1] = 0;
    out.head[2] = total;
    if (live_out) *live_out = total;
  }
}

// ---------------------------------------------------------------------------- copying
struct CopyParams {
  uint8_t *k, *v;
  int64_t layer_bytes, page_bytes, slot_bytes, head_bytes;
  int layers, Hkv, row_pieces;                     // 16-byte pieces of one head's row
  Lists lists;
  // extend
  const int32_t *seqs, *add;
  int n, width;
  int32_t *slots, *positions;
};
constexpr int COPY_THREADS = 256, UNROLL = 8;
constexpr int CHUNK = 32 * UNROLL;                 // 16-byte pieces a warp takes at a time: 4 KB (beam step of 12 sequences 12.9 us, 16 KB: 13.4)
// CTAs of an SM, 4 at a time: who is done early takes another, so that the last bytes are not left to a few.  us with 4, 16, 32, 64: 70 pages of
// 32 layers (587 MB) 211, 201, 200, 199, 20 pages 73, 69, 69, 71, none 11.0, 12.5, 15.0, 19.9; extending 64 sequences of the 70B shape 59, 55, 55, 56.
constexpr int COPY_CTAS = 16;

// WHOLE: heads and rows of a page lie side by side (its rows are one piece of memory); COMPACT: whole pages, and the table follows.
template <bool WHOLE, bool COMPACT>
__global__ void __launch_bounds__(COPY_THREADS) copy_kernel(const CacheDev c, const CopyParams p) {
  pdl_wait();
  pdl_trigger();
  const int moves = p.lists.head[0];
  const int64_t at = (int64_t)blockIdx.x * COPY_THREADS + threadIdx.x, step = (int64_t)gridDim.x * COPY_THREADS;
  if constexpr (COMPACT) {
    if (moves == 0) return;
    const int live = p.lists.head[2], blocks = (c.max_pages + COPY_THREADS - 1) / COPY_THREADS;
    for (int64_t it = blockIdx.x; it < (int64_t)c.max_seqs * blocks; it += gridDim.x) {
      const int seq = (int)(it / blocks), col = (int)(it - (int64_t)seq * blocks) * COPY_THREADS + threadIdx.x;
      if (col >= pages_of(len_of(c, seq), c.page)) continue;
      int32_t *e = c.table + (int64_t)seq * c.max_pages + col;
      const int id = *e;
      if (id >= live && id < c.n_pages) *e = p.lists.aux[id];
    }
  } else {
    const bool refused = p.lists.head[1];
    if (p.slots || p.positions)
      for (int64_t e = at; e < (int64_t)p.n * p.width; e += step) {
        const int i = (int)(e / p.width), j = (int)(e - (int64_t)i * p.width);
        int slot = -1, pos = -1;
        if (!refused && j < p.add[i]) {
          const int seq = p.seqs[i];
          pos = c.lens[seq] - p.add[i] + j;
          const int pg = pos / c.page, id = c.table[(int64_t)seq * c.max_pages + pg];
          slot = id < 0 ? -1 : id * c.page + (pos - pg * c.page);
        }
        if (p.slots) p.slots[e] = slot;
        if (p.positions) p.positions[e] = pos;
      }
  }
  const int per_row = p.Hkv * p.row_pieces;
  const int chunks = (c.page * per_row + CHUNK - 1) / CHUNK, lane = threadIdx.x & 31;
  const int64_t tasks = (int64_t)moves * p.layers * 2 * chunks;
  for (int64_t t = at >> 5; t < tasks; t += step >> 5) {
    int64_t rem = t / chunks;
    const int chunk = (int)(t - rem * chunks);
    const int lk = (int)(rem % (2 * p.layers)), mv = (int)(rem / (2 * p.layers));
    const int src = p.lists.src[mv], dst = p.lists.dst[mv];
    const int pieces = (COMPACT ? c.page : p.lists.aux[mv]) * per_row;
    if (chunk * CHUNK >= pieces) continue;
    uint8_t *base = (lk & 1 ? p.v : p.k) + (int64_t)(lk >> 1) * p.layer_bytes;
    const uint8_t *from = base + (int64_t)src * p.page_bytes;
    uint8_t *to = base + (int64_t)dst * p.page_bytes;
    const int e0 = chunk * CHUNK + lane;
    uint4 x[UNROLL];
    int64_t off[UNROLL];
#pragma unroll
    for (int j = 0; j < UNROLL; ++j) {
      const int e = min(e0 + j * 32, pieces - 1);                  // (always a valid address; stored only where it is meant)
      if (WHOLE) {
        off[j] = (int64_t)e * 16;
      } else {
        const int row = e / per_row, in = e - row * per_row, head = in / p.row_pieces;
        off[j] = row * p.slot_bytes + head * p.head_bytes + (int64_t)(in - head * p.row_pieces) * 16;
      }
      x[j] = __ldcs((const uint4 *)(from + off[j]));
    }
#pragma unroll
    for (int j = 0; j < UNROLL; ++j)
      if (e0 + j * 32 < pieces) __stcs((uint4 *)(to + off[j]), x[j]);
  }
}

int launch_copy(const char *call, const ouro_paged_cache *c, CopyParams p, bool compact, int64_t most_tasks, cudaStream_t s) {
  int dev = 0, sms = 0;
  if (!paged::device(&dev, &sms)) return paged::refuse(call, "no usable current device", OURO_ECUDA);
  const int e = c->dtype == OURO_F32 ? 4 : 2;
  p.k = (uint8_t *)c->k;
  p.v = (uint8_t *)c->v;
  p.layer_bytes = c->layer_stride * e; p.page_bytes = c->page_stride * e; p.slot_bytes = c->slot_stride * e; p.head_bytes = c->head_stride * e;
  p.layers = c->n_layers; p.Hkv = c->n_kv_heads; p.row_pieces = c->head_dim * e / 16;
  const bool whole = c->head_stride == c->head_dim && c->slot_stride == (int64_t)c->n_kv_heads * c->head_dim;
  const int64_t ctas = (most_tasks + COPY_THREADS / 32 - 1) / (COPY_THREADS / 32);
  const dim3 grid((unsigned)(ctas < 1 ? 1 : ctas < COPY_CTAS * sms ? ctas : COPY_CTAS * sms));
  cudaError_t r;
  if (compact) r = launch_pdl(whole ? copy_kernel<true, true> : copy_kernel<false, true>, grid, dim3(COPY_THREADS), 0, s, dev_of(c), p);
  else r = launch_pdl(whole ? copy_kernel<true, false> : copy_kernel<false, false>, grid, dim3(COPY_THREADS), 0, s, dev_of(c), p);
  OURO_COUNT_LAUNCH();
  return r == cudaSuccess ? OURO_OK : paged::refuse(call, cudaGetErrorString(r), OURO_ECUDA);
}

// ---------------------------------------------------------------------------- rotary positions and append
struct AppendParams {
  uint8_t *k, *v;                                  // of the layer
  const void *q, *k_new, *v_new;
  void *q_out;
  const int32_t *slots, *positions;
  const float *cos_t, *sin_t;
  int64_t page_bytes, slot_bytes, head_bytes, q_stride, kv_stride;
  int rows, H, Hkv, D, page, n_pages, n_positions;
};
constexpr int APPEND_THREADS = 256;

__device__ __forceinline__ void load(const float *p, float *x) { const float4 t = *(const float4 *)p; x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w; }
__device__ __forceinline__ void load(const __nv_bfloat16 *p, float *x) {
  const uint4 t = *(const uint4 *)p;
  const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 f = rowops::unpack(w[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
}
__device__ __forceinline__ void store(float *p, const float *x) { *(float4 *)p = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store(__nv_bfloat16 *p, const float *x) {
  *(uint4 *)p = make_uint4(rowops::pack(x[0], x[1]), rowops::pack(x[2], x[3]), rowops::pack(x[4], x[5]), rowops::pack(x[6], x[7]));
}

// A CTA has a row; a thread 16 bytes of a head's first half and the same of its second, with their angles, in every so manieth head: the
// queries first, then the keys, then the values (which are only moved).
template <typename T>
__global__ void __launch_bounds__(APPEND_THREADS) append_kernel(const AppendParams p) {
  constexpr int VEC = 16 / sizeof(T);
  const int half = p.D / 2, chunks = half / VEC, par = APPEND_THREADS / chunks;   // heads at a time
  const int ch = threadIdx.x % chunks, h0 = threadIdx.x / chunks, row = blockIdx.x;
  pdl_wait();
  pdl_trigger();
  if (h0 >= par) return;
  const int pos = p.positions[row], slot = p.slots[row];
  const bool known = pos >= 0 && pos < p.n_positions;
  const int pg = slot / p.page;
  const bool there = known && slot >= 0 && pg < p.n_pages;
  float c[VEC], s[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) c[i] = s[i] = 0.f;
  if (known) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      load(p.cos_t + (int64_t)pos * half + ch * VEC + i, c + i);
      load(p.sin_t + (int64_t)pos * half + ch * VEC + i, s + i);
    }
  }
  const int64_t at = there ? (int64_t)pg * p.page_bytes + (int64_t)(slot - pg * p.page) * p.slot_bytes : 0;
  for (int h = h0; h < p.H + 2 * p.Hkv; h += par) {
    const int kv = h - p.H, vh = kv - p.Hkv;
    const T *src;
    T *dst;
    if (kv < 0) {
      src = (const T *)p.q + row * p.q_stride + (int64_t)h * p.D;
      dst = (T *)p.q_out + ((int64_t)row * p.H + h) * p.D;
    } else {
      if (!there) break;                           // (only keys and values follow)
      src = (const T *)(vh < 0 ? p.k_new : p.v_new) + row * p.kv_stride + (int64_t)(vh < 0 ? kv : vh) * p.D;
      dst = (T *)((vh < 0 ? p.k : p.v) + at + (int64_t)(vh < 0 ? kv : vh) * p.head_bytes);
    }
    src += ch * VEC;
    dst += ch * VEC;
    if (vh >= 0) {
      const uint4 a = *(const uint4 *)src, b = *(const uint4 *)(src + half);
      *(uint4 *)dst = a;
      *(uint4 *)(dst + half) = b;
      continue;
    }
    float a[VEC], b[VEC], x[VEC], y[VEC];
    load(src, a);
    load(src + half, b);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      x[i] = known ? rowops::rotate(a[i], b[i], c[i], -s[i]) : 0.f;
      y[i] = known ? rowops::rotate(b[i], a[i], c[i], s[i]) : 0.f;
    }
    store(dst, x);
    store(dst + half, y);
  }
}

int wrong_list(const char *call, const ouro_paged_cache *c, const int32_t *a, const int32_t *b, int n) {
  if (const char *w = paged::wrong(c)) return paged::refuse(call, w);
  if (n < 0 || n > MAX_LIST) return paged::refuse(call, "n is below 0 or above OURO_MAX_LIST");
  if (n > 0 && (!a || !b)) return paged::refuse(call, "a list is NULL");
  if (!paged::words(a, b)) return paged::refuse(call, "a list is not 4-byte aligned");
  return OURO_OK;
}

int retable(const char *call, const ouro_paged_cache *c, const int32_t *src, const int32_t *dst, const int32_t *keep, int n, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  // One CTA where it has no more than four rounds of entries, else a cluster of eight.
  const int64_t rounds = ((int64_t)n * ((c->max_pages + BLOCK_COLS - 1) / BLOCK_COLS) + RETABLE_THREADS / 32 - 1) / (RETABLE_THREADS / 32);
  const unsigned ctas = rounds <= 4 ? 1 : 8;
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(RETABLE_THREADS);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = ctas;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, retable_kernel, dev_of(c), src, dst, keep, n, (int *)((char *)c->workspace + paged::layout(*c).staged));
  OURO_COUNT_LAUNCH();
  return e == cudaSuccess ? OURO_OK : paged::refuse(call, cudaGetErrorString(e), OURO_ECUDA);
}

}  // namespace

extern "C" size_t ouro_paged_workspace_bytes(const ouro_paged_cache *c) {
  if (const char *w = paged::wrong_shape(c)) return paged::refuse("ouro_paged_workspace_bytes", w), 0;
  return paged::layout(*c).bytes;
}

extern "C" int ouro_paged_reset(const ouro_paged_cache *c, void *stream) {
  const char *call = "ouro_paged_reset";
  if (const char *w = paged::wrong(c)) return paged::refuse(call, w);
  const cudaError_t e = launch_pdl(reset_kernel, dim3(128), dim3(256), 0, (cudaStream_t)stream, dev_of(c), (int *)((char *)c->workspace + paged::layout(*c).counters));
  OURO_COUNT_LAUNCH();
  return e == cudaSuccess ? OURO_OK : paged::refuse(call, cudaGetErrorString(e), OURO_ECUDA);
}

extern "C" int ouro_paged_status(const ouro_paged_cache *c, void *stream) {
  const char *call = "ouro_paged_status";
  if (const char *w = paged::wrong(c)) return paged::refuse(call, w);
  int32_t status = OURO_OK;
  cudaError_t e = cudaMemcpyAsync(&status, c->status, sizeof(status), cudaMemcpyDeviceToHost, (cudaStream_t)stream);
  if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
  if (e == cudaSuccess && status != OURO_OK) e = cudaMemsetAsync(c->status, 0, sizeof(status), (cudaStream_t)stream);
  if (e != cudaSuccess) return paged::refuse(call, cudaGetErrorString(e), OURO_ECUDA);
  if (status == OURO_EINVAL) return paged::refuse(call, "a list named a sequence outside the table or twice, or a negative or too large count");
  if (status == OURO_ECAPACITY) return paged::refuse(call, "no room in a row of the table, or too few free pages", OURO_ECAPACITY);
  if (status == OURO_ETIMEOUT) return paged::refuse(call, "a bounded device-side wait of an attention gave up", OURO_ETIMEOUT);
  return status;
}

extern "C" int ouro_paged_fork(const ouro_paged_cache *c, const int32_t *src, const int32_t *dst, int32_t n, void *stream) {
  const char *call = "ouro_paged_fork";
  const int rc = wrong_list(call, c, src, dst, n);
  return rc != OURO_OK || n == 0 ? rc : retable(call, c, src, dst, nullptr, n, (cudaStream_t)stream);
}

extern "C" int ouro_paged_truncate(const ouro_paged_cache *c, const int32_t *seqs, const int32_t *keep, int32_t n, void *stream) {
  const char *call = "ouro_paged_truncate";
  const int rc = wrong_list(call, c, seqs, keep, n);
  return rc != OURO_OK || n == 0 ? rc : retable(call, c, seqs, seqs, keep, n, (cudaStream_t)stream);
}

extern "C" int ouro_paged_extend(const ouro_paged_cache *c, const int32_t *seqs, const int32_t *add, int32_t n, int32_t width, int32_t *slots,
                                 int32_t *positions, void *stream) {
  const char *call = "ouro_paged_extend";
  const int rc = wrong_list(call, c, seqs, add, n);
  if (rc != OURO_OK || n == 0) return rc;
  if (width < 0) return paged::refuse(call, "width is below 0");
  if (!paged::words(slots, positions)) return paged::refuse(call, "slots or positions are not 4-byte aligned");
  const paged::Layout l = paged::layout(*c);
  const cudaError_t e = launch_pdl(extend_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, (cudaStream_t)stream, dev_of(c), seqs, add, n, width, lists_of(c, l));
  OURO_COUNT_LAUNCH();
  if (e != cudaSuccess) return paged::refuse(call, cudaGetErrorString(e), OURO_ECUDA);
  CopyParams p{};
  p.lists = lists_of(c, l);
  p.seqs = seqs; p.add = add; p.n = n; p.width = width; p.slots = slots; p.positions = positions;
  const int64_t pieces = (int64_t)c->page_size * c->n_kv_heads * c->head_dim * (c->dtype == OURO_F32 ? 4 : 2) / 16;
  return launch_copy(call, c, p, false, (int64_t)n * c->n_layers * 2 * ((pieces + CHUNK - 1) / CHUNK), (cudaStream_t)stream);
}

extern "C" int ouro_paged_compact(const ouro_paged_cache *c, int32_t *live, void *stream) {
  const char *call = "ouro_paged_compact";
  if (const char *w = paged::wrong(c)) return paged::refuse(call, w);
  if (!paged::words(live)) return paged::refuse(call, "live is not 4-byte aligned");
  const paged::Layout l = paged::layout(*c);
  const cudaError_t e = launch_pdl(compact_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, (cudaStream_t)stream, dev_of(c), lists_of(c, l), live);
  OURO_COUNT_LAUNCH();
  if (e != cudaSuccess) return paged::refuse(call, cudaGetErrorString(e), OURO_ECUDA);
  CopyParams p{};
  p.lists = lists_of(c, l);
  return launch_copy(call, c, p, true, INT32_MAX, (cudaStream_t)stream);
}

extern "C" int ouro_paged_append(const ouro_paged_cache *c, int32_t layer, const void *q, int64_t q_stride, const void *k, const void *v, int64_t kv_stride,
                                 int32_t rows, int32_t n_heads, const int32_t *slots, const int32_t *positions, const float *cos_t, const float *sin_t,
                                 int32_t n_positions, void *q_out, void *stream) {
  const char *call = "ouro_paged_append";
  if (const char *w = paged::wrong(c)) return paged::refuse(call, w);
  if (layer < 0 || layer >= c->n_layers) return paged::refuse(call, "no such layer");
  if (rows < 0 || n_heads < 1 || n_positions < 1) return paged::refuse(call, "rows is below 0, or n_heads or n_positions below 1");
  if (rows == 0) return OURO_OK;
  if (!q || !k || !v || !slots || !positions || !cos_t || !sin_t || !q_out) return paged::refuse(call, "a pointer is NULL");
  if (!paged::words(slots, positions)) return paged::refuse(call, "slots or positions are not 4-byte aligned");
  const int e = c->dtype == OURO_F32 ? 4 : 2;
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out | (uintptr_t)cos_t | (uintptr_t)sin_t) % 16 || q_stride * e % 16 || kv_stride * e % 16)
    return paged::refuse(call, "an array or a stride is not a multiple of 16 bytes");
  if (q_stride < (int64_t)n_heads * c->head_dim || kv_stride < (int64_t)c->n_kv_heads * c->head_dim) return paged::refuse(call, "a stride is below a row's length");
  if (q == q_out && q_stride != (int64_t)n_heads * c->head_dim) return paged::refuse(call, "q_out is q, whose rows do not lie side by side");
  AppendParams p{};
  p.k = (uint8_t *)c->k + (int64_t)layer * c->layer_stride * e;
  p.v = (uint8_t *)c->v + (int64_t)layer * c->layer_stride * e;
  p.q = q; p.k_new = k; p.v_new = v; p.q_out = q_out;
  p.slots = slots; p.positions = positions; p.cos_t = cos_t; p.sin_t = sin_t;
  p.page_bytes = c->page_stride * e; p.slot_bytes = c->slot_stride * e; p.head_bytes = c->head_stride * e; p.q_stride = q_stride; p.kv_stride = kv_stride;
  p.rows = rows; p.H = n_heads; p.Hkv = c->n_kv_heads; p.D = c->head_dim; p.page = c->page_size; p.n_pages = c->n_pages; p.n_positions = n_positions;
  const cudaError_t r = c->dtype == OURO_F32 ? launch_pdl(append_kernel<float>, dim3(rows), dim3(APPEND_THREADS), 0, (cudaStream_t)stream, p)
                                             : launch_pdl(append_kernel<__nv_bfloat16>, dim3(rows), dim3(APPEND_THREADS), 0, (cudaStream_t)stream, p);
  OURO_COUNT_LAUNCH();
  return r == cudaSuccess ? OURO_OK : paged::refuse(call, cudaGetErrorString(r), OURO_ECUDA);
}
