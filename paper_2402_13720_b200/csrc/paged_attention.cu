// Attention of the newest tokens of several sequences over a paged cache, split over the cache's length and joined.
//
//     o = sum_j e^(s_j) v_j / sum_j e^(s_j),   s_j = scale q . k_j,   j over the keys a token sees
//
// Bound by HBM: a key and a value are 4 head_dim bytes (bf16) and give 4 head_dim operations per query head that shares them, at most a
// few dozen operations a byte.  So the whole design is about reading every key and value once, without a pause, on all SMs:
//  - The query rows that share a kv head (new tokens x query heads of its group) are row tiles of 8 or 16, a sequence's kv
//    head and row tile an item, TILE keys of an item a unit.  All units of a call, in order, are dealt out to the CTAs in runs of the same
//    cost whatever the lengths are (paged_runs.cuh).  An item that lies in one CTA is finished there; of an item cut between CTAs each leaves
//    a piece (maximum, sum, unnormalised output, in 32 bits), and the CTA that is last to do so joins the pieces in ascending order
//    (so the result does not depend on who that is).
//  - A warp fetches KW keys of every unit into its part of a ring in shared memory, STAGES - 1 units ahead, across the borders of items;
//    the ids of pages are read before that, 32 units' at a time.  A warp works on the keys that it fetched; warps meet only at an item's end.
//  - bf16: S = Q K^T and O += P V as mma.sync m16n8k16 with Q, P and O in registers (the tensor cores idle most of the time
//    anyway).  P goes in as two bf16 parts, P = hi + lo up to 2^-17: one part alone would add an error as large as the output's own
//    rounding.  Up to 8 query rows the parts are the two halves of one 16-row operand, beyond that two contractions.
//    f32: multiply-adds in 32 bits, two in an instruction, bound by what comes from shared memory: a lane has two keys and an eighth of the dims for all R
//    rows, so that the queries are read once for two keys; the eight lanes' sums end up one row to a lane, which alone sees to its maximum
//    and exponentials.  (us for floors of 21, 10.7, 8.3: 70B shape, 4 x 4096 34, 32 ragged up to 473 26, 34B shape, 59 up to 146 with 5 new tokens
//    67; with a key to four lanes 41, 31, 83; with a branch for each row that is there 110, 89, 268.)
// Keys that are not there (beyond the length, on no page) have probability 0, and zeros take their values' place.
#include <cuda.h>

#include "paged_runs.cuh"

namespace {

using paged::AttnParams;
using paged::MAX_CTAS;
using paged::Walk;

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr int MAX_LIST = OURO_MAX_LIST;
constexpr int ITEM_COST = 2;                        // what an item costs besides its units, in units
// A unit takes a CTA about a microsecond alone (a chain of latencies), a join two and more.  us (with joins a microsecond longer) with runs from 1, 2, 4 units on, borders taken within
// 0, 1, 3: one sequence of 700 keys (1.1B shape) 7.9, 9.4, 12.0; one of 1024 (70B shape) 9.4, 9.4, 13.2, of 4096 14.5, 13.3, 14.9; 60 ragged up to
// 700 15.3, 14.2, 13.7; 16 of 512 15.1, 15.1, 13.7; one of 20000 with two kv heads 21.3, 21.2, 18.7; large calls the same.
constexpr int SNAP = 1;                             // units in front of or behind a cut for which it is not worth its join
constexpr int MIN_RUN = 2;                          // units for which another CTA is
// More query rows of a kv head go to paged_attention_tc.cu (head dims 64 and 128, pages of a multiple of 16).  us here and there: 35 rows, 34B drafts 16.8 and 16.6, 27 ragged up to 393
// 27.2 and 22.2; 40 rows (70B shape), 64 ragged up to 300 40.5 and 27.1, one of 11993 34.1 and 26.8; 56 rows, two up to 4998 35.3 and 23.8; 128 rows, 8 of
// 4096 153 and 48.6; 64 rows of head dim 64, one of 700 9.5 and 11.0.  At 16 rows: 16 of 1000 (70B) 21.2 and 27.2, of the 1.1B shape 11.7 and 18.2.
constexpr int MMA_ROWS = 16;
constexpr float GROWTH = 8.f;                       // (log2) a maximum may grow by this before sums are rescaled: they stay below 2^8 per key
constexpr int DRAIN_POLLS = 1 << 14;                // of a call that gave up, for a copy still under way to end (some 200 us; a copy takes a few)

// The pools as five dimensions (dim, head, row, page, layer); boxes of 64 dims x 16 rows.
struct Maps {
  CUtensorMap k, v;
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes, or zeros where there is nothing to read
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int dim, int head, int row, int page, int layer) {
  // (read once: evict first)
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5, %6, %7}], [%2], %8;" ::"r"(dst),
      "l"(map), "r"(bar), "r"(dim), "r"(head), "r"(row), "r"(page), "r"(layer), "l"(0x12F0000000000000ull)
      : "memory");
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_poll(uint32_t bar, uint32_t parity) {   // without suspending the thread
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t *r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t *r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16(float *d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&t);
}
// What two bf16 parts leave of a pair: x - bf16(x), rounded.
__device__ __forceinline__ uint32_t rest(float a, float b, uint32_t hi) {
  return pack(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
}
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

// Two 32-bit numbers at a time.
__device__ __forceinline__ u64 pair(float a, float b) {
  u64 y;
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ void unpair(u64 x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) {
  u64 y;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
  return y;
}

// T: the cache's type.  R: query rows of a tile (8 or 16; f32: 1, 4 or 8).
template <typename T, int D, int R>
struct Cfg {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int KW = BF ? 16 : 8;            // keys of a warp in a unit
  static constexpr int TILE = KW * WARPS;
  // A warp's stage: K rows, then V rows.  bf16: boxes of 64 dims, 16 rows of 128 bytes, whose 16-byte pieces are exchanged by the row (the
  // copy engine's 128-byte swizzle).  f32: rows 16 bytes longer than they are.
  static constexpr int BOXES = (D + 63) / 64, BOX = KW * 128;
  static constexpr int PITCH = D * 4 + 16;
  static constexpr int HALF_STAGE = BF ? BOXES * BOX : KW * PITCH;
  static constexpr int STAGE = 2 * HALF_STAGE;
  // (f32, 128: two CTAs on an SM with two stages, one with three: four sequences of 1024, 7B shape, 29 and 32 us, of 4096, 70B shape, 34 and 44)
  static constexpr int STAGES = BF ? (D <= 64 ? 4 : 3) : D == 128 ? 2 : D == 96 ? 3 : 4;
  [[maybe_unused]] static constexpr int KEY_LANES = D == 96 ? 1 : 128 / D;   // f32: keys whose values the lanes of a warp work on at a time
  static constexpr int OFF_RING = 0;                                      // [warp][stage]
  static constexpr int OFF_Q = WARPS * STAGES * STAGE;                    // f32: [warp][R][D]
  static constexpr int OFF_P = OFF_Q + (BF ? 0 : WARPS * R * D * 4);      // f32: [warp][key][R]
  static constexpr int OFF_ML = OFF_P + (BF ? 0 : WARPS * KW * R * 4);    // [warp][R][2]
  static constexpr int OFF_JOIN = OFF_ML + WARPS * R * 8;                // [6][THREADS]: shares of a join
  static constexpr int OFF_BAR = OFF_JOIN + 6 * THREADS * 4;                // [warp][stage]
  static constexpr int OFF_MASK = OFF_BAR + WARPS * STAGES * 8;           // [warp][stage]
  static constexpr int OFF_LEN = OFF_MASK + WARPS * STAGES * 4;           // [n]
  static constexpr int OFF_CUM = OFF_LEN + MAX_LIST * 4;                  // [n + 1] cost of a head and row tile
  static constexpr int OFF_MISC = OFF_CUM + (MAX_LIST + 1) * 4;
  static constexpr int BYTES = OFF_MISC + 64;
  static_assert(R * D * 4 <= STAGE && R <= paged::ROW_TILE, "a warp's output fits its stage");
};

// TMA: the copy engine fetches (bf16, pages of a multiple of 16 rows).
template <typename T, int D, int R, bool TMA>
__global__ void __launch_bounds__(THREADS, 2) paged_attention_kernel(const AttnParams p, const __grid_constant__ Maps maps) {
  using C = Cfg<T, D, R>;
  extern __shared__ __align__(1024) uint8_t smem[];
  int *s_len = (int *)(smem + C::OFF_LEN), *s_cum = (int *)(smem + C::OFF_CUM), *s_misc = (int *)(smem + C::OFF_MISC);
  volatile int *s_abort = s_misc + 5;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t bars = smem_u32(smem + C::OFF_BAR) + warp * C::STAGES * 8;
  if constexpr (TMA) {
    if (lane < C::STAGES) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + lane * 8) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (tid == 0) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.v) : "memory");
    }
  }
  if (tid == 0) *s_abort = 0;
  pdl_wait();
  pdl_trigger();

  const paged::Runs<C::TILE, ITEM_COST, SNAP, MIN_RUN> runs(p, gridDim.x, s_len, s_cum, s_misc, THREADS);
  if (blockIdx.x >= runs.G) return;
  Walk c = runs.place(blockIdx.x);                                 // the unit being worked on
  const Walk end = runs.place(blockIdx.x + 1);
  if (paged::same(c, end)) return;

  // ---- the warp's ring
  uint8_t *ring_p = smem + C::OFF_RING + warp * C::STAGES * C::STAGE;
  const uint32_t ring = smem_u32(ring_p);
  volatile uint32_t *s_mask = (volatile uint32_t *)(smem + C::OFF_MASK) + warp * C::STAGES;   // which keys are there
  uint32_t phases = 0;                                             // of the barriers, a bit each
  Walk f = c;                                                      // the unit to be fetched next
  bool f_on = true;
  // Pages.  Copy engine: of the warp's keys in 32 units from unit ids_base on, one a lane, and in the 32 after that; else of its keys
  // in the next unit, one a lane.
  int ids = -1, ids_after = -1, ids_base = 0, ids_seq = -1, f_row = 0;
  auto ids_from = [&](int tile) {
    const int key = (tile + lane) * C::TILE + warp * C::KW;
    return key < f.len ? f.row[key < f.len ? p.page.quot(key) : 0] : -1;
  };
  auto read_ids = [&]() {
    if (!f_on) return;
    if constexpr (TMA) {
      if (f.s != ids_seq || f.tile < ids_base || f.tile >= ids_base + 64) {
        ids_seq = f.s;
        ids_base = f.tile;
        ids = ids_from(f.tile);
        ids_after = f.tiles > f.tile + 32 ? ids_from(f.tile + 32) : -1;
      } else if (f.tile == ids_base + 32) {
        ids_base = f.tile;
        ids = ids_after;
        ids_after = f.tiles > f.tile + 32 ? ids_from(f.tile + 32) : -1;
      }
    } else {
      const int key = f.tile * C::TILE + warp * C::KW + (lane & (C::KW - 1)), pg = p.page.quot(key);
      f_row = key - pg * (int)p.page.d;
      ids = key < f.len ? f.row[key < f.len ? pg : 0] : -1;
    }
  };
  auto fetch = [&](int stage) {
    if (f_on) {
      const int head = f.head;
      const uint32_t dst = ring + stage * C::STAGE;
      if constexpr (TMA) {
        const int key = f.tile * C::TILE + warp * C::KW, id = __shfl_sync(0xffffffffu, ids, f.tile - ids_base);
        if (key < f.len) {                                         // (else the warp has no keys in the unit)
          if (elect_one() && !*s_abort) {                          // (who gave up is asked by the one thread: the warp stays together)
            const bool there = id >= 0 && id < p.n_pages;
            s_mask[stage] = there ? 0xffffu : 0u;
            const uint32_t bar = bars + stage * 8;
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(C::STAGE) : "memory");
            const int page = there ? id : p.n_pages, row = key - p.page.quot(key) * (int)p.page.d;   // beyond the pool: zeros, nothing is read
#pragma unroll
            for (int b = 0; b < C::BOXES; ++b) {
              tma_load(dst + b * C::BOX, &maps.k, bar, b * 64, head, row, page, p.layer);
              tma_load(dst + C::HALF_STAGE + b * C::BOX, &maps.v, bar, b * 64, head, row, page, p.layer);
            }
          }
          __syncwarp();
        }
      } else {
        const bool there = ids >= 0 && ids < p.n_pages;
        const int64_t off = there ? (int64_t)ids * p.page_bytes + (int64_t)f_row * p.slot_bytes + (int64_t)head * p.head_bytes : -1;
        const uint32_t mask = __ballot_sync(0xffffffffu, there) & ((1u << C::KW) - 1);
        if (lane == 0) s_mask[stage] = mask;
        constexpr int CH = D * (int)sizeof(T) / 16, N = C::KW * CH;   // 16-byte pieces of a row, of all rows
#pragma unroll
        for (int i = 0; i < (N + 31) / 32; ++i) {
          const int e = i * 32 + lane, r = e / CH, ch = e - r * CH;
          const int64_t ro = __shfl_sync(0xffffffffu, off, r & (C::KW - 1));
          if (N % 32 == 0 || e < N) {
            const int64_t o = ro < 0 ? 0 : ro + ch * 16;
            const uint32_t to = dst + (C::BF ? (ch >> 3) * C::BOX + r * 128 + (((ch & 7) ^ (r & 7)) << 4) : r * C::PITCH + ch * 16);
            cp_async16(to, p.k + o, ro >= 0);
            cp_async16(to + C::HALF_STAGE, p.v + o, ro >= 0);
          }
        }
      }
      runs.next(f);
      f_on = !paged::same(f, end);
      read_ids();
    }
    if constexpr (!TMA) asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // Bounded wait for a stage's copies.  Whoever gives up raises the status; from then on nobody in the CTA fetches or waits, and the call
  // ends with wrong results and an error.
  auto wait = [&](int stage) {
    if constexpr (TMA) {
      const uint32_t parity = phases >> stage & 1;
      bool done = false;
      for (uint32_t i = 0; i < p.wait_limit && !done; ++i) {
        done = mbar_test(bars + stage * 8, parity);
        if (!done && (i & 63) == 63 && *s_abort) break;
      }
      // (each lane polls for itself; ldmatrix and the contractions behind this want the warp together)
      if (__all_sync(0xffffffffu, done)) {
        phases ^= 1u << stage;
        return;
      }
      *s_abort = 1;
      if (lane == 0) atomicCAS(p.status, OURO_OK, OURO_ETIMEOUT);
    } else {
      asm volatile("cp.async.wait_group %0;" ::"n"(C::STAGES - 2) : "memory");
      __syncwarp();
    }
  };
  read_ids();
#pragma unroll
  for (int i = 0; i < C::STAGES - 1; ++i) fetch(i);

  // ---- state of the item.  bf16: mma fragments, rows lane / 4 (and + 8; up to 8 rows that half holds the probabilities' second parts);
  // f32: four columns a lane.
  constexpr int NACC = C::BF ? D / 2 : R * 4, NST = C::BF ? R / 8 : 1;
  float acc[NACC], m[NST], l[NST];
  uint32_t qf[C::BF ? D / 16 * 2 * NST : 1];                       // [step][row half][k half]
  int vis[NST];
  float *s_q = (float *)(smem + C::OFF_Q) + (C::BF ? 0 : warp * R * D);
  float *s_p = (float *)(smem + C::OFF_P) + (C::BF ? 0 : warp * C::KW * R);
  float *s_ml = (float *)(smem + C::OFF_ML);
  auto slot_of = [](int r, int i) { return R == 1 ? i : ((r >> 1) * 4 + i) * 2 + (r & 1); };   // f32: of row r, column i in acc: two rows side by side
  bool fresh = true;
  int first_tile = 0;                                              // of the item's part that this CTA has

  for (int stage = 0;; stage = stage + 1 == C::STAGES ? 0 : stage + 1) {
    const int rt = c.rt, kvh = c.head;
    const int rows = min(R, p.rows - rt * R);                      // of this tile
    if (fresh) {                                                   // (the queries are on their way while the keys are waited for)
      fresh = false;
      first_tile = c.tile;
#pragma unroll
      for (int i = 0; i < NACC; ++i) acc[i] = 0.f;
#pragma unroll
      for (int i = 0; i < NST; ++i) {
        const int r = C::BF ? (lane >> 2) + 8 * i : lane & (R - 1), at = rt * R + min(r, rows - 1), tok = p.group_of.quot(at);
        m[i] = -INFINITY;
        l[i] = 0.f;
        vis[i] = r < rows ? c.len - p.n_new + 1 + tok : 0;
        if constexpr (C::BF) {
          const int64_t q_at = ((int64_t)c.s * p.n_new + tok) * p.q_stride + (int64_t)(kvh * p.group + at - tok * p.group) * D;
          const uint32_t *src = (const uint32_t *)((const __nv_bfloat16 *)p.q + q_at) + (lane & 3);
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
            qf[(j * NST + i) * 2] = r < rows ? src[j * 8] : 0u;
            qf[(j * NST + i) * 2 + 1] = r < rows ? src[j * 8 + 4] : 0u;
          }
        }
      }
      if constexpr (!C::BF) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int at = rt * R + min(r, rows - 1), tok = p.group_of.quot(at);
          const int64_t q_at = ((int64_t)c.s * p.n_new + tok) * p.q_stride + (int64_t)(kvh * p.group + at - tok * p.group) * D;
          const float4 x = *(const float4 *)((const float *)p.q + q_at + min(lane, D / 4 - 1) * 4);
          if (lane < D / 4) *(float4 *)(s_q + r * D + lane * 4) = r < rows ? x : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
      if (!C::BF) __syncwarp();
    }
    const int key0 = c.tile * C::TILE + warp * C::KW;
    const bool mine = !TMA || key0 < c.len;                        // the warp has keys in the unit
    if (mine) wait(stage);
    fetch(stage == 0 ? C::STAGES - 1 : stage - 1);
    if (mine) {
      uint8_t *kp = ring_p + stage * C::STAGE, *vp = kp + C::HALF_STAGE;
      const uint32_t kb = ring + stage * C::STAGE, vb = kb + C::HALF_STAGE;
      const uint32_t mask = s_mask[stage];
      if constexpr (C::BF) {
        if (TMA && key0 + C::KW > c.len) {                         // rows of the page that are not the sequence's: 0 times them must be 0
          for (int e = lane; e < (key0 + C::KW - c.len) * 8 * C::BOXES; e += 32)
            *(uint4 *)(vp + (e & 7) * 16 + ((e >> 3) % C::BOXES) * C::BOX + (C::KW - 1 - (e >> 3) / C::BOXES) * 128) = make_uint4(0, 0, 0, 0);
          fence_async_smem();                                      // (before the copy engine writes there again)
          __syncwarp();
        }
        const int t2 = (lane & 3) * 2;
        float sc[4 * NST];                                         // [row half][key block of 8][2 keys]
        {
          float x[2][4] = {};                                      // [key block]
          const int r = (lane & 7) + ((lane & 16) >> 1), sw = ((lane >> 3) ^ lane) & 1;
          const uint32_t ka = kb + r * 128 + (((lane & 6) | sw) << 4);
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
            uint32_t b[4];
            ldsm_x4((ka ^ ((2 * j & 6) << 4)) + (j >> 2) * C::BOX, b);
            const uint32_t *q = qf + j * NST * 2;
            mma16(x[0], q[0], NST > 1 ? q[2 * (NST - 1)] : 0u, q[1], NST > 1 ? q[2 * (NST - 1) + 1] : 0u, b[0], b[1]);
            mma16(x[1], q[0], NST > 1 ? q[2 * (NST - 1)] : 0u, q[1], NST > 1 ? q[2 * (NST - 1) + 1] : 0u, b[2], b[3]);
          }
#pragma unroll
          for (int i = 0; i < 4 * NST; ++i) sc[i] = x[(i >> 1) & 1][2 * (i >> 2) + (i & 1)];
        }
        if (mask != 0xffffu || key0 + C::KW > c.len - p.n_new + 1) {   // (uniform) not every row sees every key
#pragma unroll
          for (int i = 0; i < 4 * NST; ++i) {
            const int kk = ((i >> 1) & 1) * 8 + t2 + (i & 1);
            if (!(mask >> kk & 1) || key0 + kk >= vis[i >> 2]) sc[i] = -INFINITY;
          }
        }
        bool grown = false;
        float a[NST];
#pragma unroll
        for (int h = 0; h < NST; ++h) {
          float mx = fmaxf(fmaxf(sc[4 * h], sc[4 * h + 1]), fmaxf(sc[4 * h + 2], sc[4 * h + 3]));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2)) * p.scale_log2;
          a[h] = 1.f;
          if (mx > m[h] + GROWTH) {
            a[h] = ex2(m[h] - mx);
            m[h] = mx;
            grown = true;
          }
        }
        if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
          for (int h = 0; h < NST; ++h) l[h] *= a[h];
#pragma unroll
          for (int i = 0; i < NACC; ++i) acc[i] *= a[(i >> 1) & (NST - 1)];
        }
#pragma unroll
        for (int h = 0; h < NST; ++h) {
          const float base = base_of(m[h]);
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[4 * h + i] = ex2(fmaf(sc[4 * h + i], p.scale_log2, -base));
          l[h] += (sc[4 * h] + sc[4 * h + 1]) + (sc[4 * h + 2] + sc[4 * h + 3]);
        }
        // A later token's key may lie in the tile although an earlier one does not see it; 0 times what is stored there must be 0
        // whatever it is.
        bool odd = false;
        if (p.n_new > 1 && key0 + C::KW > c.len - p.n_new) {
          for (int e = lane; e < C::HALF_STAGE / 16; e += 32) {
            if (D % 64 && (e / (C::BOX / 16) == C::BOXES - 1) && !TMA && ((e & 7) ^ ((e >> 3) & 7)) >= (D % 64) / 8) continue;   // (columns that there are not)
            const uint4 x = *(const uint4 *)(vp + e * 16);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
          }
          odd = __any_sync(0xffffffffu, odd);
        }
        if (!odd) {
          uint32_t hi[2 * NST], lo[2 * NST];                       // [row half][key block]
#pragma unroll
          for (int i = 0; i < 2 * NST; ++i) {
            hi[i] = pack(sc[2 * i], sc[2 * i + 1]);
            lo[i] = rest(sc[2 * i], sc[2 * i + 1], hi[i]);
          }
          const int sw = ((lane >> 4) ^ lane) & 1;
          const uint32_t va = vb + (lane & 15) * 128 + (((lane & 6) | sw) << 4);
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
            uint32_t b[4];
            ldsm_x4_t((va ^ ((2 * j & 6) << 4)) + (j >> 2) * C::BOX, b);
            if constexpr (NST == 1) {                              // the lower rows are the second parts
              mma16(acc + 8 * j, hi[0], lo[0], hi[1], lo[1], b[0], b[1]);
              mma16(acc + 8 * j + 4, hi[0], lo[0], hi[1], lo[1], b[2], b[3]);
            } else {
              mma16(acc + 8 * j, hi[0], hi[2], hi[1], hi[3], b[0], b[1]);
              mma16(acc + 8 * j + 4, hi[0], hi[2], hi[1], hi[3], b[2], b[3]);
              mma16(acc + 8 * j, lo[0], lo[2], lo[1], lo[3], b[0], b[1]);
              mma16(acc + 8 * j + 4, lo[0], lo[2], lo[1], lo[3], b[2], b[3]);
            }
          }
        } else {
          for (int j = 0; j < C::KW; ++j) {
            float pr[NST];
#pragma unroll
            for (int h = 0; h < NST; ++h) {
              const float x = __shfl_sync(0xffffffffu, j < 8 ? sc[4 * h] : sc[4 * h + 2], (lane & 28) + ((j & 7) >> 1));
              const float y = __shfl_sync(0xffffffffu, j < 8 ? sc[4 * h + 1] : sc[4 * h + 3], (lane & 28) + ((j & 7) >> 1));
              pr[h] = j & 1 ? y : x;
            }
            const bool on = mask >> j & 1;
#pragma unroll
            for (int b = 0; b < D / 8; ++b) {
              const uint32_t w = *(const uint32_t *)(vp + (b >> 3) * C::BOX + j * 128 + (((b & 7) ^ (j & 7)) << 4) + t2 * 2);
              const float v0 = __uint_as_float(w << 16), v1 = __uint_as_float(w & 0xffff0000u);
#pragma unroll
              for (int h = 0; h < NST; ++h)
                if (on && key0 + j < vis[h]) {
                  acc[4 * b + 2 * h] = fmaf(pr[h], v0, acc[4 * b + 2 * h]);
                  acc[4 * b + 2 * h + 1] = fmaf(pr[h], v1, acc[4 * b + 2 * h + 1]);
                }
            }
          }
        }
      } else {
        // Scores: two keys have eight lanes, each an eighth of the dims (every eighth piece of four).  All R rows, whether there or not: a branch for
        // each would put their chains one after another.
        const int part = lane & 7, pair_of = lane >> 3;
        const float *kr = (const float *)(kp + pair_of * 2 * C::PITCH);
        float x[2][R];
        {
          u64 s2[2][R];
#pragma unroll
          for (int r = 0; r < R; ++r) s2[0][r] = s2[1][r] = 0;
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            const int d = (8 * j + part) * 4;
            const ulonglong2 k0 = *(const ulonglong2 *)(kr + d), k1 = *(const ulonglong2 *)(kr + C::PITCH / 4 + d);
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const ulonglong2 qq = *(const ulonglong2 *)(s_q + r * D + d);
              s2[0][r] = fma2(k0.y, qq.y, fma2(k0.x, qq.x, s2[0][r]));
              s2[1][r] = fma2(k1.y, qq.y, fma2(k1.x, qq.x, s2[1][r]));
            }
          }
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < R; ++r) {
              float a, b;
              unpair(s2[k][r], a, b);
              x[k][r] = a + b;
            }
        }
        // The eight lanes' sums: of each two numbers a lane keeps one and hands the other over, until it has its own row's (8 rows: of both keys; fewer:
        // of one key, the second in lanes 4 to 7).
        constexpr int NX = R == 8 ? 2 : 1;
        auto halve = [&](float a, float b, int o) {                // a to the lanes without bit o, b to those with it
          const bool up = lane & o;
          return (up ? b : a) + __shfl_xor_sync(0xffffffffu, up ? a : b, o);
        };
        float sc[NX];
        if constexpr (R == 8) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int r = 0; r < 4; ++r) x[k][r] = halve(x[k][r], x[k][r + 4], 4);
#pragma unroll
            for (int r = 0; r < 2; ++r) x[k][r] = halve(x[k][r], x[k][r + 2], 2);
            sc[k] = halve(x[k][0], x[k][1], 1);
          }
        } else {
#pragma unroll
          for (int r = 0; r < R; ++r) x[0][r] = halve(x[0][r], x[1][r], 4);
          if constexpr (R == 4) {
#pragma unroll
            for (int r = 0; r < 2; ++r) x[0][r] = halve(x[0][r], x[0][r + 2], 2);
            sc[0] = halve(x[0][0], x[0][1], 1);
          } else {
            sc[0] = x[0][0];
            sc[0] += __shfl_xor_sync(0xffffffffu, sc[0], 2);
            sc[0] += __shfl_xor_sync(0xffffffffu, sc[0], 1);
          }
        }
        constexpr int KEYS_FROM = R == 8 ? 8 : 4;                  // from this bit on lanes differ in the key
        const int row = lane & (R - 1), key = pair_of * 2 + (R == 8 ? 0 : lane >> 2 & 1);
        const bool all = mask == (1u << C::KW) - 1 && key0 + C::KW <= c.len - p.n_new + 1;   // (uniform) every row sees every key
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < NX; ++i) {
          sc[i] = all || ((mask >> (key + i) & 1) && key0 + key + i < vis[0]) ? sc[i] * p.scale_log2 : -INFINITY;
          mx = fmaxf(mx, sc[i]);
        }
        if (__any_sync(0xffffffffu, mx > m[0] + GROWTH)) {
#pragma unroll
          for (int o = KEYS_FROM; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
          const float a = mx > m[0] + GROWTH ? ex2(m[0] - mx) : 1.f;
          if (mx > m[0] + GROWTH) m[0] = mx;
          l[0] *= a;
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float ar = __shfl_sync(0xffffffffu, a, r);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[slot_of(r, i)] *= ar;
          }
        }
#pragma unroll
        for (int i = 0; i < NX; ++i) {
          const float e = ex2(sc[i] - base_of(m[0]));
          l[0] += e;
          s_p[(key + i) * R + row] = e;                            // (one row: four lanes the same)
        }
        __syncwarp();
        const int kl = C::KEY_LANES > 1 ? lane / (D / 4) : 0, col = min(lane - kl * (D / 4), D / 4 - 1) * 4;
        if (p.n_new == 1 || all) {                                 // (the values of keys that are not there are zeros)
#pragma unroll
          for (int j0 = 0; j0 < C::KW; j0 += C::KEY_LANES) {
            const int j = j0 + kl;
            const float4 vv = *(const float4 *)(vp + j * C::PITCH + col * 4);
            if constexpr (R == 1) {
              const float pr = s_p[j];
              acc[0] = fmaf(pr, vv.x, acc[0]);
              acc[1] = fmaf(pr, vv.y, acc[1]);
              acc[2] = fmaf(pr, vv.z, acc[2]);
              acc[3] = fmaf(pr, vv.w, acc[3]);
            } else {
              const u64 v2[4] = {pair(vv.x, vv.x), pair(vv.y, vv.y), pair(vv.z, vv.z), pair(vv.w, vv.w)};
#pragma unroll
              for (int r = 0; r < R; r += 4) {
                const ulonglong2 pr = *(const ulonglong2 *)(s_p + j * R + r);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  float *a = acc + slot_of(r, i), *b = acc + slot_of(r + 2, i);
                  unpair(fma2(pr.x, v2[i], pair(a[0], a[1])), a[0], a[1]);
                  unpair(fma2(pr.y, v2[i], pair(b[0], b[1])), b[0], b[1]);
                }
              }
            }
          }
        } else {                                                   // (0 times what is stored there would not be 0 for all values)
          int seen[R];
#pragma unroll
          for (int r = 0; r < R; ++r) seen[r] = __shfl_sync(0xffffffffu, vis[0], r);
          for (int j = kl; j < C::KW; j += C::KEY_LANES) {
            const float4 vv = *(const float4 *)(vp + j * C::PITCH + col * 4);
#pragma unroll
            for (int r = 0; r < R; ++r)
              if ((mask >> j & 1) && key0 + j < seen[r]) {
                const float pr = s_p[j * R + r];
                acc[slot_of(r, 0)] = fmaf(pr, vv.x, acc[slot_of(r, 0)]);
                acc[slot_of(r, 1)] = fmaf(pr, vv.y, acc[slot_of(r, 1)]);
                acc[slot_of(r, 2)] = fmaf(pr, vv.z, acc[slot_of(r, 2)]);
                acc[slot_of(r, 3)] = fmaf(pr, vv.w, acc[slot_of(r, 3)]);
              }
          }
        }
      }
    }
    __syncwarp();                                                  // the stage has been read

    // ---- the item's or the run's end: the warps' parts are added up
    const Walk was = c;
    const bool item_ends = c.tile == c.tiles - 1;
    runs.next(c);
    const bool run_ends = paged::same(c, end);
    if (!item_ends && !run_ends) continue;
    {
      // The warp's part goes to the stage just read: [row][column], the columns of a row exchanged so that eight rows' stores hit different banks.
      float *part = (float *)(ring_p + stage * C::STAGE);
      if constexpr (C::BF) {
#pragma unroll
        for (int h = 0; h < NST; ++h) {
          l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
          l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
          const int r = (lane >> 2) + 8 * h;
          if (r < rows) {
#pragma unroll
            for (int b = 0; b < D / 8; ++b) {
              float2 o = make_float2(acc[4 * b + 2 * h], acc[4 * b + 2 * h + 1]);
              if (NST == 1) o = make_float2(o.x + acc[4 * b + 2], o.y + acc[4 * b + 3]);
              *(float2 *)(part + r * D + ((b * 8) ^ ((r & 3) * 8)) + (lane & 3) * 2) = o;
            }
            if ((lane & 3) == 0) *(float2 *)(s_ml + (warp * R + r) * 2) = make_float2(m[h], l[h]);
          }
        }
      } else {
#pragma unroll
        for (int o = R == 8 ? 8 : 4; o < 32; o <<= 1) l[0] += __shfl_xor_sync(0xffffffffu, l[0], o);
        if (lane < min(R, rows)) *(float2 *)(s_ml + (warp * R + lane) * 2) = make_float2(m[0], l[0]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
          for (int o = 16; o >= D / 4 && C::KEY_LANES > 1; o >>= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[slot_of(r, i)] += __shfl_xor_sync(0xffffffffu, acc[slot_of(r, i)], o);
          if (lane < D / 4 && r < rows)
            *(float4 *)(part + r * D + ((lane * 4) ^ ((r & 3) * 8))) = make_float4(acc[slot_of(r, 0)], acc[slot_of(r, 1)], acc[slot_of(r, 2)], acc[slot_of(r, 3)]);
        }
      }
      __syncthreads();
      const bool whole = item_ends && first_tile == 0;
      const int slot = first_tile == 0 ? 1 : 0;                    // pieces of a CTA: of an item it begins, of one it goes on with
      float *piece = p.pieces + ((int64_t)blockIdx.x * 2 + slot) * paged::ROW_TILE * D;
      float *mls = p.pieces + (int64_t)MAX_CTAS * 2 * paged::ROW_TILE * D;
      constexpr int C4 = D / 4;
      auto finish = [&](int r, int col, float M, float L, const float *o) {       // four columns of a row to the output
        const int at = rt * R + r, tok = p.group_of.quot(at), head = kvh * p.group + at - tok * p.group;
        const int64_t row = ((int64_t)was.s * p.n_new + tok) * p.H + head;
        const float inv = L == 0.f ? 0.f : 1.f / L;
        if constexpr (C::BF)
          *(uint2 *)((__nv_bfloat16 *)p.out + row * D + col) = make_uint2(pack(o[0] * inv, o[1] * inv), pack(o[2] * inv, o[3] * inv));
        else
          *(float4 *)((float *)p.out + row * D + col) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
        if (p.lse && col == 0) p.lse[row] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
      };
      for (int e = tid; e < rows * C4; e += THREADS) {
        const int r = e / C4, col = (e - r * C4) * 4;
        float M = -INFINITY, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WARPS; ++w) M = fmaxf(M, s_ml[(w * R + r) * 2]);
        const float base = base_of(M);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          const float a = ex2(s_ml[(w * R + r) * 2] - base);
          const float4 x = *(const float4 *)(smem + C::OFF_RING + (w * C::STAGES + stage) * C::STAGE + (r * D + (col ^ ((r & 3) * 8))) * 4);
          L = fmaf(a, s_ml[(w * R + r) * 2 + 1], L);
          o[0] = fmaf(a, x.x, o[0]);
          o[1] = fmaf(a, x.y, o[1]);
          o[2] = fmaf(a, x.z, o[2]);
          o[3] = fmaf(a, x.w, o[3]);
        }
        if (whole) {
          finish(r, col, M, L, o);
        } else {
          __stcg((float4 *)(piece + r * D + col), make_float4(o[0], o[1], o[2], o[3]));
          if (col == 0) __stcg((float2 *)(mls + (((int64_t)blockIdx.x * 2 + slot) * paged::ROW_TILE + r) * 2), make_float2(M, L));
        }
      }
      if (!whole) {
        int c0, c1;
        runs.owners(was, c0, c1);
        __syncthreads();
        if (tid == 0) {                                            // (releases what the CTA has written, acquires what the others have)
          int before;
          asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(p.counters + c0) : "memory");
          s_misc[4] = before == c1 - c0;
        }
        __syncthreads();
        if (s_misc[4]) {
          if (tid == 0) p.counters[c0] = 0;
          auto where = [&](int cta) { return ((int64_t)cta * 2 + (cta == c0 ? 1 : 0)) * paged::ROW_TILE; };
          // Four columns of a row, EACH times a thread; where that leaves threads over, the pieces are dealt out to `shares` of them.  Sums and outputs
          // of BATCH pieces are asked for at once, so that few pieces take one round trip.
          constexpr int EACH = (R * C4 + THREADS - 1) / THREADS, BATCH = EACH > 2 ? 2 : 8 / EACH;
          const int E = rows * C4, shares = E < THREADS ? THREADS / E : 1, share = shares > 1 ? tid / E : 0;
          int at[EACH];
          float M[EACH], L[EACH], o[EACH][4];
#pragma unroll
          for (int k = 0; k < EACH; ++k) {
            at[k] = min(k * THREADS + tid - share * E, E - 1);
            M[k] = -INFINITY;
            L[k] = o[k][0] = o[k][1] = o[k][2] = o[k][3] = 0.f;
          }
          for (int a0 = c0 + share; a0 <= c1; a0 += BATCH * shares) {
            float2 ml[EACH][BATCH];
            float4 y[EACH][BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
              const int64_t from = where(min(a0 + b * shares, c1));
#pragma unroll
              for (int k = 0; k < EACH; ++k) {
                ml[k][b] = __ldcg((const float2 *)(mls + (from + at[k] / C4) * 2));
                y[k][b] = __ldcg((const float4 *)(p.pieces + from * D + at[k] * 4));
              }
            }
#pragma unroll
            for (int k = 0; k < EACH; ++k) {
              float mx = M[k];
#pragma unroll
              for (int b = 0; b < BATCH; ++b) mx = fmaxf(mx, ml[k][b].x);    // (a piece twice changes no maximum)
              const float a = ex2(M[k] - base_of(mx));
              M[k] = mx;
              L[k] *= a;
#pragma unroll
              for (int i = 0; i < 4; ++i) o[k][i] *= a;
#pragma unroll
              for (int b = 0; b < BATCH; ++b) {
                if (a0 + b * shares > c1) continue;
                const float x = ex2(ml[k][b].x - base_of(mx));
                L[k] = fmaf(x, ml[k][b].y, L[k]);
                o[k][0] = fmaf(x, y[k][b].x, o[k][0]);
                o[k][1] = fmaf(x, y[k][b].y, o[k][1]);
                o[k][2] = fmaf(x, y[k][b].z, o[k][2]);
                o[k][3] = fmaf(x, y[k][b].w, o[k][3]);
              }
            }
          }
          if (shares > 1) {                                        // (EACH is 1 or has one element)
            float *s_part = (float *)(smem + C::OFF_JOIN);
            s_part[tid] = L[0];
#pragma unroll
            for (int i = 0; i < 4; ++i) s_part[(i + 1) * THREADS + tid] = o[0][i];
            s_part[5 * THREADS + tid] = M[0];
            __syncthreads();
            if (share == 0) {
              float mx = M[0];
              for (int w = 1; w < shares; ++w) mx = fmaxf(mx, s_part[5 * THREADS + w * E + tid]);
              const float a = ex2(M[0] - base_of(mx));
              M[0] = mx;
              L[0] *= a;
#pragma unroll
              for (int i = 0; i < 4; ++i) o[0][i] *= a;
              for (int w = 1; w < shares; ++w) {
                const float x = ex2(s_part[5 * THREADS + w * E + tid] - base_of(mx));
                L[0] = fmaf(x, s_part[w * E + tid], L[0]);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[0][i] = fmaf(x, s_part[(i + 1) * THREADS + w * E + tid], o[0][i]);
              }
            }
          }
#pragma unroll
          for (int k = 0; k < EACH; ++k)
            if (share == 0 && k * THREADS + tid < E) finish(at[k] / C4, at[k] % C4 * 4, M[k], L[k], o[k]);
        }
      }
      if (run_ends) break;
      if (TMA) fence_async_smem();                                 // (the parts, before the copy engine writes there again)
      __syncthreads();                                             // the stages and the sums may be written again
      fresh = true;
    }
  }
  if constexpr (!TMA) asm volatile("cp.async.wait_all;" ::: "memory");
  if constexpr (TMA)
    if (*s_abort)                                                  // copies may be under way still: a bounded time for them to end (a stage without one
      for (int i = 0; i < C::STAGES; ++i)                          // is polled in vain)
        for (int j = 0; j < DRAIN_POLLS && !mbar_poll(bars + i * 8, phases >> i & 1); ++j) {}
}

const char *CALL = "ouro_paged_attention";

}  // namespace

bool paged::make_map(CUtensorMap *m, const ouro_paged_cache *c, const void *base, int box_rows) {
  typedef CUresult (*encode_fn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static encode_fn encode = nullptr;
  if (!encode) {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess || !fn) return false;
    encode = (encode_fn)fn;
  }
  const cuuint64_t dims[5] = {(cuuint64_t)c->head_dim, (cuuint64_t)c->n_kv_heads, (cuuint64_t)c->page_size, (cuuint64_t)c->n_pages, (cuuint64_t)c->n_layers};
  // (a dimension of one element is never stepped over, but its stride must be a valid one)
  const int64_t st[4] = {c->head_stride, c->slot_stride, c->page_stride, c->layer_stride};
  cuuint64_t strides[4];
  for (int i = 0; i < 4; ++i) strides[i] = dims[i + 1] == 1 && st[i] == 0 ? (cuuint64_t)c->head_dim * 2 : (cuuint64_t)st[i] * 2;
  const cuuint32_t box[5] = {64, 1, (cuuint32_t)box_rows, 1, 1}, one[5] = {1, 1, 1, 1, 1};
  return encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

template <typename T, int D, int R, bool TMA>
int launch(const AttnParams &p, const Maps &maps, int64_t most_cost, cudaStream_t s) {
  using C = Cfg<T, D, R>;
  static int fit[paged::MAX_DEVICES] = {};                         // CTAs that are resident at once, per device
  int dev = 0, sms = 0;
  if (!paged::device(&dev, &sms)) return paged::refuse(CALL, "no usable current device", OURO_ECUDA);
  if (!fit[dev]) {
    int per_sm = 0;
    cudaError_t e = cudaFuncSetAttribute(paged_attention_kernel<T, D, R, TMA>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::BYTES);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, paged_attention_kernel<T, D, R, TMA>, THREADS, C::BYTES);
    if (e != cudaSuccess) return paged::refuse(CALL, cudaGetErrorString(e), OURO_ECUDA);
    if (per_sm < 1) return paged::refuse(CALL, "the kernel does not fit this device", OURO_ECUDA);
    fit[dev] = min(MAX_CTAS, sms * per_sm);
  }
  const int grid = (int)min((int64_t)fit[dev], max((int64_t)1, most_cost / MIN_RUN));
  const cudaError_t e = launch_pdl(paged_attention_kernel<T, D, R, TMA>, dim3(grid), dim3(THREADS), C::BYTES, s, p, maps);
  OURO_COUNT_LAUNCH();
  return e == cudaSuccess ? OURO_OK : paged::refuse(CALL, cudaGetErrorString(e), OURO_ECUDA);
}

template <int D>
int by_kind(const ouro_paged_cache *c, AttnParams p, bool tma, const Maps &maps, int64_t cost, cudaStream_t s) {
  // (us with tiles of 1, 4, 8 rows: one row, 7B shape, 4 x 1024 28.7, 29.4, 33.7, 76 x 1528 of `tiny` 33.8, 46, 54; two, 7B shape: -, 29.6, 34.1)
  if (c->dtype == OURO_F32)
    return p.rows == 1 ? launch<float, D, 1, false>(p, maps, cost, s) : p.rows <= 4 ? launch<float, D, 4, false>(p, maps, cost, s) : launch<float, D, 8, false>(p, maps, cost, s);
  if (p.rows <= 8) return tma ? launch<__nv_bfloat16, D, 8, true>(p, maps, cost, s) : launch<__nv_bfloat16, D, 8, false>(p, maps, cost, s);
  return tma ? launch<__nv_bfloat16, D, 16, true>(p, maps, cost, s) : launch<__nv_bfloat16, D, 16, false>(p, maps, cost, s);
}

}  // namespace

std::atomic<uint32_t> paged::wait_limit{paged::WAIT_LIMIT};

extern "C" int ouro_paged_debug_set_wait_limit(int64_t polls) {
  paged::wait_limit = polls < 0 || polls > paged::WAIT_LIMIT ? paged::WAIT_LIMIT : (uint32_t)polls;
  return OURO_OK;
}

extern "C" int ouro_paged_attention(const ouro_paged_cache *c, int32_t layer, const int32_t *seqs, int32_t n, int32_t n_new, const void *q,
                                    int64_t q_stride, int32_t n_heads, float scale, void *out, float *lse, void *stream) {
  if (const char *w = paged::wrong(c)) return paged::refuse(CALL, w);
  if (layer < 0 || layer >= c->n_layers) return paged::refuse(CALL, "no such layer");
  if (n < 0 || n > OURO_MAX_LIST) return paged::refuse(CALL, "n is below 0 or above OURO_MAX_LIST");
  if (n_new < 1 || n_new > OURO_MAX_NEW) return paged::refuse(CALL, "n_new is below 1 or above OURO_MAX_NEW");
  if (n_heads < 1 || n_heads % c->n_kv_heads) return paged::refuse(CALL, "n_heads is not a multiple of the cache's n_kv_heads");
  if (!(scale > 0.f) || scale > 1e30f) return paged::refuse(CALL, "scale is not a positive number");
  if (n == 0) return OURO_OK;
  if (!q || !out) return paged::refuse(CALL, "q or out is NULL");
  if (!paged::words(seqs, lse)) return paged::refuse(CALL, "seqs or lse is not 4-byte aligned");
  if (!seqs && n > c->max_seqs) return paged::refuse(CALL, "more sequences than the table has");
  const int esize = c->dtype == OURO_F32 ? 4 : 2;
  if (((uintptr_t)q | (uintptr_t)out) % 16 || (q_stride * esize) % 16) return paged::refuse(CALL, "q, out or q_stride is not a multiple of 16 bytes");
  if (q_stride < (int64_t)n_heads * c->head_dim) return paged::refuse(CALL, "q_stride is below n_heads * head_dim");
  AttnParams p{};
  p.group = n_heads / c->n_kv_heads;
  p.rows = n_new * p.group;
  const int tile = (c->dtype == OURO_F32 ? 8 : 16) * WARPS, rows_of = c->dtype == OURO_F32 ? (p.rows == 1 ? 1 : p.rows <= 4 ? 4 : 8) : p.rows <= 8 ? 8 : 16;
  p.row_tiles = (p.rows + rows_of - 1) / rows_of;
  p.cap = c->max_pages * c->page_size;
  const int64_t cost = (((int64_t)p.cap + tile - 1) / tile + 8) * c->n_kv_heads * p.row_tiles;   // (8: no kernel's item costs more)
  if (cost > INT32_MAX || cost / (c->n_kv_heads * p.row_tiles) * n > INT32_MAX) return paged::refuse(CALL, "the sequences' work is above 2^31 units");
  const paged::Layout l = paged::layout(*c);
  p.k = (const uint8_t *)c->k + (int64_t)layer * c->layer_stride * esize;
  p.v = (const uint8_t *)c->v + (int64_t)layer * c->layer_stride * esize;
  p.table = c->table; p.lens = c->lens; p.seqs = seqs; p.status = c->status;
  p.q = q; p.out = out; p.lse = lse;
  p.counters = (int *)((char *)c->workspace + l.counters);
  p.pieces = (float *)((char *)c->workspace + l.pieces);
  p.page_bytes = c->page_stride * esize; p.slot_bytes = c->slot_stride * esize; p.head_bytes = c->head_stride * esize; p.q_stride = q_stride;
  p.n = n; p.n_new = n_new; p.H = n_heads; p.Hkv = c->n_kv_heads; p.layer = layer;
  p.page.set(c->page_size); p.group_of.set(p.group);
  p.n_pages = c->n_pages; p.max_pages = c->max_pages; p.max_seqs = c->max_seqs;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.wait_limit = paged::wait_limit.load(std::memory_order_relaxed);
  int status = OURO_OK;
  if (p.rows > MMA_ROWS && paged::attention_tc(c, p, (cudaStream_t)stream, &status)) return status;
  // The copy engine fetches 16 rows of a head at a time: where pages are multiples of that.
  Maps maps{};
  const bool tma = c->dtype == OURO_BF16 && c->page_size % 16 == 0 && paged::make_map(&maps.k, c, c->k, 16) && paged::make_map(&maps.v, c, c->v, 16);
  switch (c->head_dim) {
    case 32: return by_kind<32>(c, p, tma, maps, cost * n, (cudaStream_t)stream);
    case 64: return by_kind<64>(c, p, tma, maps, cost * n, (cudaStream_t)stream);
    case 96: return by_kind<96>(c, p, tma, maps, cost * n, (cudaStream_t)stream);
    default: return by_kind<128>(c, p, tma, maps, cost * n, (cudaStream_t)stream);
  }
}
