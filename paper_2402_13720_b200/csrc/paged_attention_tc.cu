// Attention of several newest tokens over a paged cache (more than 16 query rows to a kv head): tcgen05 with TMEM accumulators.
//
// mma.sync tiles of 16 rows read every key from L2 and shared memory once per 16 rows, and a step of 16 keys takes a warp two thousand cycles
// whatever it does (128 rows behind 8 x 4096 keys of the 70B shape: 153 us for 21 us of keys and values, here 48).  Here a tile has up to 128 query rows
// (new tokens x query heads of a group), one TMEM lane each:
//     S = Q K^T    128 x 64 keys, two buffers in TMEM; Q lies in TMEM as well;
//     P            two threads per row, half of the keys each: S comes into their registers, and all that they exchange is whether a maximum grew;
//                  P goes back to TMEM as two bf16 parts (P = hi + lo up to 2^-17, see paged_attention.cu), two buffers;
//     O += P V     accumulates in TMEM over the units of an item.  It is rescaled only where a row's maximum grew by 2^8, so that nearly always
//                  nothing waits for it; V is the MN-major operand and is never transposed.
// 48 sequences of the 70B shape, up to 12345 tokens, 5 new: 213 us for 170 us of keys and values.  When it took 228, it took 334 with Q and P in shared
// memory, where a contraction waits for 8 KB of operands, and 214 with units of 128 keys, which cost 96 sequences of 5 tokens 40 % and 34B drafts 10 %.
// Warps 0-7 are the rows, warp 8 fetches (TMA straight from the pages, a box of 16, 32 or 64 rows of a page), warp 9 issues the contractions: the
// scores of a unit before the P V of the one before it, so that the row threads always have scores to work on.  Warp 10 sees to the units at a
// sequence's end before they are contracted.  Items, runs, pieces and their join are those of paged_attention.cu (paged_runs.cuh).
#include <cuda.h>

#include "paged_runs.cuh"

namespace {

using paged::AttnParams;
using paged::Walk;

constexpr int ROW_WARPS = 8, ROW_THREADS = 32 * ROW_WARPS, THREADS = ROW_THREADS + 96;
constexpr int KEYS = 64, HALF = KEYS / 2;          // of a unit, of a thread
// us with runs from 2 (borders taken within 1), 3 (2) and 5 units on: 34B drafts (with an earlier join) 20.1, 20.7, 21.5; 64 ragged up to 300 with 5 tokens (70B shape) 31.8, 30.0, 32.4;
// one sequence of 300 (34B) 11.5, 10.6, 10.7; large calls the same.
constexpr int ITEM_COST = 4;                       // what an item costs besides its units (filling and draining the chain), in units
constexpr int SNAP = 2;                            // units in front of or behind a cut for which it is not worth its join
constexpr int MIN_RUN = 3;                         // units for which another CTA is
constexpr int R = 128;                             // query rows of a tile
typedef paged::Runs<KEYS, ITEM_COST, SNAP, MIN_RUN> Share;
constexpr float GROWTH = 8.f;                      // (log2) a maximum may grow by this before sums and outputs are rescaled
constexpr uint32_t DRAIN_POLLS = 1u << 20;         // for copies and contractions under way when their warp is done: they end by themselves
constexpr int MAX_STAGES = 8, ODD_SLOTS = 16;      // (who looks at the ends of sequences is a ring ahead of the rows at most)

struct Maps {
  CUtensorMap k, v;                                // (dim, head, row, page, layer); boxes of 64 dims x box_rows rows
};

template <int D>
struct Cfg {
  static constexpr int BOXES = D / 64;
  static constexpr int KV_BOX = KEYS * 128;                        // bytes of 64 dims of all keys, 128-byte swizzle
  static constexpr int STAGE = 2 * BOXES * KV_BOX;                 // K, then V: [box of 64 dims][key][128 bytes]
  static constexpr int STAGES = D == 64 ? 8 : 6;                   // (a stage is taken from the request to the end of P V, some three microseconds)
  static constexpr int OFF_RING = 0;
  static constexpr int OFF_LEN = STAGES * STAGE;
  static constexpr int OFF_CUM = OFF_LEN + OURO_MAX_LIST * 4;
  static constexpr int OFF_X = OFF_CUM + (OURO_MAX_LIST + 2) * 4;  // [half][row]: what two threads of a row exchange
  static constexpr int OFF_MISC = OFF_X + 2 * R * 4;
  static constexpr int BYTES = OFF_MISC + 512;
  // TMEM columns: two buffers of S, O, Q (two dims a column), two buffers of P (hi and lo, two keys a column)
  static constexpr int O_COL = 2 * KEYS, Q_COL = O_COL + 128, P_COL = Q_COL + 64;
  static constexpr uint32_t COLS = 512;
  static_assert(STAGES <= MAX_STAGES && R <= paged::TC_ROWS && BYTES <= 227 * 1024, "");
};

struct Misc {
  uint64_t full[MAX_STAGES], empty[MAX_STAGES], s_full[2], s_free[2], p_full[2], pv_done[2], fixed[MAX_STAGES], q_full, drained;
  uint32_t tmem;
  int sums[THREADS / 32];
  int dead;                                        // a wait gave up: nobody issues or waits any more
  int odd[ODD_SLOTS];                             // [item mod ..]: values of the newest tokens that are no finite numbers were taken out
  uint32_t there[MAX_STAGES];                               // blocks of 16 keys of a stage that are on pages
};
static_assert(sizeof(Misc) <= 512, "");

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint64_t *bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory"); }
__device__ __forceinline__ void mbar_expect(uint64_t *bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t *bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory"); }
__device__ __forceinline__ bool mbar_test(uint64_t *bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait for the phase-th completion (from 0).  Whoever gives up raises the cache's status; then nobody in the CTA issues or waits any more, and the
// call ends with wrong results and an error.  (The loop is out of line: 48 sequences of up to 12345, 5 new, 213 us, at every wait 219; 34B drafts 16.3, 16.7.)
__device__ __noinline__ void mbar_wait_on(uint64_t *bar, uint32_t phase, Misc *ms, uint32_t limit, int *status) {
  for (uint32_t i = 0; i < limit; ++i)
    if (mbar_test(bar, phase & 1) || ((i & 63) == 63 && *(volatile int *)&ms->dead)) return;
  *(volatile int *)&ms->dead = 1;
  atomicCAS(status, OURO_OK, OURO_ETIMEOUT);
}
__device__ __forceinline__ void mbar_wait(uint64_t *bar, uint32_t phase, Misc *ms, const AttnParams &p) {
  if (!mbar_test(bar, phase & 1)) mbar_wait_on(bar, phase, ms, p.wait_limit, p.status);
}
__device__ __forceinline__ void warp_wait(uint64_t *bar, uint32_t phase, Misc *ms, const AttnParams &p) {
  mbar_wait(bar, phase, ms, p);
  __syncwarp();
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int dim, int head, int row, int page, int layer) {
  // (read once: evict first)
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5, %6, %7}], [%2], %8;" ::"r"(dst),
      "l"(map), "r"(smem_u32(bar)), "r"(dim), "r"(head), "r"(row), "r"(page), "r"(layer), "l"(0x12F0000000000000ull)
      : "memory");
}
// K-major operand in 128-byte swizzle: rows of 128 bytes, 8-row groups 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// MN-major operand in 128-byte swizzle: 64 dims per 128-byte row, 8 keys per 1024 bytes, the next 64 dims `box` bytes further.
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr, uint32_t box) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(box >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// fp32 += bf16 x bf16, 128 x n; mn: the B operand is MN-major
__host__ __device__ constexpr uint32_t idesc(uint32_t n, uint32_t mn) { return (1u << 4) | (1u << 7) | (1u << 10) | (mn << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24); }
// The A operand lies in TMEM: a lane per row, two values of K a column.
__device__ __forceinline__ void mma_bf16(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(id), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t *bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float *v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
               : "r"(addr));
}
// Waits for the loads issued so far; the registers are tied to it, so that their uses stay behind it.
__device__ __forceinline__ void tmem_ld_wait32(float *v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const float *v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::
                   "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]), "f"(v[22]), "f"(v[23]), "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31]), "r"(addr)
               : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t *v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::
                   "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(addr)
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void rows_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(ROW_THREADS) : "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&t);
}
// Whether anybody of the two warps that share rows (32 lanes of TMEM) says so.
__device__ __forceinline__ bool pair_or(int quarter, bool x) {
  uint32_t y;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %1, 0;\n\tbarrier.cta.red.or.pred p, %2, 64, q;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(y) : "r"((int)x), "r"(2 + quarter) : "memory");
  return y != 0;
}
__device__ __forceinline__ void pair_barrier(int quarter) { asm volatile("bar.sync %0, 64;" ::"r"(2 + quarter) : "memory"); }
__device__ __forceinline__ u64 pair(float a, float b) {
  u64 y;
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ void unpair(u64 x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ u64 add2(u64 a, u64 b) {
  u64 y;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) {
  u64 y;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ bool odd_pair(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }   // not finite

template <int D>
__global__ void __launch_bounds__(THREADS, 1) paged_attention_tc_kernel(const AttnParams p, const __grid_constant__ Maps maps, const int box_rows) {
  using C = Cfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  Misc *ms = reinterpret_cast<Misc *>(smem + C::OFF_MISC);
  const uint32_t sm = smem_u32(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < MAX_STAGES; ++i) {
      mbar_init(&ms->full[i], 1);
      mbar_init(&ms->empty[i], 2);                 // the contractions' commit, and warp 10: nobody may be a ring behind
      mbar_init(&ms->fixed[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ms->s_full[i], 1);
      mbar_init(&ms->s_free[i], ROW_WARPS);
      mbar_init(&ms->p_full[i], ROW_WARPS);
      mbar_init(&ms->pv_done[i], 1);
    }
    mbar_init(&ms->q_full, ROW_WARPS);
    mbar_init(&ms->drained, 1);
    for (int i = 0; i < ODD_SLOTS; ++i) ms->odd[i] = 0;
    ms->dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.v) : "memory");
  }
  if (warp == ROW_WARPS + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ms->tmem)), "r"(C::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  pdl_trigger();
  fence_before_sync();
  const Share runs(p, gridDim.x, (int *)(smem + C::OFF_LEN), (int *)(smem + C::OFF_CUM), ms->sums, THREADS);   // (two barriers)
  fence_after_sync();
  const uint32_t tmem = ms->tmem;
  const bool any = blockIdx.x < runs.G;
  const Walk begin = runs.place(any ? blockIdx.x : 0), end = runs.place(any ? blockIdx.x + 1 : 0);
  volatile int *dead = &ms->dead;
  // Units with rows behind the sequence's end, or with keys of the newest tokens that earlier ones do not see.
  auto at_tail = [&](const Walk &w) { return w.len - w.tile * KEYS < KEYS + p.n_new - 1; };

  if (!paged::same(begin, end)) {
    if (warp == ROW_WARPS) {
      // ================================================================ fetching
      Walk c = begin;
      int ids = -1, ids_tile = 0, ids_seq = -1;                    // page of the first of 16 keys, for 4 blocks of 8 units, one a lane
      int stage = 0, round = 0;
      for (; !paged::same(c, end); runs.next(c)) {
        if (c.s != ids_seq || c.tile < ids_tile || c.tile >= ids_tile + 8) {
          ids_seq = c.s;
          ids_tile = c.tile;
          const int key = c.tile * KEYS + lane * 16;
          ids = key < c.len ? c.row[key < c.len ? p.page.quot(key) : 0] : -1;
        }
        if (round > 0) warp_wait(&ms->empty[stage], round - 1, ms, p);
        if (__any_sync(0xffffffffu, *dead)) break;                 // (the same for the warp: it shuffles and elects from here on)
        const int blocks = min(4, (c.len - c.tile * KEYS + 15) / 16);    // with keys of the sequence
        const int mine = __shfl_sync(0xffffffffu, ids, (c.tile - ids_tile) * 4 + (lane & 3));
        const bool on = (lane & 3) < blocks && mine >= 0 && mine < p.n_pages;
        const uint32_t there = __ballot_sync(0xffffffffu, on) & 15u;
        const int id0 = on ? mine : p.n_pages;                     // beyond the pool: zeros, nothing is read
        if (elect_one()) ms->there[stage] = there;
        __syncwarp();
        const int step = box_rows / 16;                            // blocks in a box, all on one page
        const int boxes = blocks <= 0 ? 0 : (blocks + step - 1) / step;
        if (elect_one()) mbar_expect(&ms->full[stage], boxes * step * 16 * 128 * 2 * C::BOXES);
        __syncwarp();
        for (int b = 0; b < 4; b += step) {
          const int page = __shfl_sync(0xffffffffu, id0, b);
          if (b < blocks && elect_one()) {
            const int key = c.tile * KEYS + b * 16, row = key - p.page.quot(key) * (int)p.page.d;
            const uint32_t dst = sm + C::OFF_RING + stage * C::STAGE + b * 16 * 128;
#pragma unroll
            for (int x = 0; x < C::BOXES; ++x) {
              tma_load(dst + x * C::KV_BOX, &maps.k, &ms->full[stage], x * 64, c.head, row, page, p.layer);
              tma_load(dst + (C::BOXES + x) * C::KV_BOX, &maps.v, &ms->full[stage], x * 64, c.head, row, page, p.layer);
            }
          }
          __syncwarp();
        }
        if (++stage == C::STAGES) stage = 0, ++round;
      }
      // Nobody else is sure to wait for the copies under way once a wait has given up, so their last phases are waited for here.
      for (int i = 0; i < C::STAGES; ++i)
        if (round > 0 || i < stage)
          for (uint32_t j = 0; j < DRAIN_POLLS && !mbar_test(&ms->full[i], (round - (i >= stage)) & 1); ++j) {}
    } else if (warp == ROW_WARPS + 1) {
      // ================================================================ contractions, one thread
      if (elect_one()) {
        Walk c = begin;
        int stage = 0, round = 0, was_stage = 0;
        uint32_t u = 0, items = 0, fixes = 0;                      // (fixes: a bit per stage, the phase of its `fixed`)
        bool fresh = true, was_fresh = true;
        const uint64_t k0 = desc_k(sm + C::OFF_RING), v0 = desc_mn(sm + C::OFF_RING + C::BOXES * C::KV_BOX, C::KV_BOX);
        auto pv = [&](uint32_t v, int st, bool first) {            // O of unit v's item (+)= P V
          mbar_wait(&ms->p_full[v & 1], v >> 1, ms, p);
          fence_after_sync();
          if (*dead) return;
          const uint64_t b = v0 + ((uint32_t)(st * C::STAGE) >> 4);
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int kk = 0; kk < KEYS / 16; ++kk)
              mma_bf16(tmem + C::O_COL, tmem + C::P_COL + (v & 1) * KEYS + part * HALF + kk * 8, b + ((kk * 2048) >> 4), idesc(D, 1), !(first && part == 0 && kk == 0));
          mma_commit(&ms->pv_done[v & 1]);
          mma_commit(&ms->empty[st]);
        };
        for (; !paged::same(c, end); ++u) {
          if (fresh && u > 0) pv(u - 1, was_stage, was_fresh);     // (the rows ask for it before they bring the next queries)
          if (fresh) mbar_wait(&ms->q_full, items++, ms, p);
          if (at_tail(c)) {
            mbar_wait(&ms->fixed[stage], fixes >> stage & 1, ms, p);
            fixes ^= 1u << stage;
          } else {
            mbar_wait(&ms->full[stage], round, ms, p);
          }
          if (u >= 2) mbar_wait(&ms->s_free[u & 1], (u - 2) >> 1, ms, p);
          fence_after_sync();
          if (!*dead) {
            const uint64_t b = k0 + ((uint32_t)(stage * C::STAGE) >> 4);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
              mma_bf16(tmem + (u & 1) * KEYS, tmem + C::Q_COL + ks * 8, b + (((ks >> 2) * C::KV_BOX + (ks & 3) * 32) >> 4), idesc(KEYS, 0), ks > 0);
            mma_commit(&ms->s_full[u & 1]);
          }
          if (!fresh) pv(u - 1, was_stage, was_fresh);
          was_stage = stage;
          was_fresh = fresh;
          fresh = c.tile == c.tiles - 1;
          runs.next(c);
          if (++stage == C::STAGES) stage = 0, ++round;
        }
        pv(u - 1, was_stage, was_fresh);
        mma_commit(&ms->drained);                                  // (the same for the contractions)
        for (uint32_t j = 0; j < DRAIN_POLLS && !mbar_test(&ms->drained, 0); ++j) {}
      }
    } else if (warp == ROW_WARPS + 2) {
      // ================================================================ units at a sequence's end
      Walk c = begin;
      int stage = 0, round = 0, item = 0;
      for (; !paged::same(c, end); runs.next(c)) {
        // (Of every unit, and each is given back here too: a phase's parity tells no more than two apart, so this warp may be neither ahead of
        // `full` nor lapped by it.)
        warp_wait(&ms->full[stage], round, ms, p);
        if (at_tail(c)) {
          const int rest = c.len - c.tile * KEYS;                  // keys of the sequence from here on
          uint8_t *vp = smem + C::OFF_RING + stage * C::STAGE + C::BOXES * C::KV_BOX;
          // Keys of the newest tokens, hidden from earlier ones: 0 times their values must be 0, so what is not finite is taken out here and
          // put in again, for the rows that see it, at the item's end.
          bool odd = false;
          for (int e = lane; e < (p.n_new - 1) * 8 * C::BOXES; e += 32) {
            const int key = rest - 1 - (e >> 3) / C::BOXES;
            if (key < 0 || key >= KEYS) continue;
            uint4 *at = (uint4 *)(vp + ((e >> 3) % C::BOXES) * C::KV_BOX + key * 128 + (e & 7) * 16);
            const uint4 x = *at;
            uint32_t w[4] = {x.x, x.y, x.z, x.w};
            bool here = false;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (odd_pair(w[i])) {
                here = true;
                if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
                if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0xffffu;
              }
            if (here) *at = make_uint4(w[0], w[1], w[2], w[3]);
            odd |= here;
          }
          if (__any_sync(0xffffffffu, odd) && lane == 0) *(volatile int *)&ms->odd[item & (ODD_SLOTS - 1)] = 1;
          // no keys, or another sequence's rows
          for (int e = lane; e < (KEYS - min(KEYS, max(rest, 0))) * 8 * C::BOXES; e += 32)
            *(uint4 *)(vp + ((e >> 3) % C::BOXES) * C::KV_BOX + (KEYS - 1 - (e >> 3) / C::BOXES) * 128 + (e & 7) * 16) = make_uint4(0, 0, 0, 0);
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ms->fixed[stage]);
        }
        if (lane == 0) mbar_arrive(&ms->empty[stage]);
        item += c.tile == c.tiles - 1;
        if (++stage == C::STAGES) stage = 0, ++round;
      }
    } else {
      // ================================================================ rows
      Walk c = begin;
      uint32_t u = 0;
      int stage = 0, items = 0;
      const int quarter = warp & 3, half = warp >> 2, r = quarter * 32 + lane;
      const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
      float *xs = (float *)(smem + C::OFF_X);
      // The queries of an item's rows, which it needs from its first unit on: brought as soon as the scores of the item before are done.
      auto bring = [&](const Walk &w) {
        const int n = min(R, p.rows - w.rt * R), at = w.rt * R + min(r, n - 1), tok = p.group_of.quot(at), head = w.head * p.group + at - tok * p.group;
        if (quarter * 32 < n) {
          const uint4 *src = (const uint4 *)((const __nv_bfloat16 *)p.q + ((int64_t)w.s * p.n_new + tok) * p.q_stride + (int64_t)head * D) + half * (D / 16);
#pragma unroll
          for (int j = 0; j < D / 16; j += 4) {                    // 32 dims, 16 columns
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint4 x = src[j + i];
              w[4 * i] = x.x;
              w[4 * i + 1] = x.y;
              w[4 * i + 2] = x.z;
              w[4 * i + 3] = x.w;
            }
            tmem_st16(lanes + C::Q_COL + half * (D / 4) + j * 4, w);
          }
          tmem_st_wait();
        }
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ms->q_full);
      };
      bring(c);
      while (!paged::same(c, end)) {
        const Walk item = c;
        const int rt = c.rt, kvh = c.head, rows = min(R, p.rows - rt * R);
        const bool on = quarter * 32 < rows, mine = r < rows;      // the warp has rows; this thread has one
        const int at = rt * R + min(r, rows - 1), tok = p.group_of.quot(at), head = kvh * p.group + at - tok * p.group;
        const int vis = c.len - p.n_new + 1 + tok;
        const int64_t row = (int64_t)c.s * p.n_new + tok;
        float m = -INFINITY, l = 0.f;
        bool item_ends = false;
        for (bool first = true;; first = false) {
          const int b = u & 1, key0 = c.tile * KEYS;
          warp_wait(&ms->s_full[b], u >> 1, ms, p);
          fence_after_sync();
          float s[HALF];
          if (on) {
            tmem_ld32(lanes + b * KEYS + half * HALF, s);
            tmem_ld_wait32(s);
          }
          fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ms->s_free[b]);
          if (on) {
            const uint32_t there = *(volatile uint32_t *)&ms->there[stage];
            if (there != 15u || key0 + KEYS > c.len - p.n_new + 1) {   // (uniform) not every row sees every key
              const int n = vis - key0 - half * HALF;
#pragma unroll
              for (int i = 0; i < HALF; ++i)
                if (i >= n || !(there >> (half * 2 + i / 16) & 1)) s[i] = -INFINITY;
            }
            float mx = max3(s[0], s[1], s[2]), my = max3(s[3], s[4], s[5]);
#pragma unroll
            for (int i = 6; i + 3 < HALF; i += 4) {
              mx = max3(mx, s[i], s[i + 1]);
              my = max3(my, s[i + 2], s[i + 3]);
            }
            mx = max3(mx, s[HALF - 2], s[HALF - 1]);
            float top = fmaxf(mx, my) * p.scale_log2;
            if (pair_or(quarter, mine && top > m + GROWTH)) {       // (rare) the two halves agree on the rows' new maxima
              xs[half * R + r] = top;
              pair_barrier(quarter);
              top = fmaxf(top, xs[(half ^ 1) * R + r]);
              const bool grown = top > m + GROWTH;
              const float a = grown ? ex2(m - top) : 1.f;
              if (grown) {
                m = top;
                l *= a;
              }
              if (!first) {
                warp_wait(&ms->pv_done[(u - 1) & 1], (u - 1) >> 1, ms, p);
                fence_after_sync();
#pragma unroll
                for (int x = 0; x < D / 2; x += 32) {
                  float o[32];
                  tmem_ld32(lanes + C::O_COL + half * (D / 2) + x, o);
                  tmem_ld_wait32(o);
#pragma unroll
                  for (int i = 0; i < 32; ++i) o[i] *= a;
                  tmem_st32(lanes + C::O_COL + half * (D / 2) + x, o);
                }
                tmem_st_wait();
              }
              pair_barrier(quarter);                               // (both have read)
            }
            const float base = -base_of(m);
            const u64 base2 = pair(base, base), scale2 = pair(p.scale_log2, p.scale_log2);
            u64 sum = pair(0.f, 0.f);
            uint32_t hi[HALF / 2], lo[HALF / 2];
#pragma unroll
            for (int i = 0; i < HALF; i += 2) {
              float x, y;
              unpair(fma2(pair(s[i], s[i + 1]), scale2, base2), x, y);
              x = ex2(x);
              y = ex2(y);
              const u64 e = pair(x, y);
              sum = add2(sum, e);
              const uint32_t h = pack(x, y);
              unpair(add2(e, pair(-__uint_as_float(h << 16), -__uint_as_float(h & 0xffff0000u))), x, y);
              hi[i / 2] = h;
              lo[i / 2] = pack(x, y);
            }
            float s0, s1;
            unpair(sum, s0, s1);
            l += s0 + s1;
            if (u >= 2) {                                          // (the buffer has been read)
              warp_wait(&ms->pv_done[b], (u - 2) >> 1, ms, p);
              fence_after_sync();
            }
            tmem_st16(lanes + C::P_COL + b * KEYS + half * (HALF / 2), hi);
            tmem_st16(lanes + C::P_COL + b * KEYS + HALF + half * (HALF / 2), lo);
            tmem_st_wait();
          }
          fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ms->p_full[b]);
          ++u;
          if (++stage == C::STAGES) stage = 0;
          item_ends = c.tile == c.tiles - 1;
          runs.next(c);
          if (item_ends || paged::same(c, end)) break;
        }
        // ---- the item's or the run's end
        if (!paged::same(c, end)) bring(c);
        warp_wait(&ms->pv_done[(u - 1) & 1], (u - 1) >> 1, ms, p);
        fence_after_sync();
        const bool whole = item_ends && item.tile == 0;
        const int slot = item.tile == 0 ? 1 : 0;                   // pieces of a CTA: of an item it begins, of one it goes on with
        float *mls = p.pieces + (int64_t)paged::TC_CTAS * 2 * R * D;
        auto put = [&](int64_t to, int col, float inv, const float *o) {       // four columns of a row to the output
          *(uint2 *)((__nv_bfloat16 *)p.out + to * D + col) = make_uint2(pack(o[0] * inv, o[1] * inv), pack(o[2] * inv, o[3] * inv));
        };
        auto put_lse = [&](int64_t to, float M, float L) {
          if (p.lse) p.lse[to] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
        };
        if (on) {
          xs[half * R + r] = l;                                    // (in the same order for both)
          pair_barrier(quarter);
          l = xs[r] + xs[R + r];
          const int64_t to = row * p.H + head, piece = ((int64_t)blockIdx.x * 2 + slot) * R + r;
          const float inv = l == 0.f ? 0.f : 1.f / l;
          const bool odd = item_ends && *(volatile int *)&ms->odd[items & (ODD_SLOTS - 1)];
#pragma unroll
          for (int x0 = 0; x0 < D / 2; x0 += 32) {
            const int x = half * (D / 2) + x0;
            float o[32];
            tmem_ld32(lanes + C::O_COL + x, o);
            tmem_ld_wait32(o);
            if (odd && mine)                                       // what the newest tokens' values have that is not finite (rare)
              for (int key = max(0, item.len - p.n_new + 1); key < vis; ++key) {
                const int pg = p.page.quot(key), id = item.row[pg];
                if (id < 0 || id >= p.n_pages) continue;
                const __nv_bfloat16 *src = (const __nv_bfloat16 *)(p.v + (int64_t)id * p.page_bytes + (int64_t)(key - pg * (int)p.page.d) * p.slot_bytes +
                                                                   (int64_t)kvh * p.head_bytes) + x;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  const float y = __bfloat162float(src[i]);
                  if (!(fabsf(y) < INFINITY)) o[i] += y;
                }
              }
            if (mine) {
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                if (whole) put(to, x + i, inv, o + i);
                else __stcg((float4 *)(p.pieces + piece * D + x + i), make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]));
              }
            }
          }
          if (mine && half == 0) {
            if (whole) put_lse(to, m, l);
            else __stcg((float2 *)(mls + piece * 2), make_float2(m, l));
          }
          pair_barrier(quarter);                                   // (both have read)
        }
        fence_before_sync();
        if (item_ends) {
          rows_barrier();                                          // (everybody has looked)
          if (tid == 0) *(volatile int *)&ms->odd[items & (ODD_SLOTS - 1)] = 0;
          rows_barrier();
          ++items;
        }
      }
    }
  }
  fence_before_sync();
  __syncthreads();
  if (warp == ROW_WARPS + 1) {
    fence_after_sync();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::COLS));
  }
}

// The items that are cut, by the border of the first two runs that share one: its pieces are added up in ascending order.  One launch more, but
// on all SMs and behind the end of the kernel in front; by the CTA that was last to leave a piece it took 10 us and more (35 rows of D = 128 in 13
// pieces).  The rows of an item are shared by gridDim.y CTAs.
// (Every warp works out the runs and the item's CTAs, which is most of what few pieces cost.  us with 8 slices of 256 threads, 4 of 256, 8 of 128, 4 of 128,
// 16 of 64: 34B drafts 18.1, 16.3, 16.6, 17.7, 16.6; 64 ragged up to 300, 70B shape, 29.7, 28.0, 27.2, 26.7, 27.6; 8 of 4096 with 16 new tokens 47.2, 45.8,
// 44.6, 47.8, 45.2.)
constexpr int JOIN_THREADS = 128, JOIN_SLICES = 8;
// Pieces whose sums and outputs are asked for at once.  us with 2, 3, 4: 34B drafts 17.0, 16.5, 16.7; one of 30000 (70B shape) 41.3, 39.4, 40.5; 64 ragged up
// to 300 27.2 each.  (All maxima first, then the outputs: some 2 us more.)
constexpr int BATCH = 3;
template <int D>
__global__ void __launch_bounds__(JOIN_THREADS) paged_join_kernel(const AttnParams p, const int grid) {
  __shared__ int s_len[OURO_MAX_LIST], s_cum[OURO_MAX_LIST + 1], s_sums[JOIN_THREADS / 32];
  __shared__ float s_part[6][JOIN_THREADS];
  const int tid = threadIdx.x;
  pdl_trigger();
  // (the lengths were there before the kernel in front began)
  const Share runs(p, grid, s_len, s_cum, s_sums, JOIN_THREADS);
  const int c = blockIdx.x + 1;
  bool on = c < runs.G;
  const Walk w = runs.place(on ? c : 0);
  int c0 = 0, c1 = 0;
  on = on && w.s < p.n && w.tile > 0;
  if (on) {
    runs.owners(w, c0, c1);
    on = c == c0 + 1;
  }
  const int rows = min(R, p.rows - w.rt * R), r0 = rows * blockIdx.y / JOIN_SLICES, r1 = rows * (blockIdx.y + 1) / JOIN_SLICES;
  pdl_wait();
  constexpr int C4 = D / 4;                        // columns of four a row
  const int E = (r1 - r0) * C4;
  if (!on || E == 0) return;
  // A thread has four columns of a row, and where that leaves threads over every so manieth piece.
  const float *mls = p.pieces + (int64_t)paged::TC_CTAS * 2 * R * D;
  auto where = [&](int cta) { return ((int64_t)cta * 2 + (cta == c0 ? 1 : 0)) * R; };
  const int shares = E < JOIN_THREADS ? JOIN_THREADS / E : 1, share = shares > 1 ? tid / E : 0;
  for (int e0 = 0; e0 < E; e0 += JOIN_THREADS) {
    const int e = min(e0 + tid - share * E, E - 1), r = r0 + e / C4, col = e % C4 * 4;
    float M = -INFINITY, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    auto rescale = [&](float mx) {
      const float a = ex2(M - base_of(mx));
      M = mx;
      L *= a;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= a;
    };
    for (int j0 = c0 + share; j0 <= c1; j0 += BATCH * shares) {    // sums and outputs of BATCH pieces are asked for at once
      float2 ml[BATCH];
      float4 y[BATCH];
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const int64_t at = where(min(j0 + b * shares, c1)) + r;
        ml[b] = __ldcg((const float2 *)(mls + at * 2));
        y[b] = __ldcg((const float4 *)(p.pieces + at * D + col));
      }
      float mx = M;
#pragma unroll
      for (int b = 0; b < BATCH; ++b) mx = fmaxf(mx, ml[b].x);     // (a piece twice changes no maximum)
      rescale(mx);
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        if (j0 + b * shares > c1) continue;
        const float x = ex2(ml[b].x - base_of(mx));
        L = fmaf(x, ml[b].y, L);
        o[0] = fmaf(x, y[b].x, o[0]);
        o[1] = fmaf(x, y[b].y, o[1]);
        o[2] = fmaf(x, y[b].z, o[2]);
        o[3] = fmaf(x, y[b].w, o[3]);
      }
    }
    if (shares > 1) {
      s_part[0][tid] = L;
#pragma unroll
      for (int i = 0; i < 4; ++i) s_part[i + 1][tid] = o[i];
      s_part[5][tid] = M;
      __syncthreads();
      if (share == 0) {
        float mx = M;
        for (int k = 1; k < shares; ++k) mx = fmaxf(mx, s_part[5][k * E + tid]);
        rescale(mx);
        for (int k = 1; k < shares; ++k) {
          const float x = ex2(s_part[5][k * E + tid] - base_of(mx));
          L = fmaf(x, s_part[0][k * E + tid], L);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = fmaf(x, s_part[i + 1][k * E + tid], o[i]);
        }
      }
    }
    if (share == 0 && e0 + tid < E) {
      const int at = w.rt * R + r, tok = p.group_of.quot(at);
      const int64_t to = ((int64_t)w.s * p.n_new + tok) * p.H + w.head * p.group + at - tok * p.group;
      const float inv = L == 0.f ? 0.f : 1.f / L;
      *(uint2 *)((__nv_bfloat16 *)p.out + to * D + col) = make_uint2(pack(o[0] * inv, o[1] * inv), pack(o[2] * inv, o[3] * inv));
      if (p.lse && col == 0) p.lse[to] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
    }
  }
}

const char *CALL = "ouro_paged_attention";

template <int D>
int launch(const ouro_paged_cache *c, AttnParams p, const Maps &maps, int box_rows, cudaStream_t s) {
  using C = Cfg<D>;
  static bool ready[paged::MAX_DEVICES] = {};
  int dev = 0, sms = 0;
  if (!paged::device(&dev, &sms)) return paged::refuse(CALL, "no usable current device", OURO_ECUDA);
  if (!ready[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(paged_attention_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::BYTES);
    if (e != cudaSuccess) return paged::refuse(CALL, cudaGetErrorString(e), OURO_ECUDA);
    ready[dev] = true;
  }
  p.row_tiles = (p.rows + R - 1) / R;
  const int64_t cost = (((int64_t)p.cap + KEYS - 1) / KEYS + ITEM_COST) * c->n_kv_heads * p.row_tiles * p.n;
  const int64_t most = sms < paged::TC_CTAS ? sms : paged::TC_CTAS, want = cost / MIN_RUN;
  const int grid = (int)(want < 1 ? 1 : want < most ? want : most);
  cudaError_t e = launch_pdl(paged_attention_tc_kernel<D>, dim3(grid), dim3(THREADS), C::BYTES, s, p, maps, box_rows);
  OURO_COUNT_LAUNCH();
  if (e == cudaSuccess && grid > 1) {
    e = launch_pdl(paged_join_kernel<D>, dim3(grid - 1, JOIN_SLICES), dim3(JOIN_THREADS), 0, s, p, grid);
    OURO_COUNT_LAUNCH();
  }
  return e == cudaSuccess ? OURO_OK : paged::refuse(CALL, cudaGetErrorString(e), OURO_ECUDA);
}

}  // namespace

// 0: does not take the call (another head dim, or pages that no box fits).
int paged::attention_tc(const ouro_paged_cache *c, const paged::AttnParams &p, cudaStream_t s, int *status) {
  if (c->dtype != OURO_BF16 || (c->head_dim != 64 && c->head_dim != 128) || c->page_size % 16) return 0;
  const int box_rows = c->page_size % 64 == 0 ? 64 : c->page_size % 32 == 0 ? 32 : 16;
  Maps maps;
  if (!make_map(&maps.k, c, c->k, box_rows) || !make_map(&maps.v, c, c->v, box_rows)) return 0;
  *status = c->head_dim == 64 ? launch<64>(c, p, maps, box_rows, s) : launch<128>(c, p, maps, box_rows, s);
  return 1;
}
