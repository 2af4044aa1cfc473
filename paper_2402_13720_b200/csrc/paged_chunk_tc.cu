// Attention of chunks of new tokens over a paged cache in bf16: tcgen05 with TMEM accumulators (the formula stands in paged_chunk.cu).
//
// A CTA has an item's 256 query rows (new tokens x query heads of a group) as two tiles A and B of 128, one TMEM lane and one thread a row, and passes
// over the keys 64 at a time:
//     S = Q K^T    128 x 64 in TMEM; Q and K in shared memory;
//     P            the row's thread has all of S in its registers, so that maximum and sum need nobody else, and S is free for the next unit's scores
//                  before the exponentials are begun; P goes back to TMEM as bf16, two buffers;
//     O += P V     accumulates in TMEM.  It is rescaled only where a row's maximum grew by 2^8 (by the row's own thread), so that nearly always nothing
//                  waits for it; V is the MN-major operand and is never transposed.
// TMEM is full with that: two S of 64 columns, four P of 32, two O of 128.
// P is rounded to bf16 once.  It could go in as two bf16 parts, as it does in paged_attention_tc.cu, which is bound by memory; here that would be half as
// many contractions again.  The rounding errors of P are independent and average out as the values do: outputs are 2.2e-3 of their norm off, of which their own
// rounding is 1.7e-3.
// Warps 0-3 and 4-7 are the rows of A and B, who also bring their queries; warps 8 and 9 issue the contractions of A and of B; warp 10 fetches keys and values (TMA
// straight from the pages, boxes of 8 to 64 rows of a page); warp 11 sees to the values at a sequence's end and at the causal edge before they are contracted.
// Items, runs, pieces and their join: paged_chunk.cuh, paged_chunk.cu.
#include <cuda.h>

#include "paged_chunk.cuh"

namespace {

using paged::ChunkParams;
using paged::ChunkWalk;

constexpr int TILE = 128, R = 2 * TILE;            // query rows of a tile, of an item
constexpr int KEYS = 64;                           // of a unit
constexpr int ROW_WARPS = 8, MMA_WARP = ROW_WARPS, FETCH_WARP = MMA_WARP + 2, VALUE_WARP = FETCH_WARP + 1,
              THREADS = 32 * (VALUE_WARP + 1);
// us with an item's cost of 2, 4, 5, 6, 8 units: 1.1B shape, mixed batch 27.4, 29.1, 27.3, 27.4, 28.9; 7B shape, 2048 tokens 58.0, 55.8, 56.2, 56.8, 58.0; 34B shape, 61 behind
// 24000 56.4, 55.2, 55.6, 55.7, 55.9; 70B shape, five prompts, with pauses between them 815, 776, 778, 782, 795.
constexpr int ITEM_COST = 5, SNAP = 2, MIN_RUN = 4;
typedef paged::ChunkRuns<R, KEYS, ITEM_COST, SNAP, MIN_RUN> Share;
constexpr float GROWTH = 8.f;                      // (log2) a maximum may grow by this before sums and outputs are rescaled
// Of 32 exponentials, those that go to the special function unit, which takes 8 cycles for a warp's; the others go to the multiply-adds that wait
// meanwhile.  us with 32, 28, 24, 20, 16: 70B shape, five prompts 814, 795, 781, 792, 828; 34B shape, 61 behind 24000 62.2, 60.4, 58.3, 58.3, 61.0.
constexpr int EX2_OF_32 = 24;
constexpr uint32_t DRAIN_POLLS = 1u << 20;         // for copies and contractions under way when their warp is done: they end by themselves
constexpr int MAX_SLOTS = 12, ODD_SLOTS = 16;      // (whoever sees to the values is a ring ahead of the rows at most)

struct Maps {
  CUtensorMap k, v;                                // (dim, head, row, page, layer); boxes of 64 dims x box_rows rows
};

// D: head dims, rounded up to 64 or 128 (the copy engine fills up with zeros)
template <int D>
struct Cfg {
  static constexpr int BOXES = D / 64;
  static constexpr int Q_BOX = TILE * 128, KV_BOX = KEYS * 128;    // bytes of 64 dims of all rows or keys, 128-byte swizzle
  static constexpr int Q_TILE = BOXES * Q_BOX, SLOT = BOXES * KV_BOX;          // a tile of Q, a unit's K or V: [box of 64 dims][row][128 bytes]
  // The scores are a unit ahead of P V, and given back as soon as they are done: two more slots for values keep both as far ahead.
  static constexpr int K_SLOTS = D == 64 ? 8 : 4, V_SLOTS = K_SLOTS + 2;
  static constexpr int OFF_Q = 0, OFF_K = 2 * Q_TILE, OFF_V = OFF_K + K_SLOTS * SLOT, OFF_MISC = OFF_V + V_SLOTS * SLOT;
  static constexpr int BYTES = OFF_MISC + 1024;
  // TMEM columns: S of A and B, two P (two keys a column) of A and of B, O of A and B
  static constexpr int P_COL = 2 * KEYS, O_COL = P_COL + 2 * KEYS;
  static constexpr uint32_t COLS = 512;
  static_assert(V_SLOTS <= MAX_SLOTS && V_SLOTS < ODD_SLOTS && O_COL + 256 <= 512 && R == paged::CHUNK_TC_ROWS && BYTES <= 227 * 1024 &&
                    2 * Q_TILE >= OURO_MAX_LIST * 32, "");
};

struct Misc {
  uint64_t k_full[MAX_SLOTS], k_empty[MAX_SLOTS], v_full[MAX_SLOTS], v_ready[MAX_SLOTS], v_empty[MAX_SLOTS];
  uint64_t q_full[2], s_full[2], s_free[2], p_full[2][2], o_done[2][2], drained;           // [tile] ([buffer of P])
  ChunkWalk places[2];                             // where the run begins and ends
  uint32_t tmem;
  int dead;                                        // a wait gave up: nobody issues or waits any more
  int odd[ODD_SLOTS];                              // [part mod ..]: the last part of which values that are no finite numbers were taken out, from 1
  uint32_t there[MAX_SLOTS];                       // [slot of V] blocks of 8 keys that are on pages
};
static_assert(sizeof(Misc) <= 1024, "");

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
// call ends with wrong results and an error.
__device__ __noinline__ void mbar_wait_on(uint64_t *bar, uint32_t phase, Misc *ms, uint32_t limit, int *status) {
  for (uint32_t i = 0; i < limit; ++i)
    if (mbar_test(bar, phase & 1) || ((i & 63) == 63 && *(volatile int *)&ms->dead)) return;
  *(volatile int *)&ms->dead = 1;
  atomicCAS(status, OURO_OK, OURO_ETIMEOUT);
}
__device__ __forceinline__ void mbar_wait(uint64_t *bar, uint32_t phase, Misc *ms, const ChunkParams &p) {
  if (!mbar_test(bar, phase & 1)) mbar_wait_on(bar, phase, ms, p.wait_limit, p.status);
}
// The same for a warp together.
__device__ __forceinline__ void warp_wait(uint64_t *bar, uint32_t phase, Misc *ms, const ChunkParams &p) {
  if (!__all_sync(0xffffffffu, mbar_test(bar, phase & 1))) {
    mbar_wait_on(bar, phase, ms, p.wait_limit, p.status);
    __syncwarp();
  }
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int dim, int head, int row, int page, int layer) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
               "l"(map), "r"(smem_u32(bar)), "r"(dim), "r"(head), "r"(row), "r"(page), "r"(layer)
               : "memory");
}
// 16 bytes, or zeros where there is nothing to read
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
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
// A in shared memory, or in TMEM: a lane per row, two values of K a column.  Descriptors by their lower halves, which have the addresses.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t a_hi, uint32_t b, uint32_t b_hi, uint32_t id, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\t"
      "setp.ne.b32 p, %6, 0;\n\tmov.b64 x, {%1, %2};\n\tmov.b64 y, {%3, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %5, p;\n\t}" ::"r"(d),
      "r"(a), "r"(a_hi), "r"(b), "r"(b_hi), "r"(id), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t b_hi, uint32_t id, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\t"
      "setp.ne.b32 p, %5, 0;\n\tmov.b64 y, {%2, %3};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %4, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(b_hi), "r"(id), "r"(accumulate)
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
// 32 bytes, whole sectors: a row's thread writes its own row, and 16 bytes at a time took twice as long.
__device__ __forceinline__ void store32(void *dst, const uint32_t *v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&t);
}
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
__device__ __forceinline__ u64 mul2(u64 a, u64 b) {
  u64 y;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}
__device__ __forceinline__ float at_least(float a, float b) {       // what is no number stays none
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// 2^a and 2^b by multiply-adds: the whole part n of x comes off by rounding to it, 2^f for f in -1/2 .. 1/2 is 1 + f (c1 + f (c2 + f (c3 + f c4))), fitted here for the
// least largest relative error (2^-18.4; P keeps 8 bits of it, and a row's sum averages it), and 2^n is made of its exponent, which is that of 0 at -127 and below.
__device__ __forceinline__ u64 ex2_pair(float a, float b) {
  const u64 x = pair(at_least(a, -127.f), at_least(b, -127.f)), round = pair(12582912.f, 12582912.f), n = add2(x, round);    // (1.5 2^23)
  const u64 f = fma2(add2(n, pair(-12582912.f, -12582912.f)), pair(-1.f, -1.f), x), one = pair(1.f, 1.f);
  u64 y = fma2(f, pair(0.009582852944731712f, 0.009582852944731712f), pair(0.055906426161527634f, 0.055906426161527634f));
  y = fma2(y, f, pair(0.24024099111557007f, 0.24024099111557007f));
  y = fma2(y, f, pair(0.6931241750717163f, 0.6931241750717163f));
  y = fma2(y, f, one);
  float na, nb;
  unpair(n, na, nb);
  return mul2(y, pair(__uint_as_float((__float_as_uint(na) << 23) + 0x3f800000u), __uint_as_float((__float_as_uint(nb) << 23) + 0x3f800000u)));
}
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ bool odd_pair(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }   // not finite

// Where a run ends.
struct End {
  int s, head, rt, unit;
  __device__ __forceinline__ bool at(const ChunkWalk &w) const { return w.unit == unit && w.rt == rt && w.head == head && w.s == s; }
};

// The part of an item that lies in a run, and what each of its tiles has to do there.
struct Part {
  int first, last;                                 // units
  int rows, until_a, until_b;                      // query rows of the item; where the units end that A and B see anything of (B's tokens are later than A's)
  __device__ __forceinline__ Part(const Share &runs, const ChunkParams &p, const ChunkWalk &w, const End &end) {
    rows = min(R, w.m * p.group - w.rt * R);
    first = w.unit;
    last = w.s == end.s && w.head == end.head && w.rt == end.rt ? end.unit : w.units;
    until_a = rows > TILE ? min(last, max(1, (runs.sees(w, w.rt * R + TILE - 1) + KEYS - 1) / KEYS)) : last;
    until_b = rows > TILE ? last : 0;
  }
  __device__ __forceinline__ int until(int t) const { return t == 0 ? until_a : until_b; }
  __device__ __forceinline__ int rows_of(int t) const { return t == 0 ? min(rows, TILE) : rows - min(rows, TILE); }
};

template <int D>
__global__ void __launch_bounds__(THREADS, 1) paged_chunk_tc_kernel(const ChunkParams p, const __grid_constant__ Maps maps, const int box_rows) {
  using C = Cfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  Misc *ms = reinterpret_cast<Misc *>(smem + C::OFF_MISC);
  const uint32_t sm = smem_u32(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < MAX_SLOTS; ++i) {
      mbar_init(&ms->k_full[i], 1);
      mbar_init(&ms->k_empty[i], 2);               // both tiles
      mbar_init(&ms->v_full[i], 1);
      mbar_init(&ms->v_ready[i], 1);
      mbar_init(&ms->v_empty[i], 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ms->q_full[i], ROW_WARPS / 2);
      mbar_init(&ms->s_full[i], 1);
      mbar_init(&ms->s_free[i], ROW_WARPS / 2);
      for (int b = 0; b < 2; ++b) {
        mbar_init(&ms->p_full[i][b], ROW_WARPS / 2);
        mbar_init(&ms->o_done[i][b], 1);
      }
    }
    mbar_init(&ms->drained, 2);
    for (int i = 0; i < ODD_SLOTS; ++i) ms->odd[i] = 0;
    ms->dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.v) : "memory");
  }
  if (warp == MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ms->tmem)), "r"(C::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const Share runs(p);
  runs.touch();
  pdl_wait();
  pdl_trigger();
  fence_before_sync();
  runs.plan((int *)(smem + C::OFF_Q), (Share::Known *)(smem + C::OFF_Q) + OURO_MAX_LIST, ms->places, THREADS);         // (where the queries will be)
  fence_after_sync();
  ChunkWalk w = ms->places[0];
  const End end{ms->places[1].s, ms->places[1].head, ms->places[1].rt, ms->places[1].unit};
  if (tid == 0) p.begins[blockIdx.x] = end.at(w) ? make_int4(-1, 0, 0, 0) : make_int4(w.s, w.head, w.rt, w.unit);
  const uint32_t tmem = ms->tmem;
  volatile int *dead = &ms->dead;

  if (warp >= ROW_WARPS) {
    if (end.at(w)) {
      // (nothing to do)
    } else if (warp < FETCH_WARP) {
      // ================================================================ contractions of a tile, one thread
      if (elect_one()) {
        const int t = warp - MMA_WARP;
        uint32_t ks = 0, kph = 0, vs = 0, vph = 0;                 // slot and phase of the next keys and values
        uint32_t parts = 0, scores = 0, steps = 0;                 // of the tile: parts, Q K^T, P V
        const uint64_t q0 = desc_k(sm + C::OFF_Q + t * C::Q_TILE), k0 = desc_k(sm + C::OFF_K), v0 = desc_mn(sm + C::OFF_V, C::KV_BOX);
        const uint32_t q_lo = (uint32_t)q0, q_hi = (uint32_t)(q0 >> 32), k_lo = (uint32_t)k0, k_hi = (uint32_t)(k0 >> 32), v_lo = (uint32_t)v0, v_hi = (uint32_t)(v0 >> 32);
        const uint32_t s_at = tmem + t * KEYS, p_at = tmem + C::P_COL + t * KEYS, o_at = tmem + C::O_COL + t * 128;
        // Scores for the next keys.  Keys that the tile does not see are given back (but not before they have come: a phase's parity tells no more than two
        // apart).
        auto qk = [&](bool on, bool first) {
          mbar_wait(&ms->k_full[ks], kph, ms, p);
          if (on) {
            if (first) mbar_wait(&ms->q_full[t], parts++, ms, p);
            if (scores > 0) mbar_wait(&ms->s_free[t], scores - 1, ms, p);
            ++scores;
            fence_after_sync();
            if (!*dead) {
              const uint32_t b = k_lo + (ks * C::SLOT >> 4);
#pragma unroll
              for (int k = 0; k < D / 16; ++k)
                mma_ss(s_at, q_lo + (((k >> 2) * C::Q_BOX + (k & 3) * 32) >> 4), q_hi, b + (((k >> 2) * C::KV_BOX + (k & 3) * 32) >> 4), k_hi, idesc(KEYS, 0), k > 0);
              mma_commit(&ms->s_full[t]);
            }
          }
          mma_commit(&ms->k_empty[ks]);
          if (++ks == C::K_SLOTS) ks = 0, ++kph;
        };
        // O (+)= P V with the next values.
        auto pv = [&](bool on, bool first) {
          mbar_wait(&ms->v_ready[vs], vph, ms, p);
          if (on) {
            const uint32_t buf = steps & 1;
            mbar_wait(&ms->p_full[t][buf], steps >> 1, ms, p);     // (the rows may be a step ahead: a barrier for each buffer)
            ++steps;
            fence_after_sync();
            if (!*dead) {
              const uint32_t b = v_lo + (vs * C::SLOT >> 4);
#pragma unroll
              for (int k = 0; k < KEYS / 16; ++k) mma_ts(o_at, p_at + buf * (KEYS / 2) + k * 8, b + ((k * 2048) >> 4), v_hi, idesc(D, 1), !first || k > 0);
              mma_commit(&ms->o_done[t][buf]);
            }
          }
          mma_commit(&ms->v_empty[vs]);
          if (++vs == C::V_SLOTS) vs = 0, ++vph;
        };
        while (!end.at(w)) {
          const Part part(runs, p, w, end);
          const int until = part.until(t);
          for (int u = part.first; u <= part.last; ++u) {          // scores of a unit, P V of the one before
            if (u < part.last) qk(u < until, u == part.first);
            if (u > part.first) pv(u - 1 < until, u - 1 == part.first);
          }
          w.unit = part.last;
          if (w.unit == w.units) runs.next_item(w);
        }
        mma_commit(&ms->drained);                                  // (nobody else is sure to wait for them once a wait has given up)
        for (uint32_t j = 0; j < DRAIN_POLLS && !mbar_test(&ms->drained, 0); ++j) {}
      }
    } else if (warp == FETCH_WARP) {
      // ================================================================ fetching
      const int per = box_rows / 8;                                // blocks of 8 keys in a box, all on one page
      auto ids_of = [&](const ChunkWalk &x) {                      // page of a unit's lane-th block
        const int key = x.unit * KEYS + (lane & 7) * 8;
        return key < x.len ? x.row[p.page.quot(key)] : -1;
      };
      int ids = ids_of(w);
      uint32_t ks = 0, kph = 0, vs = 0, vph = 0;                   // slots, and how often they have been filled
      for (;;) {
        ChunkWalk nw = w;
        runs.next(nw);
        const bool more = !end.at(nw);
        const int ids_next = more ? ids_of(nw) : -1;
        if (kph > 0) warp_wait(&ms->k_empty[ks], kph - 1, ms, p);
        if (vph > 0) warp_wait(&ms->v_empty[vs], vph - 1, ms, p);
        if (__any_sync(0xffffffffu, *dead)) break;                 // (the same for the warp: it shuffles and elects from here on)
        const int blocks = min(KEYS / 8, (w.len - w.unit * KEYS + 7) / 8);     // with keys of the sequence
        const bool on = (lane & 7) < blocks && ids >= 0 && ids < p.n_pages;
        const uint32_t there = __ballot_sync(0xffffffffu, on) & 0xffu;
        const int id = on ? ids : p.n_pages;                       // beyond the pool: zeros, nothing is read
        const int boxes = blocks <= 0 ? 0 : (blocks + per - 1) / per;
        if (elect_one()) {
          ms->there[vs] = there;
          mbar_expect(&ms->k_full[ks], boxes * box_rows * 128 * C::BOXES);
          mbar_expect(&ms->v_full[vs], boxes * box_rows * 128 * C::BOXES);
        }
        __syncwarp();
#pragma unroll 1
        for (int b = 0; b < boxes; ++b) {
          const int page = __shfl_sync(0xffffffffu, id, b * per);
          if (elect_one()) {
            const int key = w.unit * KEYS + b * box_rows, row = key - p.page.quot(key) * (int)p.page.d;
#pragma unroll
            for (int x = 0; x < C::BOXES; ++x) {
              tma_load(sm + C::OFF_K + ks * C::SLOT + x * C::KV_BOX + b * box_rows * 128, &maps.k, &ms->k_full[ks], x * 64, w.head, row, page, p.layer);
              tma_load(sm + C::OFF_V + vs * C::SLOT + x * C::KV_BOX + b * box_rows * 128, &maps.v, &ms->v_full[vs], x * 64, w.head, row, page, p.layer);
            }
          }
          __syncwarp();
        }
        if (++ks == C::K_SLOTS) ks = 0, ++kph;
        if (++vs == C::V_SLOTS) vs = 0, ++vph;
        if (!more) break;
        w = nw;
        ids = ids_next;
      }
      // Nobody else is sure to wait for the copies under way once a wait has given up, so their last phases are waited for here.
      for (uint32_t i = 0; i < C::V_SLOTS; ++i) {
        if (i < C::K_SLOTS && (kph > 0 || i < ks))
          for (uint32_t j = 0; j < DRAIN_POLLS && !mbar_test(&ms->k_full[i], (kph - (i >= ks)) & 1); ++j) {}
        if (vph > 0 || i < vs)
          for (uint32_t j = 0; j < DRAIN_POLLS && !mbar_test(&ms->v_full[i], (vph - (i >= vs)) & 1); ++j) {}
      }
    } else {
      // ================================================================ values that not every row sees
      uint32_t slot = 0, phase = 0;
      int parts = 0;
      while (!end.at(w)) {
        const Part part(runs, p, w, end);
        ++parts;
        const int edge = max(0, runs.sees(w, w.rt * R));           // keys in front of it are seen by every row
        for (; w.unit < part.last; ++w.unit) {
          warp_wait(&ms->v_full[slot], phase, ms, p);
          const int key0 = w.unit * KEYS;
          if (key0 + KEYS > edge) {
            // Keys that some rows do not see: 0 times their values must be 0, so what is not finite is taken out here and put in again, for the
            // rows that see it, at the part's end.  Behind the sequence's end lie other sequences' rows, or nothing.
            // A lane has 16 bytes of every fourth key.  A number times 0 is 0, but for what is not finite.
            uint8_t *vp = smem + C::OFF_V + slot * C::SLOT + lane * 16;
            const int key = key0 + (lane >> 3);
            bool odd = false;
#pragma unroll
            for (int x = 0; x < C::BOXES; ++x) {
              uint4 v[KEYS / 4];
              __nv_bfloat162 sum = __floats2bfloat162_rn(0.f, 0.f), more = sum;
              const __nv_bfloat162 zero = sum;
#pragma unroll
              for (int i = 0; i < KEYS / 4; ++i) {
                if (key + 4 * i >= w.len) *(uint4 *)(vp + x * C::KV_BOX + i * 512) = make_uint4(0, 0, 0, 0);
                v[i] = *(const uint4 *)(vp + x * C::KV_BOX + i * 512);
              }
#pragma unroll
              for (int i = 0; i < KEYS / 4; ++i) {
                sum = __hfma2(*(const __nv_bfloat162 *)&v[i].x, zero, sum);
                more = __hfma2(*(const __nv_bfloat162 *)&v[i].y, zero, more);
                sum = __hfma2(*(const __nv_bfloat162 *)&v[i].z, zero, sum);
                more = __hfma2(*(const __nv_bfloat162 *)&v[i].w, zero, more);
              }
              sum = __hadd2(sum, more);
              if (!__any_sync(0xffffffffu, odd_pair(*(const uint32_t *)&sum))) continue;
#pragma unroll 1
              for (int i = 0; i < KEYS / 4; ++i) {                 // (rare)
                if (key + 4 * i < edge) continue;
                uint4 *at = (uint4 *)(vp + x * C::KV_BOX + i * 512);
                const uint4 y = *at;
                uint32_t z[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int c = 0; c < 4; ++c)
                  if (odd_pair(z[c])) {
                    odd = true;
                    if ((z[c] & 0x7f80u) == 0x7f80u) z[c] &= 0xffff0000u;
                    if ((z[c] & 0x7f800000u) == 0x7f800000u) z[c] &= 0xffffu;
                  }
                *at = make_uint4(z[0], z[1], z[2], z[3]);
              }
            }
            if (__any_sync(0xffffffffu, odd) && lane == 0) *(volatile int *)&ms->odd[parts % ODD_SLOTS] = parts;
            fence_async_smem();
            __syncwarp();
          }
          if (lane == 0) mbar_arrive(&ms->v_ready[slot]);
          if (++slot == C::V_SLOTS) slot = 0, ++phase;
        }
        if (__any_sync(0xffffffffu, *dead)) break;
        if (w.unit == w.units) runs.next_item(w);
      }
    }
  } else {
    // ================================================================ rows
    const int t = warp >> 2, quarter = warp & 3, r = quarter * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), s_at = lanes + t * KEYS, p_at = lanes + C::P_COL + t * KEYS, o_at = lanes + C::O_COL + t * 128;
    uint32_t steps = 0, unit0 = 0;                                 // of the tile so far; of the run, in front of the part, modulo V_SLOTS
    int parts = 0;
    // The queries of the warp's rows, 32 / PIECES rows of D / 8 pieces of 16 bytes at a time; the scores with those before are done.
    auto bring = [&](const ChunkWalk &x, int rows) {
      constexpr int PIECES = D / 8, STEP = 32 / PIECES;
      const int at = x.rt * R + t * TILE + min(r, rows - 1), tok = p.group_of.quot(at), col = lane % PIECES;
      const __nv_bfloat16 *mine = (const __nv_bfloat16 *)p.q + (int64_t)(x.start + tok) * p.q_stride + (int64_t)(x.head * p.group + at - tok * p.group) * p.head_dim;
      const uint32_t dst = sm + C::OFF_Q + t * C::Q_TILE + (col >> 3) * C::Q_BOX + quarter * 32 * 128;
#pragma unroll 4
      for (int i = 0; i < 32; i += STEP) {
        const int k = i + lane / PIECES;
        const __nv_bfloat16 *src = (const __nv_bfloat16 *)__shfl_sync(0xffffffffu, (unsigned long long)mine, k);
        const bool on = quarter * 32 + k < rows && col * 8 < p.head_dim;
        cp_async16(dst + k * 128 + (((col & 7) ^ (k & 7)) << 4), on ? src + col * 8 : p.q, on);
      }
    };
    auto brought = [&]() {
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ms->q_full[t]);
    };
    if (!end.at(w)) {
      const Part part(runs, p, w, end);
      if (part.first < part.until(t)) {
        if (quarter * 32 < part.rows_of(t)) bring(w, part.rows_of(t));
        brought();
      }
    }
    while (!end.at(w)) {
      const Part part(runs, p, w, end);
      ++parts;
      const int rows = part.rows_of(t), until = part.until(t), at0 = w.rt * R + t * TILE;
      const bool on = quarter * 32 < rows, mine = r < rows;        // the warp has rows; this thread has one
      const int at = at0 + (rows > 0 ? min(r, rows - 1) : 0);
      const int vis = runs.sees(w, at), all_see = runs.sees(w, at0);
      float m = -INFINITY, l = 0.f;
      uint32_t there_at = unit0;
      auto unit = [&](int u) {
        warp_wait(&ms->s_full[t], steps, ms, p);
        fence_after_sync();
        float s[KEYS];
        tmem_ld32(s_at, s);
        tmem_ld32(s_at + 32, s + 32);
        const uint32_t there = *(volatile uint32_t *)&ms->there[there_at];
        if (++there_at == C::V_SLOTS) there_at = 0;
        tmem_ld_wait32(s);
        tmem_ld_wait32(s + 32);
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ms->s_free[t]);
        if (there != 0xffu || u * KEYS + KEYS > all_see) {         // (uniform) not every row sees every key
#pragma unroll
          for (int x = 0; x < KEYS; x += 32) {                     // a bit for each key that the row sees
            const int ahead = min(max(vis - u * KEYS - x, 0), 32);
            const uint32_t bits = (uint32_t)((1ull << ahead) - 1) & ((((there >> (x / 8) & 15u) * 0x00204081u) & 0x01010101u) * 0xffu);
#pragma unroll
            for (int i = 0; i < 32; ++i) s[x + i] = bits >> i & 1 ? s[x + i] : -INFINITY;
          }
        }
        float mx = max3(s[0], s[1], s[2]), my = max3(s[3], s[4], s[5]);
#pragma unroll
        for (int i = 6; i + 3 < KEYS; i += 4) {
          mx = max3(mx, s[i], s[i + 1]);
          my = max3(my, s[i + 2], s[i + 3]);
        }
        mx = max3(mx, s[KEYS - 2], s[KEYS - 1]);
        const float top = fmaxf(mx, my) * p.scale_log2;
        const bool grown = top > m + GROWTH;
        if (__any_sync(0xffffffffu, grown)) {                      // (rare)
          const float a = grown ? ex2(m - top) : 1.f;
          if (grown) {
            m = top;
            l *= a;
          }
          if (u > part.first) {
            warp_wait(&ms->o_done[t][(steps - 1) & 1], (steps - 1) >> 1, ms, p);
            fence_after_sync();
#pragma unroll 1
            for (int x = 0; x < D; x += 32) {
              float o[32];
              tmem_ld32(o_at + x, o);
              tmem_ld_wait32(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] *= a;
              tmem_st32(o_at + x, o);
            }
            tmem_st_wait();
          }
        }
        const float base = -base_of(m);
        const u64 base2 = pair(base, base), scale2 = pair(p.scale_log2, p.scale_log2);
        u64 sum = pair(0.f, 0.f);
        const uint32_t buf = steps & 1;                            // (free: the scores came behind the P V that was the last to read it)
#pragma unroll
        for (int x = 0; x < KEYS; x += 32) {
          uint32_t w16[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            float a, b;
            unpair(fma2(pair(s[x + i], s[x + i + 1]), scale2, base2), a, b);
            u64 e;
            if (i < EX2_OF_32) {
              e = pair(ex2(a), ex2(b));
            } else {
              e = ex2_pair(a, b);
            }
            sum = add2(sum, e);
            unpair(e, a, b);
            w16[i / 2] = pack(a, b);
          }
          tmem_st16(p_at + buf * (KEYS / 2) + x / 2, w16);
        }
        tmem_st_wait();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ms->p_full[t][buf]);
        ++steps;
        float s0, s1;
        unpair(sum, s0, s1);
        l += s0 + s1;
      };
      if (on) {
#pragma unroll 1
        for (int u = part.first; u < until; ++u) unit(u);
      } else {
        for (int u = part.first; u < until; ++u, ++steps) {
          warp_wait(&ms->s_full[t], steps, ms, p);
          if (lane == 0) {
            mbar_arrive(&ms->s_free[t]);
            mbar_arrive(&ms->p_full[t][steps & 1]);
          }
        }
      }
      unit0 = (unit0 + part.last - part.first) % C::V_SLOTS;
      // ---- the part's end: the next one's queries, and the outputs
      // (Asked for when the last scores with these are there, they cost the 70B shape's prompts 4 %.)
      ChunkWalk nw = w;
      nw.unit = part.last;
      if (nw.unit == nw.units) runs.next_item(nw);
      bool next_on = false;
      if (!end.at(nw)) {
        const Part next(runs, p, nw, end);
        next_on = next.first < next.until(t);
        if (next_on && quarter * 32 < next.rows_of(t)) bring(nw, next.rows_of(t));
      }
      if (until > part.first) {
        warp_wait(&ms->o_done[t][(steps - 1) & 1], (steps - 1) >> 1, ms, p);
        fence_after_sync();
      }
      if (next_on) brought();                                      // (there by now, and the next scores are worked out meanwhile)
      if (on) {
        const bool whole = part.first == 0 && part.last == w.units;
        const int slot = part.first == 0 ? 1 : 0;                  // pieces of a CTA: of an item it begins, of one it goes on with
        int mine_at = at;
        asm volatile("" : "+r"(mine_at));                          // (so that what follows is not worked out before the units and kept)
        const int tok = p.group_of.quot(mine_at), head = w.head * p.group + mine_at - tok * p.group, edge = max(0, runs.sees(w, w.rt * R));
        const int64_t to = (int64_t)(w.start + tok) * p.H + head, piece = ((int64_t)blockIdx.x * 2 + slot) * R + mine_at - w.rt * R;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const bool odd = *(volatile int *)&ms->odd[parts % ODD_SLOTS] == parts;
#pragma unroll 1
        for (int x = 0; x < p.head_dim; x += 32) {
          float o[32];
          if (until > part.first) {
            tmem_ld32(o_at + x, o);
            tmem_ld_wait32(o);
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = 0.f;
          }
          if (odd && mine)                                         // what the values have that is not finite (rare)
            for (int key = max(edge, part.first * KEYS); key < min(vis, part.last * KEYS); ++key) {
              const int pg = p.page.quot(key), id = w.row[pg];
              if (id < 0 || id >= p.n_pages) continue;
              const __nv_bfloat16 *src = (const __nv_bfloat16 *)(p.v + (int64_t)id * p.page_bytes + (int64_t)(key - pg * (int)p.page.d) * p.slot_bytes +
                                                                 (int64_t)w.head * p.head_bytes) + x;
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const float y = __bfloat162float(src[i]);
                if (!(fabsf(y) < INFINITY)) o[i] += y;
              }
            }
          if (mine) {
            if (whole) {
              __nv_bfloat16 *dst = (__nv_bfloat16 *)p.out + to * p.head_dim + x;
              uint32_t y[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = pack(o[2 * i] * inv, o[2 * i + 1] * inv);
              if (p.wide_out) {
                store32(dst, y);
                store32(dst + 16, y + 8);
              } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) ((uint4 *)dst)[i] = make_uint4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
              }
            } else {
              float *dst = p.pieces + ((int64_t)blockIdx.x * 2 + slot) * R * p.head_dim + (int64_t)x * R + (mine_at - w.rt * R) * 4;   // [four columns][row]
#pragma unroll
              for (int i = 0; i < 32; i += 4) __stcg((float4 *)(dst + i * R), make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]));
            }
          }
        }
        if (mine) {
          if (!whole) __stcg((float2 *)(p.pieces + (int64_t)paged::CHUNK_TC_CTAS * 2 * R * p.head_dim + piece * 2), make_float2(m, l));
          else if (p.lse) p.lse[to] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
        }
      }
      fence_before_sync();
      w = nw;
    }
  }
  fence_before_sync();
  __syncthreads();
  if (warp == MMA_WARP) {
    fence_after_sync();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::COLS));
  }
}

const char *CALL = "ouro_paged_chunk_attention";

template <int D>
int launch(ChunkParams p, int64_t cost, int64_t tiles, const Maps &maps, int box_rows, cudaStream_t s) {
  using C = Cfg<D>;
  static bool ready[paged::MAX_DEVICES] = {};
  int dev = 0, sms = 0;
  if (!paged::device(&dev, &sms)) return paged::refuse(CALL, "no usable current device", OURO_ECUDA);
  if (!ready[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(paged_chunk_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::BYTES);
    if (e != cudaSuccess) return paged::refuse(CALL, cudaGetErrorString(e), OURO_ECUDA);
    ready[dev] = true;
  }
  const int64_t most = sms < paged::CHUNK_TC_CTAS ? sms : paged::CHUNK_TC_CTAS, want = cost / MIN_RUN;
  const int grid = (int)(want < 1 ? 1 : want < most ? want : most);
  Share::set(p, grid, tiles);
  p.wide_out = (uintptr_t)p.out % 32 == 0;
  const cudaError_t e = launch_pdl(paged_chunk_tc_kernel<D>, dim3(grid), dim3(THREADS), C::BYTES, s, p, maps, box_rows);
  OURO_COUNT_LAUNCH();
  if (e != cudaSuccess) return paged::refuse(CALL, cudaGetErrorString(e), OURO_ECUDA);
  return grid > 1 && Share::may_cut(p.cap) ? paged::chunk_tc_join(p, grid, s) : OURO_OK;
}

}  // namespace

// 0: does not take the call (pages that no box fits).
int paged::chunk_tc(const ouro_paged_cache *c, const paged::ChunkParams &p, int64_t cost, int64_t tiles, cudaStream_t s, int *status) {
  if (c->dtype != OURO_BF16 || c->page_size % 8) return 0;
  int box_rows = 8;
  while (box_rows < KEYS && c->page_size % (2 * box_rows) == 0) box_rows *= 2;
  Maps maps;
  if (!make_map(&maps.k, c, c->k, box_rows) || !make_map(&maps.v, c, c->v, box_rows)) return 0;
  *status = c->head_dim <= 64 ? launch<64>(p, cost, tiles, maps, box_rows, s) : launch<128>(p, cost, tiles, maps, box_rows, s);
  return 1;
}
