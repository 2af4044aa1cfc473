// Attention of a chunk of new tokens for each of several sequences over a paged cache: checks of the call, the kernel for f32 and for pages that no copy
// of the copy engine fits, and the kernel that joins what was cut.
//
//     o_i = sum_j e^(s_ij) v_j / sum_j e^(s_ij),   s_ij = scale q_i . k_j,   j = 0 .. len - m + i for the i-th of a sequence's m new tokens
//
// Four operations a query head, key and dimension: behind a few dozen query rows the contractions are what counts, not the keys' bytes.  bf16 goes to
// paged_chunk_tc.cu.  Here a CTA has 64 query rows in shared memory, 16 to a warp, passes over the keys 64 at a time and keeps maximum, sum and output of its
// rows in registers.  The next keys are asked for when the scores are done, the next values when the outputs are, and the ids of their pages a unit before that.
// Products of f32 are three contractions (mma.sync, 8 deep, 11 bits an operand): x y = X Y + X y' + x' Y with the upper and the lower 11 bits of each, and x' y'
// (2^-22 of the product at most, of either sign) left out.  The tensor cores round their sums towards 0, which counts in long chains (one for a score,
// one for an output: 2.5e-6 of the norm off, 44 us for 46 below): the small products and every 32 dims, or 64 keys, of the large ones have sums of their own, which are added up in
// 32 bits.  How far outputs are from 64 bits, of their norm, and those of 32-bit multiply-adds: heads of 32 6.7e-7 for 5.3e-7, 64 6.8e-7 for 6.4e-7, 96 6.0e-7 for 7.8e-7, 128
// 6.4e-7 for 9.1e-7 (sequences of 700 and 1500: what is left out of products is the same for all heads, what sums lose grows with them).  4096 tokens, four heads of 128: 372 us, 46
// TFLOP/s; multiply-adds by four rows and four keys a thread 503, bound by what came from shared memory; the contractions alone would take 180.  Two CTAs an SM
// are eight warps, too few to hide one another's chains of loads, parts and contractions.  A call of few units is best dealt out one by one (five prompts of the
// `small` shape, up to 411 tokens: 46 us).  bf16 in pages that are no multiple of 8 tokens passes here as f32 does, but for parts that 8 bits have not: 7B shape, 2048 tokens 531 us (62 on
// the tcgen05 kernel in pages of 16), 70B shape, one prompt of 4096 3.8 ms (0.30), 1.1B shape, mixed batch 82 (26): 45 to 72 TFLOP/s.
#include <cfloat>

#include "paged_chunk.cuh"
#include "row_ops.cuh"

namespace {

using paged::ChunkParams;
using paged::ChunkWalk;

const char *CALL = "ouro_paged_chunk_attention";

constexpr int R = paged::CHUNK_ROWS, KEYS = 64, THREADS = 128;
constexpr int ITEM_COST = 1, SNAP = 0, MIN_RUN = 1;
typedef paged::ChunkRuns<R, KEYS, ITEM_COST, SNAP, MIN_RUN> Share;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ void store4(float *p, float4 x) { *(float4 *)p = x; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 x) { *(uint2 *)p = make_uint2(rowops::pack(x.x, x.y), rowops::pack(x.z, x.w)); }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f; }

// 16 bytes, or zeros where there is nothing to read
__device__ __forceinline__ void cp_async16(void *dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void wait_but_one() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
// Four values of N pieces to shared memory as f32: f32 on its way, bf16 at once.
template <int N>
__device__ __forceinline__ void bring(float *const *dst, const float *const *src, const bool *there) {
#pragma unroll
  for (int i = 0; i < N; ++i) cp_async16(dst[i], src[i], there[i]);
}
template <int N>
__device__ __forceinline__ void bring(float *const *dst, const __nv_bfloat16 *const *src, const bool *there) {
  uint2 x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = there[i] ? *(const uint2 *)src[i] : make_uint2(0, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float2 a = rowops::unpack(x[i].x), b = rowops::unpack(x[i].y);
    *(float4 *)dst[i] = make_float4(a.x, a.y, b.x, b.y);
  }
}

template <int D>
struct Cfg {
  static constexpr int PITCH = D + 16, V_PITCH = D + 4;            // (fragments of 16 bytes a lane meet every bank once in eight lanes)
  static constexpr int OFF_K = R * PITCH, OFF_V = OFF_K + KEYS * PITCH, OFF_AT = OFF_V + KEYS * V_PITCH, OFF_MISC = OFF_AT + 2 * KEYS;
  static constexpr int PLAN = 5 * OURO_MAX_LIST;                   // at the beginning, until the first queries
  static constexpr int BYTES = ((OFF_MISC > PLAN ? OFF_MISC : PLAN) + 64) * 4;
};

// x = big + small, both with the 11 bits that a contraction takes (of the small part it takes the upper ones).  NEAR: big is the nearest, so that the
// products of two small parts, which are left out, are no bias; else the next towards 0, which the type's largest value has too.
template <bool NEAR>
__device__ __forceinline__ void split(float x, uint32_t &big, uint32_t &small) {
  big = (__float_as_uint(x) + (NEAR ? 0x1000u : 0u)) & 0xffffe000u;
  small = __float_as_uint(x - __uint_as_float(big));
}
template <bool NEAR, bool EXACT>                                   // EXACT: no more than 8 bits to begin with
__device__ __forceinline__ void split4(const float4 &x, uint32_t *big, uint32_t *small) {
  const float y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (EXACT) big[i] = __float_as_uint(y[i]);
    else split<NEAR>(y[i], big[i], small[i]);
}
__device__ __forceinline__ void contract(float *c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ bool finite4(const float4 &x) {
  return fabsf(x.x) <= FLT_MAX && fabsf(x.y) <= FLT_MAX && fabsf(x.z) <= FLT_MAX && fabsf(x.w) <= FLT_MAX;
}

template <typename T, int D>
__global__ void __launch_bounds__(THREADS, 2) paged_chunk_kernel(const ChunkParams p) {
  using C = Cfg<D>;
  constexpr int D4 = D / 4, Q32 = D / 32;                          // groups of four dims, of 32
  constexpr bool EXACT = sizeof(T) == 2;
  extern __shared__ __align__(16) float smem[];
  float *qs = smem, *ks = smem + C::OFF_K, *vs = smem + C::OFF_V;
  int64_t *ats = (int64_t *)(smem + C::OFF_AT);                    // where a unit's keys lie in their pool; -1: on no page
  const int tid = threadIdx.x, lane = tid & 31, g = lane >> 2, t = lane & 3, r0 = tid / 32 * 16 + g;       // the thread's rows: r0, r0 + 8
  const Share runs(p);
  runs.touch();
  pdl_wait();
  pdl_trigger();
  ChunkWalk *places = (ChunkWalk *)((uint8_t *)smem + C::BYTES - 256);
  runs.plan((int *)smem, (Share::Known *)(smem + OURO_MAX_LIST), places, THREADS);
  ChunkWalk w = places[0];
  const ChunkWalk end = places[1];
  if (tid == 0) p.begins[blockIdx.x] = paged::same(w, end) ? make_int4(-1, 0, 0, 0) : make_int4(w.s, w.head, w.rt, w.unit);

  while (!paged::same(w, end)) {
    // ---- an item, or the part of it in this run
    const int rows = min(R, w.m * p.group - w.rt * R), part_begin = w.unit;
    const int last = w.s == end.s && w.head == end.head && w.rt == end.rt ? end.unit : w.units;
    constexpr int PER = KEYS * D4 / THREADS, BATCH = PER < 8 ? PER : PER / 2;    // pieces of four values of a unit's keys, or of the queries, for a thread
    static_assert(R == KEYS && KEYS <= THREADS && KEYS * D4 % THREADS == 0 && PER % BATCH == 0, "");
    auto row_of = [&](int i) { return (tid + i * THREADS) / D4; };
    auto col_of = [&](int i) { return (tid + i * THREADS) % D4 * 4; };
    int id = -1;                                                   // of the page of a thread's key
    auto ask_id = [&](int unit) {
      const int key = unit * KEYS + tid;
      id = tid < KEYS && unit < last && key < w.len ? w.row[p.page.quot(key)] : -1;
    };
    auto place = [&](int unit) {                                   // the unit's keys, once their pages are known; true: one of the sequence's is on none
      if (tid >= KEYS) return false;
      const int key = unit * KEYS + tid;
      const bool there = id >= 0 && id < p.n_pages;
      ats[tid] = there ? (int64_t)id * p.page_bytes + (int64_t)(key - p.page.quot(key) * (int)p.page.d) * p.slot_bytes : -1;
      return unit < last && key < w.len && !there;
    };
    auto ask = [&](const uint8_t *pool, float *to, int pitch) {    // a unit's keys or values
      const uint8_t *of_head = pool + (int64_t)w.head * p.head_bytes;
#pragma unroll
      for (int i0 = 0; i0 < PER; i0 += BATCH) {
        float *dst[BATCH];
        const T *src[BATCH];
        bool there[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const int64_t at = ats[row_of(i0 + i)];
          there[i] = at >= 0;
          dst[i] = to + row_of(i0 + i) * pitch + col_of(i0 + i);
          src[i] = (const T *)(of_head + (there[i] ? at : 0)) + col_of(i0 + i);
        }
        bring<BATCH>(dst, src, there);
      }
    };
    ask_id(w.unit);
    __syncthreads();                                               // (what was there has been read)
    bool missing = place(w.unit);
#pragma unroll
    for (int i0 = 0; i0 < PER; i0 += BATCH) {
      float *dst[BATCH];
      const T *src[BATCH];
      bool there[BATCH];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int r = row_of(i0 + i);
        there[i] = r < rows;
        const int at = w.rt * R + (there[i] ? r : 0), tok = p.group_of.quot(at);
        dst[i] = qs + r * C::PITCH + col_of(i0 + i);
        src[i] = (const T *)p.q + (int64_t)(w.start + tok) * p.q_stride + (int64_t)(w.head * p.group + at - tok * p.group) * D + col_of(i0 + i);
      }
      bring<BATCH>(dst, src, there);
    }
    ask_id(w.unit + 1);
    __syncthreads();
    ask(p.k, ks, C::PITCH);
    commit();
    ask(p.v, vs, C::V_PITCH);
    commit();
    int vis[2];
    float m[2], l[2], o[Q32][4][4];                                // o[q][i]: dims 32 q + 8 t + i and + 4 of the first row, then of the second
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      vis[i] = r0 + 8 * i < rows ? runs.sees(w, w.rt * R + r0 + 8 * i) : 0;
      m[i] = -INFINITY;
      l[i] = 0.f;
    }
#pragma unroll
    for (int q = 0; q < Q32; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[q][i][c] = 0.f;
    const int all_see = runs.sees(w, w.rt * R);                    // keys that every row sees
    for (; w.unit < last; ++w.unit) {
      const int key0 = w.unit * KEYS;
      wait_but_one();
      const bool gone = __syncthreads_or(missing);                 // (queries and keys are there)
      float s[8][4];                                               // s[n]: keys 8 n + 2 t and the next of the first row, then of the second
      // Dims in any order, the same for both: a lane's 16 bytes are two steps of eight.  Contractions round their sums towards 0: products with small parts
      // are summed up by themselves, those of big parts 32 dims at a time.
#pragma unroll
      for (int n0 = 0; n0 < 8; n0 += 4) {
        float fine[4][4] = {};
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[n0 + n][c] = 0.f;
#pragma unroll 1
        for (int d0 = 0; d0 < D; d0 += 32) {
          float sum[4][4] = {};
#pragma unroll
          for (int d = 0; d < 32; d += 16) {
            uint32_t ab[2][4], as[2][4], bb[4][4], bs[4][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) split4<true, EXACT>(*(const float4 *)(qs + (r0 + 8 * i) * C::PITCH + d0 + d + 4 * t), ab[i], as[i]);
#pragma unroll
            for (int n = 0; n < 4; ++n) split4<false, EXACT>(*(const float4 *)(ks + (8 * (n0 + n) + g) * C::PITCH + d0 + d + 4 * t), bb[n], bs[n]);
#pragma unroll
            for (int h = 0; h < 4; h += 2) {
              if (!EXACT) {
#pragma unroll
                for (int n = 0; n < 4; ++n) contract(fine[n], as[0][h], as[1][h], as[0][h + 1], as[1][h + 1], bb[n][h], bb[n][h + 1]);
#pragma unroll
                for (int n = 0; n < 4; ++n) contract(fine[n], ab[0][h], ab[1][h], ab[0][h + 1], ab[1][h + 1], bs[n][h], bs[n][h + 1]);
              }
#pragma unroll
              for (int n = 0; n < 4; ++n) contract(sum[n], ab[0][h], ab[1][h], ab[0][h + 1], ab[1][h + 1], bb[n][h], bb[n][h + 1]);
            }
          }
#pragma unroll
          for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) s[n0 + n][c] += sum[n][c];
        }
        if (!EXACT)
#pragma unroll
          for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) s[n0 + n][c] += fine[n][c];
      }
      missing = place(w.unit + 1);
      __syncthreads();                                             // the keys have been read
      if (w.unit + 1 < last) ask(p.k, ks, C::PITCH);               // (behind the last unit the next item's follow)
      commit();
      ask_id(w.unit + 2);
      const bool edge = gone || key0 + KEYS > all_see;             // (the same for the CTA) not every row sees every key
      if (edge) {
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int key = key0 + 8 * n + 2 * t + e;
            bool on = key < w.len;
            if (gone && on) {
              const int of = w.row[p.page.quot(key)];
              on = of >= 0 && of < p.n_pages;
            }
            if (!on || key >= vis[0]) s[n][e] = -INFINITY;
            if (!on || key >= vis[1]) s[n][2 + e] = -INFINITY;
          }
      }
      float grown[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float top = fmaxf(s[0][2 * i], s[0][2 * i + 1]);
#pragma unroll
        for (int n = 1; n < 8; ++n) top = fmaxf(top, fmaxf(s[n][2 * i], s[n][2 * i + 1]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        top = fmaxf(m[i], top * p.scale_log2);
        const float base = base_of(top);
        grown[i] = ex2(m[i] - base);
        m[i] = top;
        l[i] *= grown[i];
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float &x = s[n][2 * i + e];
            x = ex2(fmaf(x, p.scale_log2, -base));
            l[i] += x;
          }
      }
      wait_but_one();
      __syncthreads();                                             // (values are there)
      if (edge) {
        // 0 times a value that is no finite number must be 0 for the rows that do not see it: such values are taken out, and added for those that do (rare).
        bool odd = false;
#pragma unroll
        for (int i = 0; i < PER; ++i) odd |= !finite4(*(const float4 *)(vs + row_of(i) * C::V_PITCH + col_of(i)));
        if (__syncthreads_or(odd)) {
          for (int i = 0; i < 2; ++i) grown[i] = fmaxf(grown[i], FLT_MIN);         // (an infinity times 0 would be none)
#pragma unroll 1
          for (int key = 0; key < KEYS; ++key) {
            float x[2] = {0.f, 0.f};
#pragma unroll
            for (int n = 0; n < 8; ++n)
              if (n == key / 8) {
                x[0] = key & 1 ? s[n][1] : s[n][0];
                x[1] = key & 1 ? s[n][3] : s[n][2];
              }
#pragma unroll
            for (int i = 0; i < 2; ++i) x[i] = __shfl_sync(0xffffffffu, x[i], (lane & ~3) | (key % 8 / 2));
#pragma unroll
            for (int q = 0; q < Q32; ++q)
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  const float v = vs[key * C::V_PITCH + 32 * q + 8 * t + 4 * (c & 1) + i];
                  if (!(fabsf(v) <= FLT_MAX) && key0 + key < vis[c / 2]) o[q][i][c] = fmaf(x[c / 2], v, o[q][i][c]);
                }
          }
          __syncthreads();
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            float *at = vs + row_of(i) * C::V_PITCH + col_of(i);
            for (int c = 0; c < 4; ++c)
              if (!(fabsf(at[c]) <= FLT_MAX)) at[c] = 0.f;
          }
          __syncthreads();
        }
      }
      // Keys in an order in which a row's probabilities are where the contraction wants them: 2 t and 2 t + 1 of eight are its t and t + 4.
#pragma unroll
      for (int q = 0; q < Q32; ++q) {
        float sum[4][4] = {}, fine[4][4] = {};
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          uint32_t ab[4], as[4], bb[2][4], bs[2][4];
          split4<true, false>(make_float4(s[n][0], s[n][2], s[n][1], s[n][3]), ab, as);
#pragma unroll
          for (int e = 0; e < 2; ++e) split4<false, EXACT>(*(const float4 *)(vs + (8 * n + 2 * t + e) * C::V_PITCH + 32 * q + 4 * g), bb[e], bs[e]);
#pragma unroll
          for (int i = 0; i < 4; ++i) contract(fine[i], as[0], as[1], as[2], as[3], bb[0][i], bb[1][i]);
          if (!EXACT)
#pragma unroll
            for (int i = 0; i < 4; ++i) contract(fine[i], ab[0], ab[1], ab[2], ab[3], bs[0][i], bs[1][i]);
#pragma unroll
          for (int i = 0; i < 4; ++i) contract(sum[i], ab[0], ab[1], ab[2], ab[3], bb[0][i], bb[1][i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) o[q][i][c] = fmaf(o[q][i][c], grown[c / 2], sum[i][c] + fine[i][c]);
      }
      __syncthreads();                                             // the values have been read
      if (w.unit + 1 < last) ask(p.v, vs, C::V_PITCH);
      commit();
    }
    // ---- its end
    const bool whole = part_begin == 0 && w.unit == w.units;
    const int slot = part_begin == 0 ? 1 : 0;
    float *mls = p.pieces + (int64_t)paged::CHUNK_CTAS * 2 * R * D;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = r0 + 8 * i;
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
      if (r >= rows) continue;
      const int at = w.rt * R + r, tok = p.group_of.quot(at);
      const int64_t to = (int64_t)(w.start + tok) * p.H + w.head * p.group + at - tok * p.group, piece = ((int64_t)blockIdx.x * 2 + slot) * R + r;
      const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll
      for (int q = 0; q < Q32; ++q)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int col = 32 * q + 8 * t + 4 * c, x = 2 * i + c;
          if (whole) store4((T *)p.out + to * D + col, make_float4(o[q][0][x] * inv, o[q][1][x] * inv, o[q][2][x] * inv, o[q][3][x] * inv));
          else __stcg((float4 *)(p.pieces + piece * D + col), make_float4(o[q][0][x], o[q][1][x], o[q][2][x], o[q][3][x]));
        }
      if (t == 0) {
        if (!whole) __stcg((float2 *)(mls + piece * 2), make_float2(m[i], l[i]));
        else if (p.lse) p.lse[to] = lse_of(m[i], l[i]);
      }
    }
    if (w.unit == w.units) runs.next_item(w);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// Items that are cut: the pieces of one are the second of the CTA before the first run that begins within it, the first of that run's CTA and of those behind
// that begin within it too.  gridDim.x: cut items at most, by rank; gridDim.y CTAs share the rows of one, four columns of a row for a thread, which asks for
// BATCH pieces at once.  BY_COLUMNS: a piece's outputs lie as [four columns][row], as threads that have a row each write them best, else [row][column].
constexpr int JOIN_THREADS = 256, BATCH = 4, JOIN_CTAS = 8 * 148;
template <typename T, int ROWS, int CTAS, bool BY_COLUMNS>
__global__ void __launch_bounds__(JOIN_THREADS) paged_chunk_join_kernel(const ChunkParams p, const int grid) {
  constexpr int WORDS = (CTAS + 31) / 32;
  __shared__ uint32_t s_first[WORDS], s_more[WORDS];               // a bit for each CTA: the first that begins within its item; one of those behind
  const int D = p.head_dim, tid = threadIdx.x;
  pdl_wait();
  pdl_trigger();
  for (int i = tid; i < WORDS * 32; i += JOIN_THREADS) {
    const int4 x = i < grid ? p.begins[i] : make_int4(-1, 0, 0, 0), y = i > 0 && i < grid ? p.begins[i - 1] : x;
    const bool within = x.x >= 0 && x.w > 0, more = within && i > 0 && y.w > 0 && y.x == x.x && y.y == x.y && y.z == x.z;
    const uint32_t a = __ballot_sync(0xffffffffu, within && !more), b = __ballot_sync(0xffffffffu, more);
    if ((tid & 31) == 0) s_first[i / 32] = a, s_more[i / 32] = b;
  }
  __syncthreads();
  int word = 0, rank = blockIdx.x;
  while (word < WORDS && rank >= __popc(s_first[word])) rank -= __popc(s_first[word++]);
  if (word == WORDS) return;
  uint32_t bits = s_first[word];
  for (; rank > 0; --rank) bits &= bits - 1;
  const int c = word * 32 + __ffs(bits) - 1;
  int c1 = c;
  for (int i = c + 1; i < grid; i = (i / 32 + 1) * 32) {           // ones in a row
    const uint32_t other = ~(s_more[i / 32] >> (i & 31));
    const int run = min(other ? __ffs(other) - 1 : 32, 32 - (i & 31));
    c1 += run;
    if (run < 32 - (i & 31)) break;
  }
  const int4 b = p.begins[c];
  const int start = p.starts[b.x], m = p.starts[b.x + 1] - start, rows = min(ROWS, m * p.group - b.z * ROWS), C4 = D / 4;
  const float *mls = p.pieces + (int64_t)CTAS * 2 * ROWS * D;
  // (by columns: a warp has 8 rows of 16 columns, so that it reads 128 bytes and writes 32 at a place)
  const int each = ROWS / gridDim.y;
  for (int e = tid; e < each * C4; e += JOIN_THREADS) {
    const int q = e / (BY_COLUMNS ? 8 : 1), r = each * blockIdx.y + (BY_COLUMNS ? e % 8 + q / C4 * 8 : q / C4), col = q % C4 * 4;
    if (r >= rows) continue;
    float M = -INFINITY, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = c - 1; j0 <= c1; j0 += BATCH) {
      float2 ml[BATCH];
      float4 y[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const int j = j0 + k;
        const int64_t at = ((int64_t)j * 2 + (j == c - 1 ? 1 : 0)) * ROWS;
        ml[k] = make_float2(-INFINITY, 0.f);
        y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (j > c1) continue;
        ml[k] = __ldcg((const float2 *)(mls + (at + r) * 2));
        y[k] = __ldcg((const float4 *)(p.pieces + (BY_COLUMNS ? at * D + (int64_t)col * ROWS + r * 4 : (at + r) * D + col)));
      }
      float mx = M;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) mx = fmaxf(mx, ml[k].x);
      const float base = base_of(mx), a = ex2(M - base);
      M = mx;
      L *= a;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] *= a;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const float x = ex2(ml[k].x - base);
        L = fmaf(x, ml[k].y, L);
        o[0] = fmaf(x, y[k].x, o[0]);
        o[1] = fmaf(x, y[k].y, o[1]);
        o[2] = fmaf(x, y[k].z, o[2]);
        o[3] = fmaf(x, y[k].w, o[3]);
      }
    }
    const int at = b.z * ROWS + r, tok = p.group_of.quot(at);
    const int64_t to = (int64_t)(start + tok) * p.H + b.y * p.group + at - tok * p.group;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    store4((T *)p.out + to * D + col, make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv));
    if (p.lse && col == 0) p.lse[to] = lse_of(M, L);
  }
}

template <typename T, int ROWS, int CTAS, bool BY_COLUMNS>
int join(const ChunkParams &p, int grid, cudaStream_t s) {
  const int64_t items = (((int64_t)p.rows * p.group + ROWS - 1) / ROWS + (p.n < p.rows ? p.n : p.rows)) * p.Hkv;      // at most
  // As many CTAs as are resident at once, with eight rows each at least.
  dim3 ctas((unsigned)min((int64_t)grid - 1, items), 1);
  while (ctas.y < ROWS / 8 && ctas.x * ctas.y * 2 <= JOIN_CTAS) ctas.y *= 2;
  const cudaError_t e = launch_pdl(paged_chunk_join_kernel<T, ROWS, CTAS, BY_COLUMNS>, ctas, dim3(JOIN_THREADS), 0, s, p, grid);
  OURO_COUNT_LAUNCH();
  return e == cudaSuccess ? OURO_OK : paged::refuse(CALL, cudaGetErrorString(e), OURO_ECUDA);
}

template <typename T, int D>
int launch(ChunkParams p, int64_t cost, int64_t tiles, cudaStream_t s) {
  using C = Cfg<D>;
  static int fit[paged::MAX_DEVICES] = {};                         // CTAs that are resident at once, per device
  int dev = 0, sms = 0;
  if (!paged::device(&dev, &sms)) return paged::refuse(CALL, "no usable current device", OURO_ECUDA);
  if (!fit[dev]) {
    int per_sm = 0;
    cudaError_t e = cudaFuncSetAttribute(paged_chunk_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::BYTES);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, paged_chunk_kernel<T, D>, THREADS, C::BYTES);
    if (e != cudaSuccess) return paged::refuse(CALL, cudaGetErrorString(e), OURO_ECUDA);
    if (per_sm < 1) return paged::refuse(CALL, "the kernel does not fit this device", OURO_ECUDA);
    fit[dev] = min(paged::CHUNK_CTAS, sms * per_sm);
  }
  const int grid = (int)min((int64_t)fit[dev], max((int64_t)1, cost / MIN_RUN));
  Share::set(p, grid, tiles);
  const cudaError_t e = launch_pdl(paged_chunk_kernel<T, D>, dim3(grid), dim3(THREADS), C::BYTES, s, p);
  OURO_COUNT_LAUNCH();
  if (e != cudaSuccess) return paged::refuse(CALL, cudaGetErrorString(e), OURO_ECUDA);
  return grid > 1 && Share::may_cut(p.cap) ? join<T, R, paged::CHUNK_CTAS, false>(p, grid, s) : OURO_OK;
}

template <typename T>
int by_dim(const ChunkParams &p, int64_t cost, int64_t tiles, cudaStream_t s) {
  switch (p.head_dim) {
    case 32: return launch<T, 32>(p, cost, tiles, s);
    case 64: return launch<T, 64>(p, cost, tiles, s);
    case 96: return launch<T, 96>(p, cost, tiles, s);
    default: return launch<T, 128>(p, cost, tiles, s);
  }
}

}  // namespace

int paged::chunk_tc_join(const paged::ChunkParams &p, int grid, cudaStream_t s) { return join<__nv_bfloat16, paged::CHUNK_TC_ROWS, paged::CHUNK_TC_CTAS, true>(p, grid, s); }

extern "C" int ouro_paged_chunk_attention(const ouro_paged_cache *c, int32_t layer, const int32_t *seqs, const int32_t *starts, int32_t n, int32_t rows,
                                          const void *q, int64_t q_stride, int32_t n_heads, float scale, void *out, float *lse, void *stream) {
  if (const char *w = paged::wrong(c)) return paged::refuse(CALL, w);
  if (layer < 0 || layer >= c->n_layers) return paged::refuse(CALL, "no such layer");
  if (n < 0 || n > OURO_MAX_LIST) return paged::refuse(CALL, "n is below 0 or above OURO_MAX_LIST");
  if (rows < 0) return paged::refuse(CALL, "rows is below 0");
  if (n_heads < 1 || n_heads % c->n_kv_heads) return paged::refuse(CALL, "n_heads is not a multiple of the cache's n_kv_heads");
  if (!(scale > 0.f) || scale > 1e30f) return paged::refuse(CALL, "scale is not a positive number");
  if (n == 0 || rows == 0) return OURO_OK;
  if (!q || !out || !starts) return paged::refuse(CALL, "q, out or starts is NULL");
  if (!paged::words(seqs, starts, lse)) return paged::refuse(CALL, "seqs, starts or lse is not 4-byte aligned");
  if (!seqs && n > c->max_seqs) return paged::refuse(CALL, "more sequences than the table has");
  const int esize = c->dtype == OURO_F32 ? 4 : 2;
  if (((uintptr_t)q | (uintptr_t)out) % 16 || (q_stride * esize) % 16) return paged::refuse(CALL, "q, out or q_stride is not a multiple of 16 bytes");
  if (q_stride < (int64_t)n_heads * c->head_dim) return paged::refuse(CALL, "q_stride is below n_heads * head_dim");
  ChunkParams p{};
  p.group = n_heads / c->n_kv_heads;
  p.cap = c->max_pages * c->page_size;
  if ((int64_t)rows * p.group > paged::MAX_TOKENS) return paged::refuse(CALL, "rows * n_heads / n_kv_heads is above 2^31 - 65536");
  if (p.group > 65536) return paged::refuse(CALL, "n_heads / n_kv_heads is above 65536");
  if (((int64_t)p.cap + 1024) * p.group > paged::MAX_TOKENS) return paged::refuse(CALL, "(max_pages * page_size + 1024) * n_heads / n_kv_heads is above 2^31 - 65536");
  // units of the finest kind at most: every tile may see all keys of the longest sequence
  const int64_t tiles = ((int64_t)rows * p.group + R - 1) / R + (n < rows ? n : rows), item = ((int64_t)p.cap + KEYS - 1) / KEYS + 8;
  if (tiles > Share::MAX_ITEMS / c->n_kv_heads || tiles > ((int64_t)1 << 40) / item / c->n_kv_heads) return paged::refuse(CALL, "the sequences' work may be above 2^40 units or 2^30 tiles");
  const paged::Layout l = paged::layout(*c);
  p.k = (const uint8_t *)c->k + (int64_t)layer * c->layer_stride * esize;
  p.v = (const uint8_t *)c->v + (int64_t)layer * c->layer_stride * esize;
  p.table = c->table; p.lens = c->lens; p.seqs = seqs; p.starts = starts; p.status = c->status;
  p.q = q; p.out = out; p.lse = lse;
  p.begins = (int4 *)((char *)c->workspace + l.begins);
  p.pieces = (float *)((char *)c->workspace + l.chunk_pieces);
  p.page_bytes = c->page_stride * esize; p.slot_bytes = c->slot_stride * esize; p.head_bytes = c->head_stride * esize; p.q_stride = q_stride;
  p.n = n; p.rows = rows; p.H = n_heads; p.Hkv = c->n_kv_heads; p.layer = layer; p.head_dim = c->head_dim;
  p.page.set(c->page_size); p.group_of.set(p.group);
  p.n_pages = c->n_pages; p.max_pages = c->max_pages; p.max_seqs = c->max_seqs;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.wait_limit = paged::wait_limit.load(std::memory_order_relaxed);
  const int64_t cost = tiles * item * c->n_kv_heads;
  int status = OURO_OK;
  if (paged::chunk_tc(c, p, cost, tiles, (cudaStream_t)stream, &status)) return status;
  return c->dtype == OURO_F32 ? by_dim<float>(p, cost, tiles, (cudaStream_t)stream) : by_dim<__nv_bfloat16>(p, cost, tiles, (cudaStream_t)stream);
}
