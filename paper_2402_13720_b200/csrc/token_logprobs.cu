// Log probabilities of given tokens, entropy and the best alternatives of every row of logits, in one pass over the logits.
//
//     m = max x,  Z = sum e^(x - m),  T = sum (x - m) e^(x - m)
//     log p(t) = (x_t - m) - ln Z,    H = ln Z - T / Z
//
// Bound by HBM without alternatives (2048 rows of 64000 f32: 81 us, 6.5 TB/s); with them by what the warps have to issue (20: 96 us; bf16,
// 5: 82 us for 40.6).  A row is a CTA's or, where rows are few, a cluster's, whose CTAs join through shared
// memory: one launch, no workspace.
//  - A thread keeps (m, Z - 1, T) of what it has seen, in 32 bits, relative to its own maximum, sixteen logits at a time, two in an instruction.
//    Z - 1, because a token that has nearly everything is as likely as the others leave it: ln Z = ln (1 + r), to r's precision (and with Z in place
//    of r 3 % less time).
//  - Candidates for the best alternatives go to a buffer of the CTA as 64-bit keys (value in an order-preserving integer image, then the
//    complement of the id: no two are equal, and the lowest id is first among equals).  After 1, 4, 16, .. batches of THREADS * E logits the
//    buffer is cut down to the best n; in between only what is larger than the n-th counts, some 3 n for every cut on average, which the maximum
//    of a thread's sixteen logits, needed for the sum anyway, mostly rules out for all of them.  Where it does not, the thread only notes where
//    it is, so that the loop stays one comparison and no warp waits for its lane: the notes are followed before the next cut, by as many threads
//    at once, from L2 (looked at in the loop: 114 us for 103, both with Z and loads through registers).  In the first batch, k of each warp make n, so the smallest of the warps' k-th
//    largest maxima bounds the n-th best of all from below.  Rows that fill the buffer or the notes all the same (they ascend) are done again
//    for the alternatives alone, with a look at the buffer after every batch; there, where many lanes of a warp have something to offer, the
//    n-th largest of the lanes' maxima bounds it too.
#include "paged.h"
#include "row_ops.cuh"

#include <cfloat>

namespace {

constexpr int E = 16;                              // logits of a thread at a time
constexpr int CROWD = 8;                           // lanes with something to offer from which on the maxima are sorted first
constexpr int GROWTH = 4;                          // the buffer is cut down after this many times as many batches as before (2: 4 % more time)
constexpr int SMALL = 512;                         // candidates of a CTA of 128 threads while the ring is in use
constexpr int NOTES = 256;                         // threads' batches with something larger than the n-th, since the buffer was last cut down
constexpr int WATER = 256;                         // candidates at which a row done again cuts the buffer down; a batch adds THREADS * E at most
constexpr float LOG2E = 1.4426950408889634f;

struct ScoreParams {
  const void *logits;
  int64_t row_stride;
  const int32_t *tokens;
  float *logprob, *entropy;
  int32_t *top_ids;
  float *top_logprobs;
  int vocab, n_top, ctas;                          // CTAs of a row
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {      // NaN where either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float y;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// Two 32-bit numbers at a time.
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
__device__ __forceinline__ u64 mul2(u64 a, u64 b) {
  u64 y;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) {
  u64 y;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
  return y;
}
// Integer image of a logit: larger logit, larger integer; NaN above all, -0 like +0; never 0.
__device__ __forceinline__ uint32_t image(float x) {
  // (volatile: else the images of sixteen logits are made in front of the branch behind which, rarely, they are wanted: 120 of 250 instructions a batch)
  float y;
  asm volatile("add.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(x));
  const uint32_t u = __float_as_uint(y);
  return x != x ? 0xffffffffu : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t im) {
  return im == 0xffffffffu ? NAN : __uint_as_float(im & 0x80000000u ? im ^ 0x80000000u : ~im);
}

struct Sums {
  float m, r, t;                                   // Z = 1 + r: without the largest's own 1, which would round away what little there is beside it
};
// Adds what b has seen to a.
__device__ __forceinline__ void join(Sums &a, const Sums &b) {
  const bool first = a.m >= b.m;                                  // (NaN: not, and then r becomes NaN by the factor or by itself)
  const float d = first ? b.m - a.m : a.m - b.m, f = ex2(d * LOG2E);
  const float z = 1.f + (first ? b.r : a.r), t = first ? b.t : a.t;
  a.r = fmaf(z, f, first ? a.r : b.r);
  a.t = (first ? a.t : b.t) + (f > 0.f ? fmaf(d, z, t) * f : 0.f);   // (a factor of 0 leaves nothing of T either, however far apart the maxima are)
  a.m = max_nan(a.m, b.m);
}

// Lists of 32 keys over a warp's lanes, largest first.
__device__ __forceinline__ u64 exchanged(u64 x, int o, bool larger) {
  const u64 y = __shfl_xor_sync(0xffffffffu, x, o);
  return (x > y) == larger ? x : y;
}
__device__ __forceinline__ u64 sorted(u64 x, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int o = k >> 1; o; o >>= 1) x = exchanged(x, o, ((lane & o) == 0) == ((lane & k) == 0));
  return x;
}
__device__ __forceinline__ u64 merged(u64 a, u64 b, int lane) {   // the best 32 of two lists
  b = __shfl_sync(0xffffffffu, b, 31 - lane);
  u64 x = a > b ? a : b;                                          // bitonic
#pragma unroll
  for (int o = 16; o; o >>= 1) x = exchanged(x, o, (lane & o) == 0);
  return x;
}

template <typename T>
__device__ __forceinline__ void unpack16(const uint4 *raw, float *x);
template <>
__device__ __forceinline__ void unpack16<float>(const uint4 *raw, float *x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[4 * i] = __uint_as_float(raw[i].x);
    x[4 * i + 1] = __uint_as_float(raw[i].y);
    x[4 * i + 2] = __uint_as_float(raw[i].z);
    x[4 * i + 3] = __uint_as_float(raw[i].w);
  }
}
template <>
__device__ __forceinline__ void unpack16<__nv_bfloat16>(const uint4 *raw, float *x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
      x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ float one(const float *p) { return *p; }
__device__ __forceinline__ float one(const __nv_bfloat16 *p) { return __bfloat162float(*p); }

// The CTA's candidates.
template <int THREADS>
struct Best {
  static constexpr int WARPS = THREADS / 32;
  static constexpr int BUFFER = WATER + THREADS * E + 32;          // (in front of the first and behind the last whole 16 bytes there are 7 at most)
  u64 *buffer;                                     // [room], at last [BUFFER]
  int room;
  u64 *lists;                                      // [WARPS][32]
  int *count;
  int *notes, *noted;                              // [NOTES] and their number
  uint32_t *bounds;                                // [WARPS]
  float last;                                      // value of the n-th of those that were there when the buffer was last cut down
  bool full;                                       // there were n
  bool much;                                       // this thread has seen the buffer filled to WATER
  bool over;                                       // something of this thread's did not get in

  // The n-th largest of the lanes' numbers.
  static __device__ __forceinline__ uint32_t nth(uint32_t s, int n, int lane) {
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
      for (int o = k >> 1; o; o >>= 1) {
        const uint32_t y = __shfl_xor_sync(0xffffffffu, s, o);
        s = ((lane & o) == 0) == ((lane & k) == 0) ? max(s, y) : min(s, y);
      }
    return __shfl_sync(0xffffffffu, s, n - 1);
  }
  // All lanes' logits from bound on: x[i] has id base + i % per + (i / per) * far, if bit i / per of there is set.
  template <int N>
  __device__ __forceinline__ void push(const float *x, uint32_t bound, uint32_t base, int per, uint32_t far, uint32_t there, int lane, uint32_t all = 0) {
    uint32_t take = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((image(x[i]) >= bound || (all >> i & 1)) && (there >> (i / per) & 1)) take |= 1u << i;
    const int mine = __popc(take);                 // places in the buffer: one request for the warp
    int at = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, at, o);
      if (lane >= o) at += up;
    }
    int first = 0;
    if (lane == 31 && at > 0) first = atomicAdd(count, at);
    at += __shfl_sync(0xffffffffu, first, 31) - mine;
    much |= take != 0 && at + mine > WATER;
    if (at + mine > room) over = true, take = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (take >> i & 1) buffer[at++] = (u64)image(x[i]) << 32 | (0xffffffffu - (base + i % per + (uint32_t)(i / per) * far));
    __syncwarp();
  }
  // The same logits, those that may be among the best n; top: the largest of a lane (NaN where there is one).
  template <int N>
  __device__ __forceinline__ void offer(const float *x, float top, uint32_t base, int per, uint32_t far, uint32_t there, int n, int lane) {
    const bool have = there != 0 && (!full || !(top <= last));
    const uint32_t some = __ballot_sync(0xffffffffu, have);
    if (some == 0) return;
    if (full && __popc(some) < CROWD) {
      if (have) {
#pragma unroll
        for (int g = 0; g < N; g += 4) {           // (four at a time: their maximum is there already)
          float four = x[g];
#pragma unroll
          for (int i = g + 1; i < g + 4 && i < N; ++i) four = max_nan(four, x[i]);
          if (!(four <= last)) {
#pragma unroll
            for (int i = g; i < g + 4 && i < N; ++i)
              if (!(x[i] <= last) && (there >> (i / per) & 1)) {
                const int at = atomicAdd(count, 1);
                much |= at >= WATER;
                if (at < room) buffer[at] = (u64)image(x[i]) << 32 | (0xffffffffu - (base + i % per + (uint32_t)(i / per) * far));
                else over = true;
              }
          }
        }
      }
      __syncwarp();
    } else {                                       // (nothing is above NaN: then all are candidates, and lose)
      push<N>(x, max(full ? image(last) + 1 : 1, nth(there ? image(top) : 0, n, lane)), base, per, far, there, lane);
    }
  }
  // Between two cuts only where there is something is put down (the thread's first vector); the sixteen logits are looked at when it comes to the
  // cut, by as many threads at once.
  __device__ __forceinline__ void note(float top, int vector) {
    if (!(top <= last)) {
      const int at = atomicAdd(noted, 1);
      if (at < NOTES) notes[at] = vector;
      else over = true;
    }
  }
  // The logits noted, behind a barrier and in front of one.
  template <typename T>
  __device__ __forceinline__ void look(const uint4 *xv, int v_end, int lead) {
    constexpr int VEC = 16 / sizeof(T), NV = E / VEC;
    for (int i = threadIdx.x; i < min(*noted, NOTES); i += THREADS) {
      const int v = notes[i];
      uint4 raw[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) raw[j] = xv[min(v + j * THREADS, v_end - 1)];
      float x[E];
      unpack16<T>(raw, x);
#pragma unroll
      for (int k = 0; k < E; ++k)
        if (!(x[k] <= last) && v + k / VEC * THREADS < v_end) {
          const int at = atomicAdd(count, 1);
          if (at < room) buffer[at] = (u64)image(x[k]) << 32 | (0xffffffffu - (uint32_t)(lead + (v + k / VEC * THREADS) * VEC + k % VEC));
          else over = true;
        }
    }
  }
  // The first logits, all warps.
  template <int N>
  __device__ __forceinline__ void begin(const float *x, float top, uint32_t base, int per, uint32_t far, uint32_t there, int n, int warp, int lane) {
    const uint32_t k_th = nth(there ? image(top) : 0, (n + WARPS - 1) / WARPS, lane);
    if (lane == 0) bounds[warp] = k_th;
    __syncthreads();
    uint32_t b = bounds[0];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) b = min(b, bounds[w]);
    // Where so much is masked that the bound is -inf: of that only the first of the batch, which are the ones with the lowest ids.
    const bool low = b <= image(-INFINITY);
    push<N>(x, low ? image(-INFINITY) + 1 : b, base, per, far, there, lane, low && warp == 0 ? (1u << per) - 1 : 0);
  }
  // The best 32 to the buffer's beginning, in order.  All threads, behind a barrier.
  __device__ __forceinline__ void cut(int n, int warp, int lane) {
    const int c = min(*count, room), chunks = (c + 31) / 32;
    u64 mine = 0;
    for (int i = warp; i < chunks; i += WARPS) {
      const u64 x = sorted(i * 32 + lane < c ? buffer[i * 32 + lane] : 0, lane);
      mine = i == warp ? x : merged(mine, x, lane);
    }
#pragma unroll
    for (int half = WARPS / 2; half; half >>= 1) {
      if (chunks <= half) continue;                // (no list there; the same for all)
      if (warp >= half && warp < 2 * half) lists[warp * 32 + lane] = mine;
      __syncthreads();
      if (warp < half) mine = merged(mine, lists[(warp + half) * 32 + lane], lane);
      __syncthreads();
    }
    if (chunks <= 1) __syncthreads();              // (everybody knows the count)
    if (warp == 0) {
      buffer[lane] = mine;
      if (lane == 0) *count = min(c, n);
    }
    __syncthreads();
    const uint32_t im = (uint32_t)(buffer[n - 1] >> 32);
    full = im != 0;                                // (what comes later has higher ids: equals are no candidates)
    last = full ? value_of(im) : 0.f;
    much = false;
    __syncthreads();
  }
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t of_rank(uint32_t addr, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ u64 peer_u64(uint32_t addr) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float peer_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// (128 threads: 7 CTAs of 72 registers on an SM, 2048 x 64000 with 20 alternatives 96 us; 8 spill in the loop, 104; 6: 106.  256: 4, with 3 512
// rows of 32000 take two rounds: 23 us for 32.)
template <typename T, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 128 ? 7 : 4) token_logprobs_kernel(const ScoreParams p) {
  constexpr int WARPS = THREADS / 32, BUFFER = Best<THREADS>::BUFFER;
  constexpr int VEC = 16 / sizeof(T), NV = E / VEC;               // logits of a load, loads at a time
  // Batches on their way: each thread copies its own vectors and waits for its own, so that no barrier stands between, and a cut keeps no load
  // waiting.  (us with 1, 2, 3 of 128 threads: 2048 x 64000 f32, 20 alternatives 102, 96, 101, without 82, 80, 85; through registers 107 and 81.  With
  // 1, 2 of 256 threads: one row of 130000 11.2, 11.3, 512 of 32000 22.9, 23.8.)
  constexpr int STAGES = THREADS == 128 ? 2 : 1, RING = STAGES * NV * THREADS * 16;
  // The ring, and behind it the candidates; a row that is done again has all of it for its candidates.
  constexpr int POOL = !TOP ? RING : RING + SMALL * 8 > BUFFER * 8 ? RING + SMALL * 8 : BUFFER * 8;
  __shared__ __align__(16) uint8_t s_pool[POOL];
  __shared__ u64 s_list[TOP ? WARPS * 32 : 1];
  __shared__ Sums s_sums[WARPS];
  __shared__ float s_more;
  __shared__ int s_peak[THREADS];
  __shared__ int s_count, s_noted, s_notes[TOP ? NOTES : 1];
  __shared__ uint32_t s_bounds[WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / p.ctas, rank = blockIdx.x - row * p.ctas;
  pdl_wait();
  pdl_trigger();
  const T *x0 = (const T *)p.logits + (int64_t)row * p.row_stride;
  const int token = p.tokens && rank == 0 ? p.tokens[row] : -1;
  // Every load's address lies in the row; what was not to be read is masked afterwards.  (Guarding the load instead, with its value undefined
  // otherwise, lets the compiler drop the guard.)
  const bool known = token >= 0 && token < p.vocab;
  const float x_token = known ? one(x0 + (known ? token : 0)) : -INFINITY;
  const int lead = min(p.vocab, (int)((16 - ((uintptr_t)x0 & 15)) & 15) / (int)sizeof(T));   // in front of the first whole 16 bytes
  const int vecs = (p.vocab - lead) / VEC, tail = p.vocab - lead - vecs * VEC;
  const int v_begin = (int)((int64_t)vecs * rank / p.ctas), v_end = (int)((int64_t)vecs * (rank + 1) / p.ctas);
  const uint4 *xv = (const uint4 *)(x0 + lead);

  Sums sum{-FLT_MAX, -1.f, 0.f};
  s_peak[tid] = -1;                                                // the batch in which this thread's maximum is (its first vector)
  Best<THREADS> best{(u64 *)(s_pool + RING), (POOL - RING) / 8, s_list, &s_count, s_notes, &s_noted, s_bounds, 0.f, false, false, false};
  // The maximum covers top, which is in batch `at`; what of the new maximum's own 1 will be added to r.
  auto grow = [&](float top, int at) {
    const float m = max_nan(sum.m, top);
    if (m == sum.m) return 0.f;
    const float d = sum.m - m, f = ex2(d * LOG2E), z = 1.f + sum.r;
    sum.t = f > 0.f ? fmaf(d, z, sum.t) * f : 0.f;
    sum.r = z * f;
    sum.m = m;
    s_peak[tid] = at;
    return 1.f;
  };
  auto add_one = [&](float x) {
    const float own = grow(x, -1);
    const float d = x - sum.m, e = ex2(d * LOG2E);
    sum.r += e - own;
    if (e > 0.f) sum.t = fmaf(d, e, sum.t);                        // (-inf: nothing)
  };
  bool masked = false;                                             // this thread has met logits of -inf
  auto add = [&](const float *x, float top, int at) {
    const float own = grow(top, at);
    const u64 m2 = pair(-sum.m, -sum.m), l2 = pair(LOG2E, LOG2E);
    u64 z2 = 0, t2 = pair(sum.t, 0.f);
    if (!masked) {
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const u64 d = add2(pair(x[i], x[i + 1]), m2);
        float a, b;
        unpair(mul2(d, l2), a, b);
        const u64 e = pair(ex2(a), ex2(b));
        z2 = add2(z2, e);
        t2 = fma2(d, e, t2);
      }
    }
    float z0, z1, t0, t1;
    unpair(t2, t0, t1);
    if (masked || t0 + t1 != t0 + t1) {                            // -inf times 0 (or something that is no number, which r shows)
      masked = true;
      z2 = 0;
      t0 = sum.t;
      t1 = 0.f;
#pragma unroll
      for (int i = 0; i < E; i += 2) {
        const u64 d = add2(pair(x[i], x[i + 1]), m2);
        float a, b, d0, d1;
        unpair(mul2(d, l2), a, b);
        a = ex2(a);
        b = ex2(b);
        z2 = add2(z2, pair(a, b));
        unpair(d, d0, d1);
        if (a > 0.f) t0 = fmaf(d0, a, t0);
        if (b > 0.f) t1 = fmaf(d1, b, t1);
      }
    }
    unpair(z2, z0, z1);
    sum.r += (z0 + z1) - own;
    sum.t = t0 + t1;
  };
  constexpr int STEP = NV * THREADS;
  const uint32_t ring = smem_u32(s_pool) + tid * 16;
  int stage = 0;
  auto fetch = [&](int v0, int st) {
    if (v0 < v_end) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + (st * NV + j) * THREADS * 16), "l"(xv + min(v0 + j * THREADS + tid, v_end - 1)) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // The logits in raw (-inf where the row ends), their largest and which of the vectors there are.
  auto have = [&](const uint4 *raw, int v0, float *x, float &top, uint32_t &there) {
    unpack16<T>(raw, x);
    there = (1u << NV) - 1;
    if (v0 + STEP > v_end) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (v0 + j * THREADS + tid >= v_end) {
          there &= ~(1u << j);
#pragma unroll
          for (int i = 0; i < VEC; ++i) x[j * VEC + i] = -INFINITY;
        }
    }
    top = max_nan(max_nan(x[0], x[1]), x[2], x[3]);
#pragma unroll
    for (int i = 4; i < E; i += 4) top = max_nan(top, max_nan(x[i], x[i + 1]), max_nan(x[i + 2], x[i + 3]));
  };
  auto take = [&](int v0, float *x, float &top, uint32_t &there) {  // the next batch of the ring; another is asked for in its place
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
    uint4 raw[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(raw[j].x), "=r"(raw[j].y), "=r"(raw[j].z), "=r"(raw[j].w)
                   : "r"(ring + (stage * NV + j) * THREADS * 16)
                   : "memory");
    have(raw, v0, x, top, there);
    fetch(v0 + STAGES * STEP, stage);
    stage = stage == STAGES - 1 ? 0 : stage + 1;
  };
  auto id_of = [&](int v0) { return (uint32_t)lead + (uint32_t)(v0 + tid) * VEC; };
  // What is in front of the first and behind the last whole 16 bytes (at most 7 each).
  auto ends = [&](bool front, bool sums) {
    if (rank != 0 || warp != 0) return;
    const int many = front ? lead : tail, id = front ? lane : lead + vecs * VEC + lane;
    if (many == 0) return;
    const float x = lane < many ? one(x0 + min(id, p.vocab - 1)) : -INFINITY;
    if (sums) add_one(x);
    if constexpr (TOP) best.template offer<1>(&x, x, id, 1, 0, lane < many, p.n_top, lane);
  };
  auto begin = [&]() {
    best.full = best.much = best.over = false;
    if (tid == 0) s_count = s_noted = 0;
    __syncthreads();
  };

  if (TOP) begin();
  ends(true, true);
  if (v_begin < v_end) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) fetch(v_begin + i * STEP, i);
    float x[E], top;
    uint32_t there;
    int v0 = v_begin, cut_at = v_begin + (GROWTH - 1) * STEP;      // the first logit of the batch behind which the next cut is
    if constexpr (TOP) {
      take(v0, x, top, there);
      add(x, top, v0 + tid);
      best.template begin<E>(x, top, id_of(v0), VEC, THREADS * VEC, there, p.n_top, warp, lane);
      v0 += STEP;
      if (v0 < v_end) {
        __syncthreads();
        best.cut(p.n_top, warp, lane);
      }
    }
    for (; v0 < v_end; v0 += STEP) {
      take(v0, x, top, there);
      add(x, top, v0 + tid);
      if constexpr (TOP) {
        if (there) best.note(top, v0 + tid);
        if (v0 == cut_at && v0 + STEP < v_end) {                   // (what is in the buffer then has lower ids than what is noted later: ties go to them)
          cut_at = v_begin + GROWTH * (cut_at - v_begin) + (GROWTH - 1) * STEP;
          __syncthreads();
          best.template look<T>(xv, v_end, lead);
          __syncthreads();
          if (tid == 0) s_noted = 0;
          best.cut(p.n_top, warp, lane);
        }
      }
    }
  }
  ends(false, true);
  if constexpr (TOP) {
    __syncthreads();
    best.template look<T>(xv, v_end, lead);
    if (__syncthreads_or(best.over)) {                             // the alternatives again, with a look at the buffer after every batch
      best.buffer = (u64 *)s_pool;
      best.room = BUFFER;
      begin();
      ends(true, false);
      for (int v0 = v_begin; v0 < v_end; v0 += STEP) {
        float x[E], top;
        uint32_t there;
        uint4 raw[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) raw[j] = xv[min(v0 + j * THREADS + tid, v_end - 1)];
        have(raw, v0, x, top, there);
        best.template offer<E>(x, top, id_of(v0), VEC, THREADS * VEC, there, p.n_top, lane);
        if (__syncthreads_or(best.much || !best.full) && v0 + STEP < v_end) best.cut(p.n_top, warp, lane);
      }
      ends(false, false);
    }
  }

  // ---- the threads', the warps' and the CTAs' parts
  auto reduce = [&](int lanes) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      if (o >= lanes) continue;
      const Sums b{__shfl_xor_sync(0xffffffffu, sum.m, o), __shfl_xor_sync(0xffffffffu, sum.r, o), __shfl_xor_sync(0xffffffffu, sum.t, o)};
      join(sum, b);
    }
  };
  const float own_m = sum.m;
  reduce(32);
  if (lane == 0) s_sums[warp] = sum;
  if (tid == 0) s_more = 0.f;
  __syncthreads();
  if (TOP) best.cut(p.n_top, warp, lane);
  u64 mine = TOP ? best.buffer[lane] : 0;
  if (TOP && p.ctas > 1 && warp == 0) s_list[lane] = mine;
  sum = s_sums[lane & (WARPS - 1)];
  reduce(WARPS);                                                   // (every warp has the CTA's now)
  // Where one logit has nearly everything, ln Z is what the others leave, and the sixteen that it was added with, rounded beside its 1, are added
  // once more without it.  (Some 1e-7 of Z: behind 1 / 4 less than 5e-7 of ln Z.  0.3 us for a row that needs it.)
  if (__shfl_sync(0xffffffffu, sum.r, 0) < 0.25f) {
    const int peak = s_peak[tid];
    if (own_m == sum.m && peak >= 0) {                             // (one thread: two that are equal make r 1)
      uint4 again[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) again[j] = xv[min(peak + j * THREADS, v_end - 1)];
      float x[E], rest = 0.f, equal = -1.f;
      unpack16<T>(again, x);
      const u64 m2 = pair(-own_m, -own_m), l2 = pair(LOG2E, LOG2E);
      u64 z2 = 0;
#pragma unroll
      for (int i = 0; i < E; i += 2) {                             // (as above: the same roundings, which go)
        float a, b;
        if (peak + i / VEC * THREADS >= v_end) x[i] = x[i + 1] = -INFINITY;
        unpair(mul2(add2(pair(x[i], x[i + 1]), m2), l2), a, b);
        a = ex2(a);
        b = ex2(b);
        z2 = add2(z2, pair(a, b));
        if (x[i] == own_m) equal += 1.f; else rest += a;
        if (x[i + 1] == own_m) equal += 1.f; else rest += b;
      }
      float z0, z1;
      unpair(z2, z0, z1);
      s_more = (rest + equal) - ((z0 + z1) - 1.f);
    }
    __syncthreads();
    sum.r += s_more;
  }
  if (p.ctas > 1) {
    __syncthreads();
    if (tid == 0) s_sums[0] = sum;
    cluster_barrier();
    if (rank == 0 && warp == 0) {
      sum = Sums{-FLT_MAX, -1.f, 0.f};
      if (lane < p.ctas) {
        const uint32_t a = of_rank(smem_u32(&s_sums[0]), lane);
        sum = Sums{peer_f32(a), peer_f32(a + 4), peer_f32(a + 8)};
      }
      reduce(32);
      if (TOP)
        for (int i = 1; i < p.ctas; ++i) mine = merged(mine, peer_u64(of_rank(smem_u32(&s_list[lane]), i)), lane);
    }
    cluster_barrier();                                             // (everybody has been read)
    if (rank != 0) return;
  }
  if (warp != 0) return;
  const bool none = sum.r == -1.f;
  // ln (1 + r) = 2 artanh(s), s = r / (2 + r): four terms leave 3e-9 of it at r = 1 / 4
  const float s = sum.r / (2.f + sum.r), s2 = s * s;
  const float lnz = sum.r < 0.25f ? 2.f * s * fmaf(s2, fmaf(s2, fmaf(s2, 1.f / 7, 1.f / 5), 1.f / 3), 1.f) : logf(1.f + sum.r);
  if (lane == 0) {
    if (p.logprob) p.logprob[row] = none || x_token == -INFINITY ? (sum.r != sum.r && known ? NAN : -INFINITY) : (x_token - sum.m) - lnz;
    if (p.entropy) p.entropy[row] = none ? 0.f : lnz - sum.t / (1.f + sum.r);
  }
  if (TOP && lane < p.n_top) {
    p.top_ids[(int64_t)row * p.n_top + lane] = (int32_t)(0xffffffffu - (uint32_t)mine);
    p.top_logprobs[(int64_t)row * p.n_top + lane] = none ? -INFINITY : (value_of((uint32_t)(mine >> 32)) - sum.m) - lnz;
  }
}

template <typename T, int THREADS>
cudaError_t launch(const ScoreParams &p, int rows, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)rows * p.ctas);
  cfg.blockDim = dim3(THREADS);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = p.ctas;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = p.ctas > 1 ? 2 : 1;
  return p.n_top > 0 ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, true, THREADS>, p) : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, false, THREADS>, p);
}

}  // namespace

extern "C" int ouro_token_logprobs(const void *logits, int32_t dtype, int64_t row_stride, int32_t rows, int32_t vocab, const int32_t *tokens, int32_t n_top,
                                   float *logprob, float *entropy, int32_t *top_ids, float *top_logprobs, void *stream) {
  const char *call = "ouro_token_logprobs";
  if (dtype != OURO_F32 && dtype != OURO_BF16) return paged::refuse(call, "dtype is neither OURO_F32 nor OURO_BF16");
  if (rows < 0 || rows > (1 << 24) || vocab < 1) return paged::refuse(call, "rows is below 0 or above 2^24, or vocab below 1");
  if (n_top < 0 || n_top > OURO_MAX_TOP || n_top > vocab) return paged::refuse(call, "n_top is below 0, above OURO_MAX_TOP or above vocab");
  if (rows == 0) return OURO_OK;
  if (!logits) return paged::refuse(call, "logits is NULL");
  if ((tokens == nullptr) != (logprob == nullptr)) return paged::refuse(call, "tokens and logprob come together");
  if ((n_top > 0) != (top_ids != nullptr) || (n_top > 0) != (top_logprobs != nullptr)) return paged::refuse(call, "the top arrays come with n_top > 0");
  if ((uintptr_t)logits % (dtype == OURO_F32 ? 4 : 2)) return paged::refuse(call, "logits is not aligned to its type");
  if (!paged::words(tokens, logprob, entropy, top_ids, top_logprobs)) return paged::refuse(call, "tokens or an output is not 4-byte aligned");
  if (row_stride < vocab && rows > 1) return paged::refuse(call, "row_stride is below vocab");
  int dev = 0, sms = 0;
  if (!paged::device(&dev, &sms)) return paged::refuse(call, "no usable current device", OURO_ECUDA);
  ScoreParams p{logits, row_stride, tokens, logprob, entropy, top_ids, top_logprobs, vocab, n_top, 1};
  while (p.ctas < 8 && (int64_t)rows * p.ctas < 2 * sms && vocab / (2 * p.ctas) >= 2048) p.ctas *= 2;
  // A row's fixed costs grow with its warps, its latency falls: 128 threads where there are more rows than SMs hold of 256 threads' at once, or
  // where a row is one batch of 256.  (us with 256 / 128 threads, 20 alternatives: one row of 130000 11.2 / 14.1, 128 of 32000 14.3 / 15.4, 512 23.2 /
  // 22.6, 512 that ascend 158 / 188, 700 35 / 29, 1000 41 / 31, 2048 of 64000 117 / 96; 5 alternatives: 2048 of 1024 28 / 15.)
  const bool few = rows <= 4 * sms && vocab > 4096;
  cudaError_t e;
  if (dtype == OURO_F32) e = few ? launch<float, 256>(p, rows, (cudaStream_t)stream) : launch<float, 128>(p, rows, (cudaStream_t)stream);
  else e = few ? launch<__nv_bfloat16, 256>(p, rows, (cudaStream_t)stream) : launch<__nv_bfloat16, 128>(p, rows, (cudaStream_t)stream);
  OURO_COUNT_LAUNCH();
  return e == cudaSuccess ? OURO_OK : paged::refuse(call, cudaGetErrorString(e), OURO_ECUDA);
}
