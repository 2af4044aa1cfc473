// Log probabilities of given tokens, entropy and the best alternatives of every row of logits, in one pass over the logits.
//
//     m = max x,  Z = sum e^(x - m),  T = sum (x - m) e^(x - m)
//     log p(t) = (x_t - m) - ln Z,    H = ln Z - T / Z
//
// Bound by HBM: a logit is read once and costs a dozen instructions.  A row is a CTA's or, where rows are few, a cluster's, whose
// CTAs join through shared memory: one launch, no workspace.
//  - A thread keeps (m, Z, T) of what it has seen, in 32 bits, relative to its own maximum, sixteen logits at a time.
//  - A warp keeps the best alternatives it has seen sorted over its lanes, as 64-bit keys (value in an order-preserving integer image,
//    then the complement of the id: no two are equal, and the lowest id is first among equals).  The maximum of a thread's sixteen logits, which
//    the sum needs anyway, is compared to the last of them; only where it is larger does anybody look closer.  Where many lanes have something
//    to offer (at the beginning, or in rows that ascend), the n-th largest of the lanes' maxima is found first: what is below it cannot be
//    among the best n.
#include "paged.h"
#include "row_ops.cuh"

#include <cfloat>

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int E = 16;                              // logits of a thread at a time
constexpr int CROWD = 8;                           // lanes with something to offer from which on the maxima are sorted first
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
// Integer image of a logit: larger logit, larger integer; NaN above all, -0 like +0; never 0.
__device__ __forceinline__ uint32_t image(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return x != x ? 0xffffffffu : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t im) {
  return im == 0xffffffffu ? NAN : __uint_as_float(im & 0x80000000u ? im ^ 0x80000000u : ~im);
}

struct Sums {
  float m, z, t;
};
// Adds what b has seen to a.
__device__ __forceinline__ void join(Sums &a, const Sums &b) {
  const float m = max_nan(a.m, b.m);
  const float da = a.m - m, db = b.m - m, fa = ex2(da * LOG2E), fb = ex2(db * LOG2E);
  // (a factor of 0 leaves nothing of T either, however far apart the maxima are; a NaN is kept by Z)
  const float ta = fa > 0.f ? fmaf(da, a.z, a.t) * fa : 0.f, tb = fb > 0.f ? fmaf(db, b.z, b.t) * fb : 0.f;
  a.z = a.z * fa + b.z * fb;
  a.t = ta + tb;
  a.m = m;
}

// Lists of 32 keys over a warp's lanes, largest first.
__device__ __forceinline__ u64 sorted(u64 x, int lane) {          // x is bitonic
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const u64 y = __shfl_xor_sync(0xffffffffu, x, o);
    x = (lane & o) == 0 ? (x > y ? x : y) : (x > y ? y : x);
  }
  return x;
}
__device__ __forceinline__ u64 merged(u64 a, u64 b, int lane) {   // the best 32 of two lists
  b = __shfl_sync(0xffffffffu, b, 31 - lane);
  return sorted(a > b ? a : b, lane);
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
__device__ __forceinline__ float one(const float *p) { return __ldg(p); }
__device__ __forceinline__ float one(const __nv_bfloat16 *p) { return __bfloat162float(__ldg(p)); }

// The best alternatives a warp has seen.
struct Best {
  u64 mine = 0;                                    // lane i: the i-th best, 0: none yet
  float last = 0.f;                                // value of the n-th
  bool full = false;                               // there are n

  __device__ __forceinline__ void insert(u64 k, int lane) {
    const int at = __popc(__ballot_sync(0xffffffffu, mine > k));
    const u64 up = __shfl_up_sync(0xffffffffu, mine, 1);
    mine = lane < at ? mine : lane == at ? k : up;
  }
  // N logits of every lane: x[i] has id base + i % per + (i / per) * far, if bit i / per of there is set; top: the largest of them
  // (NaN where there is one).
  template <int N>
  __device__ __forceinline__ void offer(const float *x, float top, uint32_t base, int per, uint32_t far, uint32_t there, int n, int lane) {
    const uint32_t some = __ballot_sync(0xffffffffu, there != 0 && (!full || !(top <= last)));
    if (some == 0) return;
    uint32_t bound = full ? image(last) + 1 : 1;
    if (__popc(some) >= CROWD) {
      uint32_t s = there ? image(top) : 0;
#pragma unroll
      for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int o = k >> 1; o; o >>= 1) {
          const uint32_t y = __shfl_xor_sync(0xffffffffu, s, o);
          s = ((lane & o) == 0) == ((lane & k) == 0 || k == 32) ? max(s, y) : min(s, y);
        }
      bound = max(bound, __shfl_sync(0xffffffffu, s, n - 1));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t im = image(x[i]), id = base + i % per + (uint32_t)(i / per) * far;
      uint32_t who = __ballot_sync(0xffffffffu, (there >> (i / per) & 1) && im >= bound);
      while (who) {
        const int src = __ffs(who) - 1;
        who &= who - 1;
        insert((u64)__shfl_sync(0xffffffffu, im, src) << 32 | (0xffffffffu - __shfl_sync(0xffffffffu, id, src)), lane);
      }
    }
    const uint32_t nth = (uint32_t)(__shfl_sync(0xffffffffu, mine, n - 1) >> 32);
    full = nth != 0;
    last = full ? value_of(nth) : 0.f;
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

template <typename T, bool TOP>
__global__ void __launch_bounds__(THREADS) token_logprobs_kernel(const ScoreParams p) {
  constexpr int VEC = 16 / sizeof(T), NV = E / VEC;               // logits of a load, loads at a time
  __shared__ u64 s_list[WARPS][32];
  __shared__ Sums s_sums[WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / p.ctas, rank = blockIdx.x - row * p.ctas;
  pdl_wait();
  pdl_trigger();
  const T *x0 = (const T *)p.logits + (int64_t)row * p.row_stride;
  const int token = p.tokens && rank == 0 ? __ldg(p.tokens + row) : -1;
  const float x_token = token >= 0 && token < p.vocab ? one(x0 + token) : -INFINITY;
  const int lead = min(p.vocab, (int)((16 - ((uintptr_t)x0 & 15)) & 15) / (int)sizeof(T));   // in front of the first whole 16 bytes
  const int vecs = (p.vocab - lead) / VEC, tail = p.vocab - lead - vecs * VEC;
  const int v_begin = (int)((int64_t)vecs * rank / p.ctas), v_end = (int)((int64_t)vecs * (rank + 1) / p.ctas);
  const uint4 *xv = (const uint4 *)(x0 + lead);

  Sums sum{-FLT_MAX, 0.f, 0.f};
  Best best;
  auto add = [&](const float *x, auto n_of, float top) {
    constexpr int N = decltype(n_of)::value;
    const float m = max_nan(sum.m, top);
    if (m != sum.m) {
      const float d = sum.m - m, f = ex2(d * LOG2E);
      sum.t = f > 0.f ? fmaf(d, sum.z, sum.t) * f : 0.f;
      sum.z *= f;
      sum.m = m;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = x[i] - sum.m, e = ex2(d * LOG2E);
      sum.z += e;
      if (e > 0.f) sum.t = fmaf(d, e, sum.t);                      // (-inf: nothing)
    }
  };
  if (rank == 0 && warp == 0 && lead > 0) {                        // (at most 7)
    const float x = lane < lead ? one(x0 + lane) : -INFINITY;
    add(&x, std::integral_constant<int, 1>(), x);
    if constexpr (TOP) best.offer<1>(&x, x, lane, 1, 0, lane < lead, p.n_top, lane);
  }
  uint4 raw[NV];
  auto fetch = [&](int v0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int v = v0 + j * THREADS + tid;
      if (v < v_end) raw[j] = __ldg(xv + v);
    }
  };
  fetch(v_begin);
  for (int v0 = v_begin; v0 < v_end; v0 += NV * THREADS) {
    float x[E];
    unpack16<T>(raw, x);
    uint32_t there = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (v0 + j * THREADS + tid < v_end) {
        there |= 1u << j;
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[j * VEC + i] = -INFINITY;
      }
    }
    if (v0 + NV * THREADS < v_end) fetch(v0 + NV * THREADS);
    float top = x[0];
#pragma unroll
    for (int i = 1; i < E; ++i) top = max_nan(top, x[i]);
    add(x, std::integral_constant<int, E>(), top);
    if constexpr (TOP) best.offer<E>(x, top, (uint32_t)lead + (uint32_t)(v0 + tid) * VEC, VEC, THREADS * VEC, there, p.n_top, lane);
  }
  if (rank == 0 && warp == 0 && tail > 0) {                        // (at most 7)
    const int id = lead + vecs * VEC + lane;
    const float x = lane < tail ? one(x0 + id) : -INFINITY;
    add(&x, std::integral_constant<int, 1>(), x);
    if constexpr (TOP) best.offer<1>(&x, x, id, 1, 0, lane < tail, p.n_top, lane);
  }

  // ---- the threads', the warps' and the CTAs' parts
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const Sums b{__shfl_xor_sync(0xffffffffu, sum.m, o), __shfl_xor_sync(0xffffffffu, sum.z, o), __shfl_xor_sync(0xffffffffu, sum.t, o)};
    join(sum, b);
  }
  auto over_warps = [&](int many) {                                // afterwards in warp 0
    if (lane == 0) s_sums[warp] = sum;
    if (TOP) s_list[warp][lane] = best.mine;
    __syncthreads();
    if (warp == 0) {
      sum = lane < many ? s_sums[lane] : Sums{-FLT_MAX, 0.f, 0.f};
#pragma unroll
      for (int o = WARPS / 2; o; o >>= 1) {
        const Sums b{__shfl_xor_sync(0xffffffffu, sum.m, o), __shfl_xor_sync(0xffffffffu, sum.z, o), __shfl_xor_sync(0xffffffffu, sum.t, o)};
        join(sum, b);
      }
      sum = Sums{__shfl_sync(0xffffffffu, sum.m, 0), __shfl_sync(0xffffffffu, sum.z, 0), __shfl_sync(0xffffffffu, sum.t, 0)};
      if constexpr (TOP)
        for (int w = 1; w < many; ++w) best.mine = merged(best.mine, s_list[w][lane], lane);
    }
  };
  over_warps(WARPS);
  if (p.ctas > 1) {
    __syncthreads();
    if (warp == 0) {
      if (lane == 0) s_sums[0] = sum;
      if (TOP) s_list[0][lane] = best.mine;
    }
    cluster_barrier();
    if (rank == 0) {
      const bool on = warp < p.ctas;
      if (on) {
        const uint32_t a = of_rank(smem_u32(&s_sums[0]), warp), b = of_rank(smem_u32(&s_list[0][lane]), warp);
        sum = Sums{peer_f32(a), peer_f32(a + 4), peer_f32(a + 8)};
        if (TOP) best.mine = peer_u64(b);
      }
    }
    cluster_barrier();                                             // (everybody has been read)
    if (rank != 0) return;
    over_warps(p.ctas);
  }
  if (warp != 0) return;
  const bool none = sum.z == 0.f;
  const float lnz = logf(sum.z);
  if (lane == 0) {
    if (p.logprob) p.logprob[row] = none || x_token == -INFINITY ? (sum.z != sum.z && token >= 0 && token < p.vocab ? NAN : -INFINITY) : (x_token - sum.m) - lnz;
    if (p.entropy) p.entropy[row] = none ? 0.f : lnz - sum.t / sum.z;
  }
  if (TOP && lane < p.n_top) {
    p.top_ids[(int64_t)row * p.n_top + lane] = (int32_t)(0xffffffffu - (uint32_t)best.mine);
    p.top_logprobs[(int64_t)row * p.n_top + lane] = none ? -INFINITY : (value_of((uint32_t)(best.mine >> 32)) - sum.m) - lnz;
  }
}

template <typename T>
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
  return p.n_top > 0 ? cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, true>, p) : cudaLaunchKernelEx(&cfg, token_logprobs_kernel<T, false>, p);
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
  if (row_stride < vocab && rows > 1) return paged::refuse(call, "row_stride is below vocab");
  int dev = 0, sms = 0;
  if (!paged::device(&dev, &sms)) return paged::refuse(call, "no usable current device", OURO_ECUDA);
  ScoreParams p{logits, row_stride, tokens, logprob, entropy, top_ids, top_logprobs, vocab, n_top, 1};
  while (p.ctas < 8 && (int64_t)rows * p.ctas < 2 * sms && vocab / (2 * p.ctas) >= 2048) p.ctas *= 2;
  const cudaError_t e = dtype == OURO_F32 ? launch<float>(p, rows, (cudaStream_t)stream) : launch<__nv_bfloat16>(p, rows, (cudaStream_t)stream);
  OURO_COUNT_LAUNCH();
  return e == cudaSuccess ? OURO_OK : paged::refuse(call, cudaGetErrorString(e), OURO_ECUDA);
}
