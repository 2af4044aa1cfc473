// Rules on which tokens may come, on rows of logits: penalties for tokens that a text has already, biases, grammar masks.
//
//     c = how often the row's history has the token
//     y = x;  where c > 0:  y = y > 0 ? y / repetition : y * repetition,  y -= frequency * c + presence;   y += bias;   not allowed: y = -inf
//
// Bound by HBM: a logit is read and written once.  The counts never leave the SM: a CTA has a slice of a row, clears a count in shared memory for every
// token of it, goes through the row's whole history (a few KB, from L2 but for the first CTA) and adds up what falls into the slice.  Its logits are asked
// for before that and are there when the counts are.  Counts are whole numbers, so that the order of additions changes nothing.
#include "paged.h"
#include "row_ops.cuh"

namespace {

struct ConstrainParams {
  const void *in;
  void *out;
  const int32_t *tokens, *lens;
  const float *repetition, *presence, *frequency, *bias;
  const uint32_t *allowed;
  int64_t in_stride, out_stride, token_stride, bias_stride, allowed_stride;
  int rows, vocab, width, slices;
};
constexpr int THREADS = 256;

template <typename T> struct Piece;                // 16 bytes of logits
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4 &t, float *x) {
    x[0] = __uint_as_float(t.x); x[1] = __uint_as_float(t.y); x[2] = __uint_as_float(t.z); x[3] = __uint_as_float(t.w);
  }
  static __device__ __forceinline__ uint4 pack(const float *x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  static __device__ __forceinline__ float get(const float *p) { return *p; }
  static __device__ __forceinline__ void put(float *p, float x) { *p = x; }
};
template <> struct Piece<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4 &t, float *x) {
    const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint4 pack(const float *x) {
    return make_uint4(rowops::pack(x[0], x[1]), rowops::pack(x[2], x[3]), rowops::pack(x[4], x[5]), rowops::pack(x[6], x[7]));
  }
  static __device__ __forceinline__ float get(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void put(__nv_bfloat16 *p, float x) { *p = __float2bfloat16_rn(x); }
};

// A slice has U pieces a thread.  Pieces begin where the row's addresses are multiples of 16 bytes: the row's first may begin in front of it, its last
// may end behind it; those two go element by element, and all do where the output's row is aligned differently.
template <typename T, int U, bool COUNTS>
__global__ void __launch_bounds__(THREADS) constrain_kernel(const ConstrainParams p) {
  using P = Piece<T>;
  constexpr int N = P::N, SLICE = THREADS * N * U;
  __shared__ __align__(16) uint32_t s_count[COUNTS ? SLICE : 1];
  const int tid = threadIdx.x, row = blockIdx.x / p.slices, slice = blockIdx.x - row * p.slices;
  const T *in = (const T *)p.in + row * p.in_stride;
  T *out = (T *)p.out + row * p.out_stride;
  const int skew = (int)((uintptr_t)in % 16 / sizeof(T));          // elements of the first piece in front of the row
  const bool alike = (int)((uintptr_t)out % 16 / sizeof(T)) == skew;
  const int base = slice * SLICE - skew;                           // token of the slice's first element
  if (COUNTS)
    for (int i = tid; i < SLICE / 4; i += THREADS) ((uint4 *)s_count)[i] = make_uint4(0, 0, 0, 0);
  pdl_wait();
  pdl_trigger();
  const float *bias = p.bias ? p.bias + row * p.bias_stride : nullptr;
  const uint32_t *allowed = p.allowed ? p.allowed + row * p.allowed_stride : nullptr;
  // (the mask's words as early as the logits: 64 rows of 32000 5.5 -> 4.4 us, 1000 of 64000 91 -> 89, in bf16 75 -> 71; the biases too would take 22 registers
  // more, and with them a CTA of five: 98)
  uint4 raw[U];
  uint32_t bits_lo[U], bits_hi[U];                                 // the words of the mask with a piece's first and last bit
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int e0 = base + (u * THREADS + tid) * N;
    if (alike && e0 >= 0 && e0 + N <= p.vocab) {
      raw[u] = __ldcs((const uint4 *)(in + e0));
      if (allowed) {
        bits_lo[u] = __ldg(allowed + (e0 >> 5));
        bits_hi[u] = __ldg(allowed + ((e0 + N - 1) >> 5));
      }
    }
  }
  float rep = 1.f, pres = 0.f, freq = 0.f;
  if (COUNTS) {
    __syncthreads();
    const int len = p.lens ? min(max(p.lens[row], 0), p.width) : p.width;
    const int32_t *told = p.tokens + row * p.token_stride;
    const int lo = max(base, 0), here = max(min(base + SLICE, p.vocab) - lo, 0);        // tokens of the slice
    auto count = [&](int t) {
      if ((uint32_t)(t - lo) < (uint32_t)here) atomicAdd(&s_count[t - base], 1u);
    };
    const int head = min(len, (int)((16 - (uintptr_t)told % 16) % 16 / 4)), fours = (len - head) / 4;
    const int4 *told4 = (const int4 *)(told + head);
    for (int i = tid; i < fours; i += 2 * THREADS) {               // eight tokens under way at once
      const int4 a = told4[i], b = i + THREADS < fours ? told4[i + THREADS] : make_int4(-1, -1, -1, -1);
      count(a.x); count(a.y); count(a.z); count(a.w);
      count(b.x); count(b.y); count(b.z); count(b.w);
    }
    if (tid < head) count(told[tid]);
    if (tid < len - head - 4 * fours) count(told[head + 4 * fours + tid]);
    if (p.repetition) rep = p.repetition[row];
    if (p.presence) pres = p.presence[row];
    if (p.frequency) freq = p.frequency[row];
    __syncthreads();
  }
  // A product with the reciprocal is 2^-23 of the quotient off at most.  (Where histories are long, nearly every
  // 128 logits of a warp have somebody's token: 1000 rows of 64000 took 173 us with divisions behind branches.)
  const float inv = 1.f / rep;
  auto told_of = [&](float x, uint32_t c) {
    const float n = __uint_as_float(c | 0x4b000000u) - 8388608.f;   // c below 2^23, without the slow conversion
    const float y = __fsub_rn(__fmul_rn(x, x > 0.f ? inv : rep), fmaf(freq, n, pres));
    return c ? y : x;
  };
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int local = (u * THREADS + tid) * N, e0 = base + local;
    if (e0 >= p.vocab) break;
    if (alike && e0 >= 0 && e0 + N <= p.vocab) {
      float x[N];
      P::unpack(raw[u], x);
      if (COUNTS) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
          const uint4 c = *(const uint4 *)(s_count + local + i);
          if (c.x | c.y | c.z | c.w) {
            x[i] = told_of(x[i], c.x);
            x[i + 1] = told_of(x[i + 1], c.y);
            x[i + 2] = told_of(x[i + 2], c.z);
            x[i + 3] = told_of(x[i + 3], c.w);
          }
        }
      }
      if (bias) {
        if (((uintptr_t)(bias + e0) & 15) == 0) {
#pragma unroll
          for (int i = 0; i < N; i += 4) {
            const float4 b = __ldg((const float4 *)(bias + e0 + i));
            x[i] += b.x; x[i + 1] += b.y; x[i + 2] += b.z; x[i + 3] += b.w;
          }
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] += bias[e0 + i];
        }
      }
      if (allowed) {
        const uint32_t bits = __funnelshift_r(bits_lo[u], bits_hi[u], e0 & 31);
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (!(bits >> i & 1)) x[i] = -INFINITY;
      }
      __stcs((uint4 *)(out + e0), P::pack(x));
    } else {
      for (int i = 0; i < N; ++i) {
        const int e = e0 + i;
        if (e < 0 || e >= p.vocab) continue;
        float x = P::get(in + e);
        if (COUNTS && s_count[local + i]) x = told_of(x, s_count[local + i]);
        if (bias) x += bias[e];
        if (allowed && !(allowed[e >> 5] >> (e & 31) & 1)) x = -INFINITY;
        P::put(out + e, x);
      }
    }
  }
}

template <typename T, int U>
cudaError_t launch(ConstrainParams p, cudaStream_t s) {
  constexpr int SLICE = THREADS * Piece<T>::N * U;
  p.slices = (int)(((int64_t)p.vocab + Piece<T>::N - 1 + SLICE - 1) / SLICE);    // (a row may begin N - 1 elements behind its first piece)
  const dim3 grid((unsigned)(p.slices * p.rows));
  return p.tokens ? launch_pdl(constrain_kernel<T, U, true>, grid, dim3(THREADS), 0, s, p) : launch_pdl(constrain_kernel<T, U, false>, grid, dim3(THREADS), 0, s, p);
}
// Small slices end sooner while all of them are under way at once; the more there are, the more it counts that every slice goes through the row's whole history.
// us a launch (histories of 512, penalty and mask; U of 1 / of 4) with 1, 8, 20, 40, 128 rows of 32000 and 1000 rows of 64000 with histories of 2048:
//     f32   1.8/2.3, 2.0/2.4, 3.4/2.7, 4.3/3.3, 11.1/6.3, 172/89        bf16   1.9/2.8, 2.0/2.8, 2.4/2.9, 4.0/3.4, 7.0/5.8, 102/59
// (1000 rows with U of 2, 4, 8: f32 113, 89, 92, bf16 71, 59, 82; CTAs of 128 threads with 4 and 8: 102, 101 and 68, 82, of 512 with 4: 107 and 73.)
template <typename T>
cudaError_t by_size(const ConstrainParams &p, int sms, cudaStream_t s) {
  const int64_t pieces = (int64_t)p.rows * (p.vocab / Piece<T>::N + 1);
  return pieces < (int64_t)sms * THREADS * 3 ? launch<T, 1>(p, s) : launch<T, 4>(p, s);
}

}  // namespace

extern "C" int ouro_constrain_logits(const void *logits, int32_t dtype, int64_t row_stride, int32_t rows, int32_t vocab, const int32_t *tokens,
                                     int64_t token_stride, int32_t width, const int32_t *lens, const float *repetition, const float *presence,
                                     const float *frequency, const float *bias, int64_t bias_stride, const uint32_t *allowed, int64_t allowed_stride,
                                     void *out, int64_t out_stride, void *stream) {
  const char *call = "ouro_constrain_logits";
  if (dtype != OURO_F32 && dtype != OURO_BF16) return paged::refuse(call, "dtype is neither OURO_F32 nor OURO_BF16");
  if (rows < 0 || rows > (1 << 24) || vocab < 1 || vocab > (1 << 28)) return paged::refuse(call, "rows is below 0 or above 2^24, or vocab below 1 or above 2^28");
  if ((int64_t)rows * (vocab / 1024 + 2) > INT32_MAX) return paged::refuse(call, "rows * vocab is above 2^41");
  if (rows == 0) return OURO_OK;
  if (!logits || !out) return paged::refuse(call, "logits or out is NULL");
  const int e = dtype == OURO_F32 ? 4 : 2;
  if (((uintptr_t)logits | (uintptr_t)out) % e) return paged::refuse(call, "logits or out is not aligned to its type");
  if (!paged::words(tokens, lens, repetition, presence, frequency, bias, allowed)) return paged::refuse(call, "an array of 32-bit numbers is not 4-byte aligned");
  if (rows > 1 && (row_stride < vocab || out_stride < vocab)) return paged::refuse(call, "row_stride or out_stride is below vocab");
  if (logits == out && rows > 1 && row_stride != out_stride) return paged::refuse(call, "out is logits, with other rows");
  if (tokens) {
    if (width < 0 || width >= 1 << 23 || (rows > 1 && token_stride < width && token_stride != 0)) return paged::refuse(call, "width is below 0 or above 2^23 - 1, or token_stride below width");
  } else if (lens || repetition || presence || frequency) {
    return paged::refuse(call, "lens and penalties come with tokens");
  }
  const int words = (vocab + 31) / 32;
  if (bias && rows > 1 && bias_stride != 0 && bias_stride < vocab) return paged::refuse(call, "bias_stride is neither 0 nor a row's length");
  if (allowed && rows > 1 && allowed_stride != 0 && allowed_stride < words) return paged::refuse(call, "allowed_stride is neither 0 nor a row's length");
  int dev = 0, sms = 0;
  if (!paged::device(&dev, &sms)) return paged::refuse(call, "no usable current device", OURO_ECUDA);
  ConstrainParams p{};
  p.in = logits; p.out = out; p.tokens = tokens; p.lens = lens;
  p.repetition = repetition; p.presence = presence; p.frequency = frequency; p.bias = bias; p.allowed = allowed;
  p.in_stride = row_stride; p.out_stride = out_stride; p.token_stride = token_stride; p.bias_stride = bias_stride; p.allowed_stride = allowed_stride;
  p.rows = rows; p.vocab = vocab; p.width = width;
  const cudaError_t r = dtype == OURO_F32 ? by_size<float>(p, sms, (cudaStream_t)stream) : by_size<__nv_bfloat16>(p, sms, (cudaStream_t)stream);
  OURO_COUNT_LAUNCH();
  return r == cudaSuccess ? OURO_OK : paged::refuse(call, cudaGetErrorString(r), OURO_ECUDA);
}
