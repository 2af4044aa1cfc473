// Rotary positions computed from frequencies, for new queries and keys, and the keys and values into a paged cache.
//
//     (a, b) -> m (a cos t - b sin t, b cos t + a sin t),   t = position * frequency of the pair
//
// for pairs (i, i + rotary_dim / 2) or (2 i, 2 i + 1) of the head's first rotary_dim dims; the others pass.  Bound by HBM: every row is read and written
// once.  There is no table of cosines: a stretched context has a million positions, and a table of them is read a row at a time for nothing.  A row's
// angles are worked out once, a pair a thread, while the row itself is on its way: in turns, position * turns in 64 bits, of which the nearest quarter
// comes off exactly, so that what is left is at most an eighth of a turn and loses nothing in 32 bits (at position 2^31 the fastest pair, a radian a
// position, has made 3.4e8 turns, which 64 bits know to 2^-24 of a turn; at a million to 2^-35).
#include "paged.h"
#include "row_ops.cuh"

namespace {

struct RotaryParams {
  uint8_t *k, *v;                                  // of the layer
  const void *q, *k_new, *v_new;
  void *q_out;
  const int32_t *slots, *positions;
  const double *turns;
  int64_t page_bytes, slot_bytes, head_bytes, q_stride, kv_stride;
  int rows, H, Hkv, D, rotary, page, n_pages;
  float magnitude;
};
constexpr int THREADS = 128;

__device__ __forceinline__ void unpack(uint4 t, float *x, float) {
  x[0] = __uint_as_float(t.x); x[1] = __uint_as_float(t.y); x[2] = __uint_as_float(t.z); x[3] = __uint_as_float(t.w);
}
__device__ __forceinline__ void unpack(uint4 t, float *x, __nv_bfloat16) {
  const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 f = rowops::unpack(w[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
}
__device__ __forceinline__ uint4 pack(const float *x, float) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 pack(const float *x, __nv_bfloat16) {
  return make_uint4(rowops::pack(x[0], x[1]), rowops::pack(x[2], x[3]), rowops::pack(x[4], x[5]), rowops::pack(x[6], x[7]));
}

// A CTA has a row.  A thread has two pieces of 16 bytes of every so manieth head: those of the pairs' two halves, or two side by side; queries first,
// then keys, then values (which are only moved).  The first AHEAD heads' pieces are on their way while the angles are worked out (70B shape, 4100 rows: 32.0 us
// without that and with 256 threads, which 2, 3, 5 ahead left at 31.9, 32.5, 36.3; 128 threads with 2, 4, 6 31.0, 30.5, 31.9; 64 34.8; 25.3 at the copy peak).
constexpr int AHEAD = 4;
template <typename T, bool INTERLEAVED>
__global__ void __launch_bounds__(THREADS) append_rotary_kernel(const RotaryParams p) {
  constexpr int VEC = 16 / sizeof(T);
  __shared__ float s_cos[paged::TEXT_DIM / 2], s_sin[paged::TEXT_DIM / 2];
  const int tid = threadIdx.x, chunks = p.D / (2 * VEC), turned = p.rotary / (2 * VEC), par = THREADS / chunks;   // heads at a time
  const int ch = tid % chunks, h0 = tid / chunks, row = blockIdx.x, heads = h0 < par ? p.H + 2 * p.Hkv : 0;
  const bool rotates = ch < turned;
  // the two pieces, in elements of the head, and the first pair
  const int first = INTERLEAVED || !rotates ? ch * 2 * VEC : ch * VEC, second = INTERLEAVED || !rotates ? first + VEC : first + p.rotary / 2;
  const int pair = ch * VEC;
  const T *q = (const T *)p.q + row * p.q_stride, *k = (const T *)p.k_new + row * p.kv_stride, *v = (const T *)p.v_new + row * p.kv_stride;
  auto source = [&](int h) { return h < p.H ? q + (int64_t)h * p.D : h < p.H + p.Hkv ? k + (int64_t)(h - p.H) * p.D : v + (int64_t)(h - p.H - p.Hkv) * p.D; };
  pdl_wait();
  pdl_trigger();
  const int pos = p.positions[row], slot = p.slots[row];
  uint4 ahead[AHEAD][2];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (h0 + i * par < heads) {
      const T *src = source(h0 + i * par);
      ahead[i][0] = __ldcs((const uint4 *)(src + first));
      ahead[i][1] = __ldcs((const uint4 *)(src + second));
    }
  const bool known = pos >= 0;
  if (known && tid < p.rotary / 2) {
    const double t = pos * p.turns[tid], n = rint(4.0 * t);
    float s, c;
    sincospif(2.f * (float)fma(n, -0.25, t), &s, &c);
    const int quarter = (int)((long long)n & 3);                   // (cos, sin) of n quarter turns more
    const float x = quarter & 1 ? -s : c, y = quarter & 1 ? c : s;
    s_cos[tid] = p.magnitude * (quarter & 2 ? -x : x);
    s_sin[tid] = p.magnitude * (quarter & 2 ? -y : y);
  }
  const int pg = slot / p.page;
  const bool there = known && slot >= 0 && pg < p.n_pages;
  const int64_t at = there ? (int64_t)pg * p.page_bytes + (int64_t)(slot - pg * p.page) * p.slot_bytes : 0;
  __syncthreads();
  auto head = [&](int h, uint4 a, uint4 b) {
    const int kv = h - p.H, vh = kv - p.Hkv;
    if (kv >= 0 && !there) return;
    T *dst = kv < 0 ? (T *)p.q_out + ((int64_t)row * p.H + h) * p.D : (T *)((vh < 0 ? p.k : p.v) + at + (int64_t)(vh < 0 ? kv : vh) * p.head_bytes);
    if (!known) {
      a = b = make_uint4(0, 0, 0, 0);
    } else if (vh < 0 && rotates) {
      float x[2 * VEC], y[2 * VEC];
      unpack(a, x, T{});
      unpack(b, x + VEC, T{});
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int m = INTERLEAVED ? 2 * i : i, n = INTERLEAVED ? 2 * i + 1 : i + VEC;
        const float c = s_cos[pair + i], s = s_sin[pair + i];
        y[m] = rowops::rotate(x[m], x[n], c, -s);
        y[n] = rowops::rotate(x[n], x[m], c, s);
      }
      a = pack(y, T{});
      b = pack(y + VEC, T{});
    }
    *(uint4 *)(dst + first) = a;
    *(uint4 *)(dst + second) = b;
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (h0 + i * par < heads) head(h0 + i * par, ahead[i][0], ahead[i][1]);
  for (int h = h0 + AHEAD * par; h < heads; h += par) {
    const T *src = source(h);
    head(h, *(const uint4 *)(src + first), *(const uint4 *)(src + second));
  }
}

}  // namespace

extern "C" int ouro_paged_append_rotary(const ouro_paged_cache *c, int32_t layer, const void *q, int64_t q_stride, const void *k, const void *v,
                                        int64_t kv_stride, int32_t rows, int32_t n_heads, const int32_t *slots, const int32_t *positions,
                                        const ouro_rotary *rotary, void *q_out, void *stream) {
  const char *call = "ouro_paged_append_rotary";
  if (const char *w = paged::wrong(c)) return paged::refuse(call, w);
  if (layer < 0 || layer >= c->n_layers) return paged::refuse(call, "no such layer");
  if (!rotary || !rotary->turns) return paged::refuse(call, "rotary or its turns are NULL");
  if (rotary->rotary_dim < 16 || rotary->rotary_dim % 16 || rotary->rotary_dim > c->head_dim) return paged::refuse(call, "rotary_dim is not a multiple of 16 up to head_dim");
  if (rotary->interleaved != 0 && rotary->interleaved != 1) return paged::refuse(call, "interleaved is neither 0 nor 1");
  if (!(rotary->magnitude > 0.f) || rotary->magnitude > 1e30f) return paged::refuse(call, "magnitude is not a positive number");
  if ((uintptr_t)rotary->turns % 8) return paged::refuse(call, "turns is not 8-byte aligned");
  if (rows < 0 || n_heads < 1) return paged::refuse(call, "rows is below 0, or n_heads below 1");
  if (rows == 0) return OURO_OK;
  if (!q || !k || !v || !slots || !positions || !q_out) return paged::refuse(call, "a pointer is NULL");
  if (!paged::words(slots, positions)) return paged::refuse(call, "slots or positions are not 4-byte aligned");
  const int e = c->dtype == OURO_F32 ? 4 : 2;
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out) % 16 || q_stride * e % 16 || kv_stride * e % 16)
    return paged::refuse(call, "an array or a stride is not a multiple of 16 bytes");
  if (q_stride < (int64_t)n_heads * c->head_dim || kv_stride < (int64_t)c->n_kv_heads * c->head_dim) return paged::refuse(call, "a stride is below a row's length");
  if (q == q_out && q_stride != (int64_t)n_heads * c->head_dim) return paged::refuse(call, "q_out is q, whose rows do not lie side by side");
  RotaryParams p{};
  p.k = (uint8_t *)c->k + (int64_t)layer * c->layer_stride * e;
  p.v = (uint8_t *)c->v + (int64_t)layer * c->layer_stride * e;
  p.q = q; p.k_new = k; p.v_new = v; p.q_out = q_out;
  p.slots = slots; p.positions = positions; p.turns = rotary->turns;
  p.page_bytes = c->page_stride * e; p.slot_bytes = c->slot_stride * e; p.head_bytes = c->head_stride * e; p.q_stride = q_stride; p.kv_stride = kv_stride;
  p.rows = rows; p.H = n_heads; p.Hkv = c->n_kv_heads; p.D = c->head_dim; p.rotary = rotary->rotary_dim; p.page = c->page_size; p.n_pages = c->n_pages;
  p.magnitude = rotary->magnitude;
  const cudaStream_t s = (cudaStream_t)stream;
  cudaError_t r;
  if (c->dtype == OURO_F32) r = launch_pdl(rotary->interleaved ? append_rotary_kernel<float, true> : append_rotary_kernel<float, false>, dim3(rows), dim3(THREADS), 0, s, p);
  else r = launch_pdl(rotary->interleaved ? append_rotary_kernel<__nv_bfloat16, true> : append_rotary_kernel<__nv_bfloat16, false>, dim3(rows), dim3(THREADS), 0, s, p);
  OURO_COUNT_LAUNCH();
  return r == cudaSuccess ? OURO_OK : paged::refuse(call, cudaGetErrorString(r), OURO_ECUDA);
}
