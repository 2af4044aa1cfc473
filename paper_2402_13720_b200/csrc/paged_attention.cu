// Attention of the newest tokens of several sequences over a paged cache, split over the cache's length and joined.
//
//     o = sum_j e^(s_j) v_j / sum_j e^(s_j),   s_j = scale q . k_j,   j over the keys a token sees
//
// Bound by HBM: a key and a value are 4 head_dim bytes (bf16) and give 4 head_dim operations per query head that shares them, at most a
// few dozen operations a byte.  So the whole design is about reading every key and value once, without a pause, on all SMs:
//  - The query rows that share a kv head (new tokens x query heads of its group) are one row tile of up to 16, a sequence's kv
//    head and row tile an item.  Items are cut along the keys into units of TILE keys; all units of a call, in order, are dealt out to
//    the CTAs in equal runs whatever the lengths are.  An item that lies in one CTA is finished there; of an item cut between CTAs each leaves
//    a piece (maximum, sum, unnormalised output, in 32 bits), and the CTA that is last to do so joins the pieces in ascending order
//    (so the result does not depend on who that is).
//  - A warp has KW keys of every unit and its own ring of shared memory, filled by 16-byte asynchronous copies STAGES - 1 units ahead,
//    across the borders of items; the ids of pages are read one unit before that.  Warps meet only at an item's end.
//  - bf16: S = Q K^T and O += P V as mma.sync m16n8k16 with Q, P and O in registers (the tensor cores idle most of the time
//    anyway).  P goes in as two bf16 parts, P = hi + lo up to 2^-17: one part alone would add an error as large as the output's own
//    rounding.  f32: multiply-adds in 32 bits.
// Keys that are not there (beyond the length, on no page) are not read: zeros take their place, and their probability is 0.
#include "paged.h"

namespace {

using paged::MAX_CTAS;

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr int MAX_LIST = OURO_MAX_LIST;

struct AttnParams {
  const uint8_t *k, *v;                 // of the layer
  const int32_t *table, *lens, *seqs;
  const void *q;
  void *out;
  float *lse;
  int *counters;
  float *pieces;                        // [CTA][2][ROW_TILE][D], then [CTA][2][ROW_TILE][2]
  int64_t page_bytes, slot_bytes, head_bytes, q_stride;
  int n, n_new, H, Hkv, group, rows, row_tiles;   // rows = n_new * group
  int n_pages, page, max_pages, max_seqs, cap;
  float scale_log2;
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes, or zeros where there is nothing to read
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t *r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t *r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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

template <typename T, int D>
struct Cfg {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int KW = BF ? 16 : 8;            // keys of a warp in a unit
  static constexpr int TILE = KW * WARPS;
  static constexpr int ROWS = BF ? 16 : 8;          // query rows of a tile
  static constexpr int ROWB = D * (int)sizeof(T);
  static constexpr int PITCH = ROWB + 16;           // an odd number of 16-byte pieces: eight rows' equal columns lie in different banks
  static constexpr int STAGE = 2 * KW * PITCH;      // K rows, V rows of one warp
  static constexpr int STAGES = 3;
  static constexpr int OFF_RING = 0;                                      // [warp][stage]
  static constexpr int OFF_Q = WARPS * STAGES * STAGE;                    // f32: [warp][ROWS][D]
  static constexpr int OFF_ML = OFF_Q + (BF ? 0 : WARPS * ROWS * D * 4);  // [warp][ROWS][2]
  static constexpr int OFF_MASK = OFF_ML + WARPS * ROWS * 8;              // [warp][stage]
  static constexpr int OFF_LEN = OFF_MASK + WARPS * STAGES * 4;           // [n]
  static constexpr int OFF_CUM = OFF_LEN + MAX_LIST * 4;                  // [n + 1] units of a head and row tile
  static constexpr int OFF_MISC = OFF_CUM + (MAX_LIST + 1) * 4;
  static constexpr int BYTES = OFF_MISC + 64;
  static_assert(ROWS * D * 4 <= STAGE, "a warp's output fits its stage");
};

// A place in the list of units: sequence, head and row tile, unit of the item.
struct Walk {
  int s, hr, tile, tiles, len;
  const int32_t *row;
};

template <typename T, int D>
__global__ void __launch_bounds__(THREADS) paged_attention_kernel(const AttnParams p) {
  using C = Cfg<T, D>;
  extern __shared__ __align__(128) uint8_t smem[];
  int *s_len = (int *)(smem + C::OFF_LEN), *s_cum = (int *)(smem + C::OFF_CUM), *s_misc = (int *)(smem + C::OFF_MISC);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_trigger();

  // ---- how many units every sequence has, and where this CTA's run of them begins
  {
    const int per = (p.n + THREADS - 1) / THREADS;
    int sum = 0;
    for (int i = tid * per; i < min(p.n, (tid + 1) * per); ++i) {
      const int sid = p.seqs ? __ldg(p.seqs + i) : i;
      int len = 0;
      if (sid >= 0 && sid < p.max_seqs) len = min(max(__ldg(p.lens + sid), 0), p.cap);
      s_len[i] = len;
      sum += max(1, (len + C::TILE - 1) / C::TILE);
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += up;
    }
    if (lane == 31) s_misc[warp] = inc;
    __syncthreads();
    int at = inc - sum;
    for (int w = 0; w < warp; ++w) at += s_misc[w];
    for (int i = tid * per; i < min(p.n, (tid + 1) * per); ++i) {
      s_cum[i] = at;
      at += max(1, (s_len[i] + C::TILE - 1) / C::TILE);
    }
    if (tid == THREADS - 1) s_cum[p.n] = at;
    __syncthreads();
  }
  const int F = p.Hkv * p.row_tiles;                              // items of a sequence
  const int64_t U = (int64_t)s_cum[p.n] * F, G = min((int64_t)gridDim.x, U);   // (each of G CTAs has a unit at least)
  if (blockIdx.x >= G) return;
  const int64_t u_begin = U * blockIdx.x / G, u_end = U * (blockIdx.x + 1) / G;

  auto enter = [&](Walk &w) {
    w.len = s_len[w.s];
    w.tiles = s_cum[w.s + 1] - s_cum[w.s];
    const int sid = p.seqs ? __ldg(p.seqs + w.s) : w.s;
    w.row = p.table + (int64_t)(w.len > 0 ? sid : 0) * p.max_pages;
  };
  auto next = [&](Walk &w) {
    if (++w.tile < w.tiles) return;
    w.tile = 0;
    if (++w.hr < F) return;
    w.hr = 0;
    if (++w.s < p.n) enter(w);
  };
  Walk c;                                                         // the unit being worked on
  {
    int lo = 0, hi = p.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if ((int64_t)s_cum[mid] * F <= u_begin) lo = mid; else hi = mid - 1;
    }
    c.s = lo;
    enter(c);
    const int in = (int)(u_begin - (int64_t)s_cum[lo] * F);       // fits: a sequence's units are counted in 32 bits on the host
    c.hr = in / c.tiles;
    c.tile = in - c.hr * c.tiles;
  }

  // ---- the warp's ring
  const uint32_t ring = smem_u32(smem + C::OFF_RING) + warp * C::STAGES * C::STAGE;
  uint8_t *ring_p = smem + C::OFF_RING + warp * C::STAGES * C::STAGE;
  volatile uint32_t *s_mask = (volatile uint32_t *)(smem + C::OFF_MASK) + warp * C::STAGES;
  Walk f = c;                                                     // the unit to be fetched next
  int64_t f_u = u_begin;
  int f_pid, f_row;                                               // page and row of the key of this lane (lane mod KW) in it
  auto read_ids = [&]() {
    const int key = f.tile * C::TILE + warp * C::KW + (lane & (C::KW - 1));
    const int pg = key / p.page;
    f_row = key - pg * p.page;
    f_pid = f_u < u_end && key < f.len ? __ldg(f.row + pg) : -1;
  };
  auto fetch = [&](int stage) {
    if (f_u < u_end) {
      const bool there = f_pid >= 0 && f_pid < p.n_pages;
      const int64_t off = there ? (int64_t)f_pid * p.page_bytes + (int64_t)f_row * p.slot_bytes + (int64_t)(f.hr / p.row_tiles) * p.head_bytes : -1;
      const uint32_t mask = __ballot_sync(0xffffffffu, there) & ((1u << C::KW) - 1);
      if (lane == 0) s_mask[stage] = mask;
      constexpr int CH = C::ROWB / 16, N = C::KW * CH;            // 16-byte pieces of a row, of all rows
      const uint32_t dst = ring + stage * C::STAGE;
#pragma unroll
      for (int i = 0; i < (N + 31) / 32; ++i) {
        const int e = i * 32 + lane, r = e / CH, ch = e - r * CH;
        const int64_t ro = __shfl_sync(0xffffffffu, off, r & (C::KW - 1));
        if (N % 32 == 0 || e < N) {
          const int64_t o = ro < 0 ? 0 : ro + ch * 16;
          cp_async16(dst + r * C::PITCH + ch * 16, p.k + o, ro >= 0);
          cp_async16(dst + (C::KW + r) * C::PITCH + ch * 16, p.v + o, ro >= 0);
        }
      }
      next(f);
      ++f_u;
      read_ids();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  read_ids();
#pragma unroll
  for (int i = 0; i < C::STAGES - 1; ++i) fetch(i);

  // ---- state of the item: bf16 as mma fragments (rows lane / 4 and + 8), f32 with four columns a lane
  constexpr int NACC = C::BF ? D / 2 : C::ROWS * 4;
  constexpr int NST = C::BF ? 2 : C::ROWS;
  float acc[NACC], m[NST], l[NST];
  uint32_t qf[C::BF ? D / 4 : 1];
  int vis[NST];
  float *s_q = (float *)(smem + C::OFF_Q) + (C::BF ? 0 : warp * C::ROWS * D);
  float *s_ml = (float *)(smem + C::OFF_ML);
  bool fresh = true;
  int first_tile = c.tile;                                        // of the item's part that this CTA has

  int stage = 0;
  for (int64_t u = u_begin; u < u_end; ++u) {
    asm volatile("cp.async.wait_group %0;" ::"n"(C::STAGES - 2) : "memory");
    __syncwarp();
    fetch(stage == 0 ? C::STAGES - 1 : stage - 1);
    const int rt = c.hr % p.row_tiles, kvh = c.hr / p.row_tiles;
    const int rows = min(C::ROWS, p.rows - rt * C::ROWS);         // of this tile
    if (fresh) {
      fresh = false;
      first_tile = c.tile;
#pragma unroll
      for (int i = 0; i < NACC; ++i) acc[i] = 0.f;
      if constexpr (C::BF) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = (lane >> 2) + 8 * i, at = rt * C::ROWS + r, tok = at / p.group;
          m[i] = -INFINITY;
          l[i] = 0.f;
          vis[i] = r < rows ? c.len - p.n_new + 1 + tok : 0;
          const uint32_t *src = (const uint32_t *)((const __nv_bfloat16 *)p.q + ((int64_t)c.s * p.n_new + tok) * p.q_stride +
                                                   (int64_t)(kvh * p.group + at - tok * p.group) * D);
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
            qf[4 * j + i] = r < rows ? __ldg(src + j * 8 + (lane & 3)) : 0u;
            qf[4 * j + 2 + i] = r < rows ? __ldg(src + j * 8 + 4 + (lane & 3)) : 0u;
          }
        }
      } else {
#pragma unroll
        for (int r = 0; r < C::ROWS; ++r) {
          const int at = rt * C::ROWS + r, tok = at / p.group;
          m[r] = -INFINITY;
          l[r] = 0.f;
          vis[r] = r < rows ? c.len - p.n_new + 1 + tok : 0;
          const float *src = (const float *)p.q + ((int64_t)c.s * p.n_new + tok) * p.q_stride + (int64_t)(kvh * p.group + at - tok * p.group) * D;
          for (int d = lane; d < D; d += 32) s_q[r * D + d] = r < rows ? __ldg(src + d) : 0.f;
        }
        __syncwarp();
      }
    }
    const uint32_t mask = s_mask[stage];
    const uint32_t kb = ring + stage * C::STAGE, vb = kb + C::KW * C::PITCH;
    const int key0 = c.tile * C::TILE + warp * C::KW;
    if constexpr (C::BF) {
      float sc[8];                                                // [key block of 8][row, row: two keys each]
#pragma unroll
      for (int i = 0; i < 8; ++i) sc[i] = 0.f;
      const uint32_t ka = kb + ((lane & 7) + ((lane & 16) >> 1)) * C::PITCH + ((lane & 8) << 1);
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        uint32_t b[4];
        ldsm_x4(ka + j * 32, b);
        mma16(sc, qf + 4 * j, b[0], b[1]);
        mma16(sc + 4, qf + 4 * j, b[2], b[3]);
      }
      const int t2 = (lane & 3) * 2;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int kk = (i >> 2) * 8 + t2 + (i & 1);
        sc[i] = (mask >> kk & 1) && key0 + kk < vis[(i >> 1) & 1] ? sc[i] * p.scale_log2 : -INFINITY;
      }
      float a[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float mx = fmaxf(fmaxf(sc[2 * i], sc[2 * i + 1]), fmaxf(sc[4 + 2 * i], sc[5 + 2 * i]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        const float mn = fmaxf(m[i], mx), base = base_of(mn);
        a[i] = ex2(m[i] - base);
        m[i] = mn;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          sc[4 * h + 2 * i] = ex2(sc[4 * h + 2 * i] - base);
          sc[4 * h + 2 * i + 1] = ex2(sc[4 * h + 2 * i + 1] - base);
        }
        l[i] = l[i] * a[i] + ((sc[2 * i] + sc[2 * i + 1]) + (sc[4 + 2 * i] + sc[5 + 2 * i]));
      }
      if (__any_sync(0xffffffffu, a[0] != 1.f || a[1] != 1.f)) {
#pragma unroll
        for (int i = 0; i < NACC; ++i) acc[i] *= a[(i >> 1) & 1];
      }
      // A later token's key may lie in the tile although an earlier one does not see it; 0 times what is stored there must be 0
      // whatever it is.
      bool odd = false;
      if (p.n_new > 1 && key0 + C::KW > c.len - p.n_new) {
        constexpr int CH = C::ROWB / 16;
        for (int e = lane; e < C::KW * CH; e += 32) {
          const uint4 x = *(const uint4 *)(ring_p + stage * C::STAGE + (C::KW + e / CH) * C::PITCH + (e % CH) * 16);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
        }
        odd = __any_sync(0xffffffffu, odd);
      }
      if (!odd) {
        uint32_t hi[4], lo[4];                                    // A operand: (row, keys), (row + 8, keys), (row, keys + 8), (row + 8, keys + 8)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = sc[(i >> 1) * 4 + (i & 1) * 2], y = sc[(i >> 1) * 4 + (i & 1) * 2 + 1];
          hi[i] = pack(x, y);
          lo[i] = rest(x, y, hi[i]);
        }
        const uint32_t va = vb + ((lane & 7) + (lane & 8)) * C::PITCH + (lane & 16);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          uint32_t b[4];
          ldsm_x4_t(va + j * 32, b);
          mma16(acc + 8 * j, hi, b[0], b[1]);
          mma16(acc + 8 * j + 4, hi, b[2], b[3]);
          mma16(acc + 8 * j, lo, b[0], b[1]);
          mma16(acc + 8 * j + 4, lo, b[2], b[3]);
        }
      } else {
        for (int j = 0; j < C::KW; ++j) {
          float pr[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float even = __shfl_sync(0xffffffffu, j < 8 ? sc[2 * i] : sc[4 + 2 * i], (lane & 28) + ((j & 7) >> 1));
            const float oddk = __shfl_sync(0xffffffffu, j < 8 ? sc[2 * i + 1] : sc[5 + 2 * i], (lane & 28) + ((j & 7) >> 1));
            pr[i] = j & 1 ? oddk : even;
          }
          const bool on = mask >> j & 1;
          const uint8_t *vr = ring_p + stage * C::STAGE + (C::KW + j) * C::PITCH + t2 * 2;
#pragma unroll
          for (int b = 0; b < D / 8; ++b) {
            const uint32_t w = *(const uint32_t *)(vr + b * 16);
            const float v0 = __uint_as_float(w << 16), v1 = __uint_as_float(w & 0xffff0000u);
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (on && key0 + j < vis[i]) {
                acc[4 * b + 2 * i] = fmaf(pr[i], v0, acc[4 * b + 2 * i]);
                acc[4 * b + 2 * i + 1] = fmaf(pr[i], v1, acc[4 * b + 2 * i + 1]);
              }
          }
        }
      }
    } else {
      // scores: a key has four lanes, each a quarter of the dims (every fourth piece of four)
      const int key = lane >> 2, part = lane & 3;
      const float *kr = (const float *)(ring_p + stage * C::STAGE + key * C::PITCH);
      float s[C::ROWS];
#pragma unroll
      for (int r = 0; r < C::ROWS; ++r) s[r] = 0.f;
      for (int j = 0; j < D / 16; ++j) {
        const int d = (4 * j + part) * 4;
        const float4 kk = *(const float4 *)(kr + d);
#pragma unroll
        for (int r = 0; r < C::ROWS; ++r) {
          if (r >= rows) break;
          const float4 qq = *(const float4 *)(s_q + r * D + d);
          s[r] = fmaf(kk.x, qq.x, fmaf(kk.y, qq.y, fmaf(kk.z, qq.z, fmaf(kk.w, qq.w, s[r]))));
        }
      }
      const bool there = mask >> key & 1;
#pragma unroll
      for (int r = 0; r < C::ROWS; ++r) {
        if (r >= rows) break;
        float x = s[r];
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        x = there && key0 + key < vis[r] ? x * p.scale_log2 : -INFINITY;
        float mx = x;
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        const float mn = fmaxf(m[r], mx), base = base_of(mn), a = ex2(m[r] - base);
        m[r] = mn;
        s[r] = ex2(x - base);
        l[r] = l[r] * a + (part == 0 ? s[r] : 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[4 * r + i] *= a;
      }
      const int col = min(lane, D / 4 - 1) * 4;                   // (lanes beyond the columns take part in the exchange below)
      for (int j = 0; j < C::KW; ++j) {
        const float4 vv = *(const float4 *)(ring_p + stage * C::STAGE + (C::KW + j) * C::PITCH + col * 4);
#pragma unroll
        for (int r = 0; r < C::ROWS; ++r) {
          if (r >= rows) break;
          const float pr = __shfl_sync(0xffffffffu, s[r], j * 4);
          if (!((mask >> j & 1) && key0 + j < vis[r])) continue;   // (uniform: 0 times what is stored there would not be 0 for all values)
          acc[4 * r] = fmaf(pr, vv.x, acc[4 * r]);
          acc[4 * r + 1] = fmaf(pr, vv.y, acc[4 * r + 1]);
          acc[4 * r + 2] = fmaf(pr, vv.z, acc[4 * r + 2]);
          acc[4 * r + 3] = fmaf(pr, vv.w, acc[4 * r + 3]);
        }
      }
    }

    // ---- the item's or the run's end: the warps' parts are added up
    const bool item_ends = c.tile == c.tiles - 1;
    if (item_ends || u == u_end - 1) {
      float *mine = (float *)(ring_p + stage * C::STAGE);          // [row][column], columns of a row exchanged so that eight rows' stores spread over the banks
      __syncwarp();                                                // the stage has been read
      if constexpr (C::BF) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
          l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
          const int r = (lane >> 2) + 8 * i;
          if (r < rows) {
#pragma unroll
            for (int b = 0; b < D / 8; ++b)
              *(float2 *)(mine + r * D + ((b * 8) ^ ((r & 3) * 8)) + (lane & 3) * 2) = make_float2(acc[4 * b + 2 * i], acc[4 * b + 2 * i + 1]);
            if ((lane & 3) == 0) *(float2 *)(s_ml + (warp * C::ROWS + r) * 2) = make_float2(m[i], l[i]);
          }
        }
      } else {
#pragma unroll
        for (int r = 0; r < C::ROWS; ++r) {
          if (r >= rows) break;
          float x = l[r];
          x += __shfl_xor_sync(0xffffffffu, x, 4);
          x += __shfl_xor_sync(0xffffffffu, x, 8);
          x += __shfl_xor_sync(0xffffffffu, x, 16);
          if (lane < D / 4) *(float4 *)(mine + r * D + ((lane * 4) ^ ((r & 3) * 8))) = make_float4(acc[4 * r], acc[4 * r + 1], acc[4 * r + 2], acc[4 * r + 3]);
          if (lane == 0) *(float2 *)(s_ml + (warp * C::ROWS + r) * 2) = make_float2(m[r], x);
        }
      }
      __syncthreads();
      const int64_t item0 = (int64_t)s_cum[c.s] * F + (int64_t)c.hr * c.tiles;   // the item's first unit
      const bool whole = item_ends && first_tile == 0;
      const int slot = item0 <= u_begin ? 0 : 1;
      float *piece = p.pieces + ((int64_t)blockIdx.x * 2 + slot) * paged::ROW_TILE * D;
      float *piece_ml = p.pieces + (int64_t)MAX_CTAS * 2 * paged::ROW_TILE * D + ((int64_t)blockIdx.x * 2 + slot) * paged::ROW_TILE * 2;
      constexpr int C4 = D / 4;
      auto finish = [&](int r, int col, float M, float L, const float *o) {       // four columns of a row to the output
        const int at = rt * C::ROWS + r, tok = at / p.group, head = kvh * p.group + at - tok * p.group;
        const int64_t row = ((int64_t)c.s * p.n_new + tok) * p.H + head;
        const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);               // (a sum that is not a number stays one)
        if constexpr (C::BF)
          *(uint2 *)((__nv_bfloat16 *)p.out + row * D + col) = make_uint2(pack(o[0] * inv, o[1] * inv), pack(o[2] * inv, o[3] * inv));
        else
          *(float4 *)((float *)p.out + row * D + col) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
        if (p.lse && col == 0) p.lse[row] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
      };
      for (int e = tid; e < rows * C4; e += THREADS) {
        const int r = e / C4, col = (e - r * C4) * 4;
        float mw[WARPS], M = -INFINITY, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          mw[w] = s_ml[(w * C::ROWS + r) * 2];
          M = fmaxf(M, mw[w]);
        }
        const float base = base_of(M);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          const float a = ex2(mw[w] - base);
          const float4 x = *(const float4 *)(smem + C::OFF_RING + (w * C::STAGES + stage) * C::STAGE + (r * D + (col ^ ((r & 3) * 8))) * 4);
          L = fmaf(a, s_ml[(w * C::ROWS + r) * 2 + 1], L);
          o[0] = fmaf(a, x.x, o[0]);
          o[1] = fmaf(a, x.y, o[1]);
          o[2] = fmaf(a, x.z, o[2]);
          o[3] = fmaf(a, x.w, o[3]);
        }
        if (whole) {
          finish(r, col, M, L, o);
        } else {
          __stcg((float4 *)(piece + r * D + col), make_float4(o[0], o[1], o[2], o[3]));
          if (col == 0) __stcg((float2 *)(piece_ml + r * 2), make_float2(M, L));
        }
      }
      if (!whole) {
        const int64_t last = item0 + c.tiles - 1;
        const int c0 = (int)(((item0 + 1) * G - 1) / U), c1 = (int)(((last + 1) * G - 1) / U);   // the CTAs that have its first and last unit
        __threadfence();
        __syncthreads();
        if (tid == 0) s_misc[4] = atomicAdd(p.counters + c0, 1) == c1 - c0;
        __syncthreads();
        if (s_misc[4]) {
          if (tid == 0) p.counters[c0] = 0;
          __threadfence();
          const float *pieces = p.pieces, *mls = p.pieces + (int64_t)MAX_CTAS * 2 * paged::ROW_TILE * D;
          for (int r = warp; r < rows; r += WARPS) {
            auto where = [&](int cta) { return (int64_t)cta * 2 + (cta == c0 && U * cta / G < item0 ? 1 : 0); };
            float M = -INFINITY;
            for (int a = c0 + lane; a <= c1; a += 32) M = fmaxf(M, __ldcg(mls + (where(a) * paged::ROW_TILE + r) * 2));
#pragma unroll
            for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
            const float base = base_of(M);
            float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
            for (int a0 = c0; a0 <= c1; a0 += 32) {
              float2 ml = make_float2(-INFINITY, 0.f);
              if (a0 + lane <= c1) ml = __ldcg((const float2 *)(mls + (where(a0 + lane) * paged::ROW_TILE + r) * 2));
              const float wt = ex2(ml.x - base), wl = wt * ml.y;
              const int many = min(32, c1 - a0 + 1);
#pragma unroll 8
              for (int j = 0; j < many; ++j) {
                const float x = __shfl_sync(0xffffffffu, wt, j);
                L += __shfl_sync(0xffffffffu, wl, j);
                const float4 y = __ldcg((const float4 *)(pieces + (where(a0 + j) * paged::ROW_TILE + r) * D + min(lane, C4 - 1) * 4));
                o[0] = fmaf(x, y.x, o[0]);
                o[1] = fmaf(x, y.y, o[1]);
                o[2] = fmaf(x, y.z, o[2]);
                o[3] = fmaf(x, y.w, o[3]);
              }
            }
            if (lane < C4) finish(r, lane * 4, M, L, o);
          }
        }
      }
      __syncthreads();                                             // the stages and the sums may be written again
      fresh = true;
    }
    next(c);
    stage = stage + 1 == C::STAGES ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename T, int D>
int launch(const AttnParams &p, int64_t units, cudaStream_t s) {
  static int fit[paged::MAX_DEVICES] = {};                         // CTAs that are resident at once, per device
  int dev = 0, sms = 0;
  if (!paged::device(&dev, &sms)) return paged::refuse("ouro_paged_attention", "no usable current device", OURO_ECUDA);
  if (!fit[dev]) {
    int per_sm = 0;
    if (cudaFuncSetAttribute(paged_attention_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<T, D>::BYTES) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, paged_attention_kernel<T, D>, THREADS, Cfg<T, D>::BYTES) != cudaSuccess || per_sm < 1)
      return paged::launched("ouro_paged_attention") == OURO_OK ? paged::refuse("ouro_paged_attention", "the kernel does not fit this device", OURO_ECUDA) : OURO_ECUDA;
    fit[dev] = min(MAX_CTAS, sms * per_sm);
  }
  const int grid = (int)min((int64_t)fit[dev], units);
  const cudaError_t e = launch_pdl(paged_attention_kernel<T, D>, dim3(grid), dim3(THREADS), Cfg<T, D>::BYTES, s, p);
  OURO_COUNT_LAUNCH();
  return e == cudaSuccess ? OURO_OK : paged::refuse("ouro_paged_attention", cudaGetErrorString(e), OURO_ECUDA);
}

template <typename T>
int by_dim(int d, const AttnParams &p, int64_t units, cudaStream_t s) {
  switch (d) {
    case 32: return launch<T, 32>(p, units, s);
    case 64: return launch<T, 64>(p, units, s);
    case 96: return launch<T, 96>(p, units, s);
    default: return launch<T, 128>(p, units, s);
  }
}

}  // namespace

extern "C" int ouro_paged_attention(const ouro_paged_cache *c, int32_t layer, const int32_t *seqs, int32_t n, int32_t n_new, const void *q,
                                    int64_t q_stride, int32_t n_heads, float scale, void *out, float *lse, void *stream) {
  const char *call = "ouro_paged_attention";
  if (const char *w = paged::wrong(c)) return paged::refuse(call, w);
  if (layer < 0 || layer >= c->n_layers) return paged::refuse(call, "no such layer");
  if (n < 0 || n > OURO_MAX_LIST) return paged::refuse(call, "n is below 0 or above OURO_MAX_LIST");
  if (n_new < 1 || n_new > OURO_MAX_NEW) return paged::refuse(call, "n_new is below 1 or above OURO_MAX_NEW");
  if (n_heads < 1 || n_heads % c->n_kv_heads) return paged::refuse(call, "n_heads is not a multiple of the cache's n_kv_heads");
  if (n == 0) return OURO_OK;
  if (!q || !out) return paged::refuse(call, "q or out is NULL");
  if (!seqs && n > c->max_seqs) return paged::refuse(call, "more sequences than the table has");
  const int esize = c->dtype == OURO_F32 ? 4 : 2;
  if (((uintptr_t)q | (uintptr_t)out) % 16 || (q_stride * esize) % 16) return paged::refuse(call, "q, out or q_stride is not a multiple of 16 bytes");
  if (q_stride < (int64_t)n_heads * c->head_dim) return paged::refuse(call, "q_stride is below n_heads * head_dim");
  const int tile = c->dtype == OURO_F32 ? 8 * WARPS : 16 * WARPS, rows_of = c->dtype == OURO_F32 ? 8 : 16;
  AttnParams p{};
  p.group = n_heads / c->n_kv_heads;
  p.rows = n_new * p.group;
  p.row_tiles = (p.rows + rows_of - 1) / rows_of;
  p.cap = c->max_pages * c->page_size;
  const int64_t units = ((int64_t)(p.cap + tile - 1) / tile) * c->n_kv_heads * p.row_tiles;
  if (units > INT32_MAX) return paged::refuse(call, "a sequence's work is above 2^31 units");
  const paged::Layout l = paged::layout(*c);
  p.k = (const uint8_t *)c->k + (int64_t)layer * c->layer_stride * esize;
  p.v = (const uint8_t *)c->v + (int64_t)layer * c->layer_stride * esize;
  p.table = c->table; p.lens = c->lens; p.seqs = seqs;
  p.q = q; p.out = out; p.lse = lse;
  p.counters = (int *)((char *)c->workspace + l.counters);
  p.pieces = (float *)((char *)c->workspace + l.pieces);
  p.page_bytes = c->page_stride * esize; p.slot_bytes = c->slot_stride * esize; p.head_bytes = c->head_stride * esize; p.q_stride = q_stride;
  p.n = n; p.n_new = n_new; p.H = n_heads; p.Hkv = c->n_kv_heads;
  p.n_pages = c->n_pages; p.page = c->page_size; p.max_pages = c->max_pages; p.max_seqs = c->max_seqs;
  p.scale_log2 = scale * 1.4426950408889634f;
  return c->dtype == OURO_F32 ? by_dim<float>(c->head_dim, p, units * n, (cudaStream_t)stream)
                              : by_dim<__nv_bfloat16>(c->head_dim, p, units * n, (cudaStream_t)stream);
}
