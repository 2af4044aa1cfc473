// What the paged cache's translation units share: checks of a cache's description, the workspace's layout, errors without a context.
#pragma once

#include <atomic>
#include <string>

#include "ouro_internal.h"

void ouro_set_global_error(const std::string &msg);

namespace paged {

constexpr int MAX_CTAS = 444;        // of the attention kernel: three per SM at most
constexpr int ROW_TILE = 16;         // query rows a CTA works on at a time at most
constexpr int TC_CTAS = 160;         // the same for many query rows to a kv head: one per SM
constexpr int TC_ROWS = 128;
constexpr int TEXT_DIM = 128;        // largest head dim
// Tokens of a pool, of a row of the table, and 16-byte pieces of a page: kernels round them up to tiles and step over them in 32 bits.
constexpr int MAX_TOKENS = INT32_MAX - 65535;

// Workspace: counters that are zero between calls, then what a call needs while it runs.
struct Layout {
  size_t counters, pieces, staged, lists, bytes;
};
inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
inline Layout layout(const ouro_paged_cache &c) {
  Layout l{};
  l.counters = 0;
  l.pieces = up256(MAX_CTAS * sizeof(int));
  // attention: two pieces a CTA, each a tile's rows of (maximum, sum, head_dim values)
  const size_t rows_few = (size_t)MAX_CTAS * ROW_TILE, rows_many = (size_t)TC_CTAS * TC_ROWS;
  const size_t pieces = 2 * (rows_few > rows_many ? rows_few : rows_many) * (c.head_dim + 2) * sizeof(float);
  // page calls: entries of the rows a fork rewrites; pairs of pages to copy and the pages' new ids
  l.staged = l.pieces;
  const size_t rows = c.max_seqs < OURO_MAX_LIST ? c.max_seqs : OURO_MAX_LIST;
  l.lists = up256(l.staged + rows * c.max_pages * sizeof(int));
  const size_t lists = l.lists + up256((4 * (size_t)(c.n_pages > OURO_MAX_LIST ? c.n_pages : OURO_MAX_LIST) + 64) * sizeof(int));
  const size_t attn = l.pieces + pieces;
  l.bytes = up256(lists > attn ? lists : attn);
  return l;
}

// Arrays of 32-bit numbers (NULL where one may be left out).
template <typename... P>
inline bool words(const P *...p) { return ((((uintptr_t)p % 4) == 0) && ...); }

inline int refuse(const char *call, const char *why, int code = OURO_EINVAL) {
  ouro_set_global_error(std::string(call) + ": " + why);
  return code;
}

// Polls of the attention kernels' bounded waits.
constexpr uint32_t WAIT_LIMIT = 1u << 22;
extern std::atomic<uint32_t> wait_limit;

inline const char *wrong_shape(const ouro_paged_cache *c) {
  if (!c) return "the cache is NULL";
  if (c->n_layers < 1 || c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || c->max_seqs < 1 || c->max_pages < 1) return "a size is below 1";
  if (c->head_dim < 32 || c->head_dim > TEXT_DIM || c->head_dim % 32) return "head_dim is not 32, 64, 96 or 128";
  if (c->dtype != OURO_F32 && c->dtype != OURO_BF16) return "dtype is neither OURO_F32 nor OURO_BF16";
  if (c->max_seqs > OURO_MAX_SEQS) return "max_seqs is above OURO_MAX_SEQS";
  if ((int64_t)c->n_pages * c->page_size > MAX_TOKENS) return "n_pages * page_size is above 2^31 - 65536";
  if ((int64_t)c->max_pages * c->page_size > MAX_TOKENS) return "max_pages * page_size is above 2^31 - 65536";
  const int64_t row = (int64_t)c->n_kv_heads * (c->head_dim * (c->dtype == OURO_F32 ? 4 : 2) / 16);
  if (row > MAX_TOKENS / c->page_size) return "a page of a layer is above 2^31 - 65536 pieces of 16 bytes";
  return nullptr;
}
inline const char *wrong(const ouro_paged_cache *c) {
  if (const char *w = wrong_shape(c)) return w;
  if (!c->k || !c->v || !c->table || !c->lens || !c->refs || !c->status || !c->workspace) return "a pointer of the cache is NULL";
  if (((uintptr_t)c->k | (uintptr_t)c->v) % 16) return "k and v are not 16-byte aligned";
  if (!words(c->table, c->lens, c->refs, c->status)) return "table, lens, refs and status are not 4-byte aligned";
  if ((uintptr_t)c->workspace % 256) return "the workspace is not 256-byte aligned";
  const int64_t unit = c->dtype == OURO_F32 ? 4 : 8;
  if (c->layer_stride % unit || c->page_stride % unit || c->slot_stride % unit || c->head_stride % unit) return "a stride is not a multiple of 16 bytes";
  if (c->layer_stride < 0 || c->page_stride < 0 || c->slot_stride < 0 || c->head_stride < 0) return "a stride is negative";
  if (c->workspace_bytes < layout(*c).bytes) return "the workspace is too small";
  return nullptr;
}

// SMs of the current device, and which device it is; false: none usable.
constexpr int MAX_DEVICES = 64;
inline bool device(int *dev, int *sms) {
  static int n[MAX_DEVICES] = {};
  if (cudaGetDevice(dev) != cudaSuccess || *dev < 0 || *dev >= MAX_DEVICES) return false;
  if (!n[*dev] && cudaDeviceGetAttribute(&n[*dev], cudaDevAttrMultiProcessorCount, *dev) != cudaSuccess) return false;
  *sms = n[*dev];
  return true;
}

}  // namespace paged
