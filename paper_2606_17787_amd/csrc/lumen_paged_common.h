// What the sources of the 16-bit paged cache's operators share: the layer of a
// layout, and its checks.
#ifndef LUMEN_PAGED_COMMON_H
#define LUMEN_PAGED_COMMON_H

#include <initializer_list>

#include "lumen_attn_common.h"
#include "lumen_paged.h"

namespace lumen_paged_detail {

using namespace lumen_attn_detail;

// Division by a number that the host knows: the product with its reciprocal is the
// quotient or one less.
struct Divisor {
  uint32_t d, m;
};

inline Divisor divisor(int32_t d) {
  return Divisor{uint32_t(d), uint32_t(UINT32_MAX / uint32_t(d))};
}

__device__ __forceinline__ int quotient(const Divisor &by, int x, int *rest) {
  uint32_t q = __umulhi(uint32_t(x), by.m), r = uint32_t(x) - q * by.d;
  const bool more = r >= by.d;
  *rest = int(more ? r - by.d : r);
  return int(more ? q + 1 : q);
}
__device__ __forceinline__ int quotient(const Divisor &by, int x) {
  int rest;
  return quotient(by, x, &rest);
}

// Sizes of a 16-bit cache, in bytes.
struct Pages {
  int64_t half;     // K or V of a layer
  int64_t page;     // K or V of a block
  int32_t slot;     // from a token's row of a head to the next token's
  int32_t head;     // from a head's rows to the next head's
  int32_t row;
};

inline int check_pages(const lumen_kv_layout *l, int32_t layer, int32_t layers, Pages *out) {
  if (!l || l->num_layers < 1 || l->num_kv_heads < 1 || l->block_size < 1 ||
      l->num_blocks < 0 || layer < 0 || layers < 0 || layer > l->num_layers - layers)
    return LUMEN_ERR_INVALID_ARG;
  if (l->elem_bytes != 2 ||
      (l->head_dim != 64 && l->head_dim != 128 && l->head_dim != 256) ||
      (l->cache_order != LUMEN_CACHE_NHD && l->cache_order != LUMEN_CACHE_HND))
    return LUMEN_ERR_UNSUPPORTED;
  const int32_t row = 2 * l->head_dim;
  const int64_t rows = int64_t(l->block_size) * l->num_kv_heads;
  if (rows > INT32_MAX / row) return LUMEN_ERR_UNSUPPORTED;
  int64_t half;
  if (__builtin_mul_overflow(rows * row, l->num_blocks, &half) ||
      half > INT64_MAX / 2 / l->num_layers)
    return LUMEN_ERR_INVALID_ARG;
  const bool hnd = l->cache_order == LUMEN_CACHE_HND;
  *out = Pages{half, rows * row, hnd ? row : l->num_kv_heads * row,
               hnd ? l->block_size * row : row, row};
  return LUMEN_OK;
}

// Words of the ledger's weights, or positions, of a layer.
inline int64_t ledger_words(const lumen_kv_layout *l) {
  return l->num_blocks * l->num_kv_heads * l->block_size;
}

// Words of the ledger before a layer's.
inline int64_t ledger_before(const lumen_kv_layout *l, int32_t layer) {
  return int64_t(layer) * 2 * ledger_words(l);
}

// Places that a block table row has.
inline int64_t places_of(const lumen_kv_layout *l, int32_t bt_cols) {
  return int64_t(bt_cols) * l->block_size;
}

// The sizes of a call with queries.
inline int check_queries(const lumen_kv_layout *l, int32_t bt_cols, int32_t num_reqs,
                         int64_t num_tokens, int32_t max_new, int32_t q_heads) {
  if (bt_cols < 0 || num_reqs < 0 || num_tokens < 0 || max_new < 0 || q_heads < 1 ||
      q_heads % l->num_kv_heads)
    return LUMEN_ERR_INVALID_ARG;
  if ((l->head_dim != 64 && l->head_dim != 128) || num_tokens > INT32_MAX ||
      num_tokens * (q_heads / l->num_kv_heads) > LUMEN_PAGED_MAX_ROWS)
    return LUMEN_ERR_UNSUPPORTED;
  return num_reqs > LUMEN_ATTN_MAX_REQS ? LUMEN_ERR_TOO_MANY : LUMEN_OK;
}

// Starts a load of 16 bytes a lane from the lane's address into LDS at byte `to` +
// 16 * lane, kept in caches; see load_to_lds.
__device__ __forceinline__ void load_row(const void *from, uint32_t to) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :: "{m0}"(to), "v"(from) : "memory");
}

// Rows of places that are left out are read from here, so that what the cache
// holds there reaches nothing.
__device__ __attribute__((aligned(16))) const uint16_t kZeroRow[128] = {};

// What a kernel of a call with queries needs of it.
struct Call {
  Rows q;
  const uint8_t *k, *v;  // of the layer
  int64_t page;
  int32_t slot_bytes, head_bytes;
  int32_t block_size;
  int64_t num_blocks;
  const int32_t *bt;
  int32_t bt_cols;
  int32_t cap;  // places that a table row has, held to kMostPlaces
  const int32_t *lens, *cu;
  int32_t num_reqs;
  int64_t num_q;
  int32_t max_new;
  int32_t q_heads, kv_heads, group;
  Divisor by_block, by_group;  // block_size, group
  float scale_log2;
  int32_t *status;
};

// A range of bytes.
struct Span {
  const void *at;
  size_t bytes;
};

inline bool overlap(const Span &a, const Span &b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
  return a.bytes && b.bytes && (x < y ? y - x < a.bytes : x - y < b.bytes);
}

// Whether one of the ranges that a call writes shares bytes with another of them or
// with one that it reads.
inline bool overlap(std::initializer_list<Span> written, std::initializer_list<Span> read) {
  for (const Span *w = written.begin(); w != written.end(); ++w) {
    for (const Span *v = w + 1; v != written.end(); ++v)
      if (overlap(*w, *v)) return true;
    for (const Span &r : read)
      if (overlap(*w, r)) return true;
  }
  return false;
}

// What the rows of a call's tokens take, from the first to the last.
inline Span span_of(const lumen_attn_rows *r, int64_t tokens, int32_t heads, int32_t head_dim) {
  return Span{r->d_base, size_t((tokens - 1) * r->token_stride +
                                int64_t(heads - 1) * r->head_stride + head_dim) * 2};
}

// So that a step's places are counted in 32 bits.
constexpr int64_t kMostPlaces = INT32_MAX - 255;

inline Call call_of(const lumen_kv_layout *l, const Pages &p, int32_t layer, const void *cache,
                    const int32_t *bt, int32_t bt_cols, const int32_t *lens, const int32_t *cu,
                    int32_t num_reqs, const lumen_attn_rows *q, int64_t num_tokens,
                    int32_t max_new, int32_t q_heads, float scale, int32_t *status) {
  Call c;
  c.q = rows_of(q, 0);
  c.k = static_cast<const uint8_t *>(cache) + int64_t(layer) * 2 * p.half;
  c.v = c.k + p.half;
  c.page = p.page;
  c.slot_bytes = p.slot;
  c.head_bytes = p.head;
  c.block_size = l->block_size;
  c.num_blocks = l->num_blocks;
  c.bt = bt;
  c.bt_cols = bt_cols;
  const int64_t cap = places_of(l, bt_cols);
  c.cap = int32_t(cap < kMostPlaces ? cap : kMostPlaces);
  c.lens = lens;
  c.cu = cu;
  c.num_reqs = num_reqs;
  c.num_q = num_tokens;
  c.max_new = max_new;
  c.q_heads = q_heads;
  c.kv_heads = l->num_kv_heads;
  c.group = q_heads / l->num_kv_heads;
  c.by_block = divisor(c.block_size);
  c.by_group = divisor(c.group);
  c.scale_log2 = scale_log2(scale);
  c.status = status;
  return c;
}

// One request of a call: its first query, new tokens and places.
struct Request {
  int q0, m, n;
};

// Returns an error code; a request that is skipped has no tokens.
__device__ __forceinline__ int request(const Call &a, int r, Request *out) {
  const int32_t q0 = a.cu[r], q1 = a.cu[r + 1], n = a.lens[r];
  *out = Request{q0, 0, n < 0 ? 0 : n};
  if (q0 < 0 || q1 < q0 || q1 > a.num_q || q1 - q0 > a.max_new) return LUMEN_ERR_RANGE;
  out->m = q1 - q0;
  return n < 0 || n > a.cap ? LUMEN_ERR_RANGE : LUMEN_OK;
}

}  // namespace lumen_paged_detail

#endif  // LUMEN_PAGED_COMMON_H
