// Argument checks that the entry points of the paged cache share.
#pragma once

#include <algorithm>
#include <cstdint>

#include "../../include/ipv.h"
#include "ipv_pages.hpp"

#define IPV_TRY(x)               \
  do {                           \
    const ipv_status _s = (x);   \
    if (_s != IPV_OK) return _s; \
  } while (0)

namespace {

using namespace ipv;

static_assert(kFmtBf16 == IPV_PAGES_BF16 && kFmtF32 == IPV_PAGES_F32 && kFmtFp8 == IPV_PAGES_FP8 && kFmtFp4 == IPV_PAGES_FP4,
              "the formats of the header");
static_assert((int)kFmtBf16 == IPV_BF16 && (int)kFmtF32 == IPV_F32, "rows in the cache's types");
static_assert(kDevNan == IPV_DEV_NAN && kDevBadPage == IPV_DEV_BAD_PAGE, "the error bits of the header");

constexpr int32_t kMaxPosition = 1 << 30;  // positions and their tiles' ends stay in 31 bits
constexpr int64_t kGridThreads = 0xffffffffll;  // threads of a grid along one dimension, at most

[[maybe_unused]] bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

[[maybe_unused]] ipv_status launched(hipError_t e) { return e == hipSuccess ? IPV_OK : IPV_ERR_HIP; }

[[maybe_unused]] ipv_status check_pool_shape(const ipv_page_shape* s) {
  if (!s) return IPV_ERR_NULL;
  if (s->format < IPV_PAGES_BF16 || s->format > IPV_PAGES_FP4) return IPV_ERR_DTYPE;
  if (s->pages < 1 || s->layers < 1 || s->kv_heads < 1 || s->page_rows < 1 || s->page_rows > kMaxPosition) return IPV_ERR_SHAPE;
  if (s->head_dim != 32 && s->head_dim != 64 && s->head_dim != 128 && s->head_dim != 256) return IPV_ERR_SHAPE;
  // rows of the pool, and their bytes, in 63 bits
  const double rows = (double)s->pages * s->layers * s->kv_heads * s->page_rows;
  if (rows > 0x1p50) return IPV_ERR_SHAPE;
  return IPV_OK;
}

[[maybe_unused]] ipv_status check_pool(const ipv_page_shape* s, const void* K, const void* V, const uint8_t* Ks,
                                       const uint8_t* Vs, const int32_t* table, int32_t cols, int32_t streams, Pool* p) {
  IPV_TRY(check_pool_shape(s));
  const bool scaled = fmt_scaled(s->format);
  if (!K || !V || (scaled && (!Ks || !Vs))) return IPV_ERR_NULL;
  if (!aligned(K, 16) || !aligned(V, 16)) return IPV_ERR_ALIGN;
  if (scaled && (!aligned(Ks, 4) || !aligned(Vs, 4))) return IPV_ERR_ALIGN;
  if (table && !aligned(table, 4)) return IPV_ERR_ALIGN;
  if (streams < 1 || cols < 1) return IPV_ERR_SHAPE;
  if (!table && (cols != 1 || streams > s->pages)) return IPV_ERR_SHAPE;
  p->K = static_cast<char*>(const_cast<void*>(K));
  p->V = static_cast<char*>(const_cast<void*>(V));
  p->Ks = const_cast<uint8_t*>(Ks);
  p->Vs = const_cast<uint8_t*>(Vs);
  p->table = table;
  p->cols = cols;
  p->pages = s->pages;
  p->layer_rows = (int64_t)s->kv_heads * s->page_rows;
  p->page_rows_all = (int64_t)s->layers * p->layer_rows;
  p->T = make_fastdiv((uint32_t)s->page_rows);
  return IPV_OK;
}

// Rows that a stream's table covers (at most: positions stay in 31 bits).
[[maybe_unused]] int64_t table_rows(const ipv_page_shape* s, int32_t cols) {
  return std::min<int64_t>((int64_t)cols * s->page_rows, kMaxPosition);
}

[[maybe_unused]] ipv_status check_strides(const int64_t* strides, int n) {
  if (!strides) return IPV_ERR_NULL;
  for (int i = 0; i < n; ++i)
    if (strides[i] % 8 != 0) return IPV_ERR_ALIGN;
  return IPV_OK;
}

[[maybe_unused]] ipv_status check_word(const void* ws, size_t ws_bytes, size_t need) {
  if (!ws) return IPV_ERR_WORKSPACE;
  if (!aligned(ws, 256)) return IPV_ERR_ALIGN;
  return ws_bytes < need ? IPV_ERR_WORKSPACE : IPV_OK;
}

constexpr int32_t kMaxParts = 1024;  // workgroups of a launch of attention that splits, at most
// Attention's workspace: error word, counters (zero before and after a call), parts' maxima and sums, parts.
constexpr size_t kZeroed = kWsHeader + kMaxParts * sizeof(uint32_t);
static_assert(kZeroed == 4352, "the bytes to be zeroed that the header names");

[[maybe_unused]] ipv_status check_heads(const ipv_page_shape* s, int32_t streams, int32_t q_heads, int32_t max_rows) {
  if (streams < 1 || q_heads < 1 || max_rows < 1 || q_heads % s->kv_heads != 0) return IPV_ERR_SHAPE;
  if ((int64_t)q_heads * max_rows > kMaxPosition) return IPV_ERR_SHAPE;
  return IPV_OK;
}

// Blocks of rows.
[[maybe_unused]] ipv_status check_block_rows(const ipv_page_shape* s, int32_t block_rows, BlockMap* map) {
  if (block_rows < 16 || block_rows % 16 != 0 || s->page_rows % block_rows != 0) return IPV_ERR_SHAPE;
  map->R = make_fastdiv((uint32_t)block_rows);
  map->slices = (int64_t)s->layers * s->kv_heads;
  map->per = (uint32_t)(s->page_rows / block_rows);
  return IPV_OK;
}

// Bounds that are kept of them (none: NULL).
[[maybe_unused]] ipv_status check_bounds(const ipv_page_shape* s, const void* bounds, int32_t block_rows, BlockMap* map) {
  *map = BlockMap{make_fastdiv(1), (int64_t)s->layers * s->kv_heads, 1};
  if (!bounds) return IPV_OK;
  if (!aligned(bounds, 16)) return IPV_ERR_ALIGN;
  return check_block_rows(s, block_rows, map);
}

}  // namespace
