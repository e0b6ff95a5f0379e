// C entry points of new tokens, block bounds, compaction and copies of pages: argument
// checks and launches. Every check that the host can make comes before the first
// launch, and nothing here allocates, throws or waits.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/ipv.h"
#include "ipv_rows.hpp"
#include "ipv_paged_host.hpp"

using namespace ipv;

static_assert(kDevBadKeep == IPV_DEV_BAD_KEEP, "the error bits of the header");

namespace {

int64_t row_blocks(int D, int64_t rows) {
  const int64_t per = kPageThreads / (D / 16);
  return (rows + per - 1) / per;
}

// Blocks that positions [first, first + rows) reach into.
int64_t touched(int32_t first, int32_t rows, int32_t block_rows) {
  return rows == 0 ? 0 : ((int64_t)first + rows - 1) / block_rows - first / block_rows + 1;
}

// `what` for the kernel of this format, and head size.
template <int D, class CALL>
hipError_t by_format(int format, const CALL& what) {
  switch (format) {
    case IPV_PAGES_BF16: what(std::integral_constant<int, kFmtBf16>(), std::integral_constant<int, D>()); break;
    case IPV_PAGES_F32: what(std::integral_constant<int, kFmtF32>(), std::integral_constant<int, D>()); break;
    case IPV_PAGES_FP8: what(std::integral_constant<int, kFmtFp8>(), std::integral_constant<int, D>()); break;
    default: what(std::integral_constant<int, kFmtFp4>(), std::integral_constant<int, D>()); break;
  }
  return hipGetLastError();
}
template <class CALL>
hipError_t by_shape(const ipv_page_shape* s, const CALL& what) {
  switch (s->head_dim) {
    case 32: return by_format<32>(s->format, what);
    case 64: return by_format<64>(s->format, what);
    case 128: return by_format<128>(s->format, what);
    default: return by_format<256>(s->format, what);
  }
}

// Whether a grid holds that many workgroups side by side.
bool in_grid(int64_t blocks) { return blocks * kPageThreads <= kGridThreads; }

// Counts of positions from first[b] on, as ipv_page_write checks them; blocks(b): workgroups that a stream's take.
template <class BLOCKS>
ipv_status check_positions(const ipv_page_shape* s, int32_t cols, int32_t streams, const int32_t* first, const int32_t* rows,
                           const float* rotary, int32_t rotary_rows, const BLOCKS& blocks) {
  for (int32_t b = 0; b < streams; ++b) {
    if (rows[b] < 0 || first[b] < 0) return IPV_ERR_SHAPE;
    const int64_t end = (int64_t)first[b] + rows[b];
    if (rows[b] > 0 && end > table_rows(s, cols)) return IPV_ERR_SHAPE;
    if (!in_grid(blocks(b))) return IPV_ERR_SHAPE;
    if (rows[b] > 0 && rotary && end > rotary_rows) return IPV_ERR_ARG;
  }
  return IPV_OK;
}

}  // namespace

extern "C" {

ipv_status ipv_qkv_write(const ipv_page_shape* pool, void* K_pages, void* V_pages, uint8_t* K_scales, uint8_t* V_scales,
                         void* bounds, int32_t block_rows, const int32_t* page_table, int32_t table_cols, int32_t streams,
                         const int32_t* first_row, const int32_t* rows, int32_t layer, const void* q,
                         const int64_t* q_strides, int32_t q_heads, const void* k, const void* v, const int64_t* kv_strides,
                         int32_t dtype, const float* q_norm, const float* k_norm, double eps, const float* rotary,
                         int32_t rotary_rows, void* q_out, const int64_t* out_strides, void* ws, size_t ws_bytes,
                         void* stream) {
  TokenCall c;
  IPV_TRY(check_pool(pool, K_pages, V_pages, K_scales, V_scales, page_table, table_cols, streams, &c.pool));
  IPV_TRY(check_bounds(pool, bounds, block_rows, &c.map));
  if (!first_row || !rows || !q || !k || !v || !q_out) return IPV_ERR_NULL;
  if (dtype != IPV_BF16 && dtype != IPV_F32) return IPV_ERR_DTYPE;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || (rotary && !aligned(rotary, 16)) ||
      (q_norm && !aligned(q_norm, 4)) || (k_norm && !aligned(k_norm, 4)))
    return IPV_ERR_ALIGN;
  IPV_TRY(check_strides(q_strides, 3));
  IPV_TRY(check_strides(kv_strides, 3));
  IPV_TRY(check_strides(out_strides, 3));
  if (layer < 0 || layer >= pool->layers || q_heads < 1 || q_heads % pool->kv_heads != 0) return IPV_ERR_SHAPE;
  if ((q_norm || k_norm) && (!(eps > 0) || !std::isnormal((float)eps))) return IPV_ERR_ARG;
  const auto blocks_of = [&](int32_t b) {
    const int64_t blocks = row_blocks(pool->head_dim, rows[b]);
    return bounds ? std::max(blocks, touched(first_row[b], rows[b], block_rows)) : blocks;
  };
  IPV_TRY(check_positions(pool, table_cols, streams, first_row, rows, rotary, rotary_rows, blocks_of));
  const int32_t kv_groups = (pool->kv_heads + kTokenHeads - 1) / kTokenHeads;
  const int64_t q_groups = ((int64_t)q_heads + kTokenHeads - 1) / kTokenHeads;
  const int64_t groups = q_groups + kv_groups + (bounds ? pool->kv_heads : kv_groups);
  if (groups > 65535) return IPV_ERR_SHAPE;  // a grid's second dimension
  IPV_TRY(check_word(ws, ws_bytes, kWsHeader));
  c.q = static_cast<const char*>(q), c.k = static_cast<const char*>(k), c.v = static_cast<const char*>(v);
  c.q_out = static_cast<char*>(q_out);
  c.bounds = static_cast<char*>(bounds);
  c.q_b = q_strides[0], c.q_h = q_strides[1], c.q_m = q_strides[2];
  c.k_b = kv_strides[0], c.k_h = kv_strides[1], c.k_m = kv_strides[2];
  c.o_b = out_strides[0], c.o_h = out_strides[1], c.o_m = out_strides[2];
  c.q_norm = q_norm, c.k_norm = k_norm, c.rotary = rotary;
  c.eps = eps;
  c.err = static_cast<uint32_t*>(ws);
  c.A = q_heads, c.H = pool->kv_heads, c.layer = layer;
  c.q_groups = (int32_t)q_groups, c.v_groups = kv_groups;
  hipStream_t st = static_cast<hipStream_t>(stream);
  for (int32_t b0 = 0; b0 < streams; b0 += kPageStreams) {
    const int32_t nb = std::min(kPageStreams, streams - b0);
    int64_t blocks = 0;
    for (int32_t i = 0; i < nb; ++i) {
      c.first[i] = first_row[b0 + i], c.rows[i] = rows[b0 + i];
      blocks = std::max(blocks, blocks_of(b0 + i));
    }
    if (blocks == 0) continue;
    c.b0 = b0;
    const dim3 grid((uint32_t)blocks, (uint32_t)groups, (uint32_t)nb), block(kPageThreads);
    IPV_TRY(launched(by_shape(pool, [&](auto f, auto d) {
      constexpr int F = decltype(f)::value, D = decltype(d)::value;
      if (dtype == IPV_BF16) k_qkv_write<F, kFmtBf16, D><<<grid, block, 0, st>>>(c);
      else k_qkv_write<F, kFmtF32, D><<<grid, block, 0, st>>>(c);
    })));
  }
  return IPV_OK;
}

ipv_status ipv_block_bounds(const ipv_page_shape* pool, const void* K_pages, const uint8_t* K_scales, void* bounds,
                            int32_t block_rows, const int32_t* page_table, int32_t table_cols, int32_t streams,
                            const int32_t* first_row, const int32_t* rows, int32_t first_layer, int32_t layers, void* ws,
                            size_t ws_bytes, void* stream) {
  BoundsCall c;
  IPV_TRY(check_pool(pool, K_pages, K_pages, K_scales, K_scales, page_table, table_cols, streams, &c.pool));
  if (!bounds || !first_row || !rows) return IPV_ERR_NULL;
  IPV_TRY(check_bounds(pool, bounds, block_rows, &c.map));
  if (first_layer < 0 || layers < 1 || layers > pool->layers - first_layer) return IPV_ERR_SHAPE;
  const int64_t slices = (int64_t)layers * pool->kv_heads;
  if (slices > 65535) return IPV_ERR_SHAPE;  // a grid's second dimension
  const auto blocks_of = [&](int32_t b) { return touched(first_row[b], rows[b], block_rows); };
  IPV_TRY(check_positions(pool, table_cols, streams, first_row, rows, nullptr, 0, blocks_of));
  IPV_TRY(check_word(ws, ws_bytes, kWsHeader));
  c.bounds = static_cast<char*>(bounds);
  c.err = static_cast<uint32_t*>(ws);
  c.first_slice = (uint32_t)(first_layer * pool->kv_heads);
  hipStream_t st = static_cast<hipStream_t>(stream);
  for (int32_t b0 = 0; b0 < streams; b0 += kPageStreams) {
    const int32_t nb = std::min(kPageStreams, streams - b0);
    int64_t blocks = 0;
    for (int32_t i = 0; i < nb; ++i) {
      c.first[i] = first_row[b0 + i], c.rows[i] = rows[b0 + i];
      blocks = std::max(blocks, blocks_of(b0 + i));
    }
    if (blocks == 0) continue;
    c.b0 = b0;
    const dim3 grid((uint32_t)blocks, (uint32_t)slices, (uint32_t)nb);
    IPV_TRY(launched(by_shape(pool, [&](auto f, auto d) {
      k_block_bounds<decltype(f)::value, decltype(d)::value><<<grid, dim3(kPageThreads), 0, st>>>(c);
    })));
  }
  return IPV_OK;
}

ipv_status ipv_page_compact(const ipv_page_shape* pool, void* K_pages, void* V_pages, uint8_t* K_scales, uint8_t* V_scales,
                            void* bounds, int32_t block_rows, const int32_t* page_table, int32_t table_cols,
                            const int32_t* new_table, int32_t new_cols, int32_t streams, const int32_t* n_tokens,
                            const int32_t* keep_idx, int32_t C, const int32_t* rows, const float* rotary,
                            int32_t rotary_rows, void* ws, size_t ws_bytes, void* stream) {
  CompactCall c;
  IPV_TRY(check_pool(pool, K_pages, V_pages, K_scales, V_scales, page_table, table_cols, streams, &c.pool));
  IPV_TRY(check_bounds(pool, bounds, block_rows, &c.map));
  if (!new_table || !n_tokens || !keep_idx || !rows) return IPV_ERR_NULL;
  if (!aligned(new_table, 4) || !aligned(keep_idx, 4) || (rotary && !aligned(rotary, 16))) return IPV_ERR_ALIGN;
  if (new_cols < 1 || C < 1) return IPV_ERR_SHAPE;
  if (2 * c.map.slices > 65535) return IPV_ERR_SHAPE;  // a grid's second dimension
  const auto blocks_of = [&](int32_t b) {
    int64_t blocks = 0;
    for (bool with : {false, bounds != nullptr}) {
      const int64_t per = compact_run(with, c.map.R.d);
      blocks = std::max(blocks, (rows[b] + per - 1) / per);
    }
    return blocks;
  };
  for (int32_t b = 0; b < streams; ++b) {
    if (n_tokens[b] < 0 || n_tokens[b] > table_rows(pool, table_cols)) return IPV_ERR_SHAPE;
    if (rows[b] < 0 || rows[b] > C || rows[b] > table_rows(pool, new_cols)) return IPV_ERR_SHAPE;
    if (!in_grid(blocks_of(b))) return IPV_ERR_SHAPE;
    if (rows[b] > 0 && rotary && (n_tokens[b] > rotary_rows || rows[b] > rotary_rows)) return IPV_ERR_ARG;
  }
  IPV_TRY(check_word(ws, ws_bytes, kWsHeader));
  c.bounds = static_cast<char*>(bounds);
  c.new_table = new_table;
  c.keep = keep_idx;
  c.rotary = rotary;
  c.err = static_cast<uint32_t*>(ws);
  c.new_cols = new_cols;
  c.C = C;
  hipStream_t st = static_cast<hipStream_t>(stream);
  for (int32_t b0 = 0; b0 < streams; b0 += kPageStreams) {
    const int32_t nb = std::min(kPageStreams, streams - b0);
    int64_t blocks = 0;
    for (int32_t i = 0; i < nb; ++i) {
      c.n[i] = n_tokens[b0 + i], c.rows[i] = rows[b0 + i];
      blocks = std::max(blocks, blocks_of(b0 + i));
    }
    if (blocks == 0) continue;
    c.b0 = b0;
    const dim3 grid((uint32_t)blocks, (uint32_t)(2 * ((c.map.slices + kCompactWaves - 1) / kCompactWaves)), (uint32_t)nb);
    IPV_TRY(launched(by_shape(pool, [&](auto f, auto d) {
      constexpr int F = decltype(f)::value, D = decltype(d)::value;
      const dim3 block(kPageThreads);
      if (rotary && bounds) k_page_compact<F, D, true, true><<<grid, block, 0, st>>>(c);
      else if (rotary) k_page_compact<F, D, true, false><<<grid, block, 0, st>>>(c);
      else if (bounds) k_page_compact<F, D, false, true><<<grid, block, 0, st>>>(c);
      else k_page_compact<F, D, false, false><<<grid, block, 0, st>>>(c);
    })));
  }
  return IPV_OK;
}

ipv_status ipv_page_copy(const ipv_page_shape* pool, void* K_pages, void* V_pages, uint8_t* K_scales, uint8_t* V_scales,
                         void* bounds, int32_t block_rows, const int32_t* from, const int32_t* to, int32_t count,
                         int32_t rows, void* ws, size_t ws_bytes, void* stream) {
  Pool p;
  BlockMap map;
  IPV_TRY(check_pool(pool, K_pages, V_pages, K_scales, V_scales, nullptr, 1, 1, &p));
  IPV_TRY(check_bounds(pool, bounds, block_rows, &map));
  if (!from || !to) return IPV_ERR_NULL;
  if (!aligned(from, 4) || !aligned(to, 4)) return IPV_ERR_ALIGN;
  if (count < 0 || rows < 1 || rows > pool->page_rows) return IPV_ERR_SHAPE;
  const int D = pool->head_dim, format = pool->format;
  const int64_t T = pool->page_rows;
  const bool scaled = fmt_scaled(format);
  // `held` of `all` bytes of each of a page's slices
  const auto part = [&](void* base, int64_t held, int64_t all, int unit) {
    CopyPart c;
    c.base = static_cast<char*>(base);
    c.page_units = map.slices * all / unit;
    c.slice_units = held == all ? 1 : all / unit;
    c.units = make_fastdiv(held == all ? 1u : (uint32_t)(held / unit));
    c.all = held == all ? c.page_units : map.slices * (held / unit);
    return c;
  };
  CopyCall rows_call, scales_call;
  const int64_t row = fmt_row_bytes(format, D), scale = D / kScaleBlock, bound = bound_bytes(format, D);
  if (map.slices * T * row / 16 > kGridThreads) return IPV_ERR_SHAPE;  // a page's 16 bytes are counted in 32 bits
  rows_call.part[0] = part(K_pages, rows * row, T * row, 16);
  rows_call.part[1] = part(V_pages, rows * row, T * row, 16);
  int parts = 2;
  if (bounds) rows_call.part[parts++] = part(bounds, (rows + block_rows - 1) / block_rows * bound, T / block_rows * bound, 16);
  // scales: whole pages, or their slices, by words where those are whole words
  const bool whole = rows == T;
  const bool words = whole ? map.slices * T * scale % 4 == 0 : rows * scale % 4 == 0 && T * scale % 4 == 0;
  if (scaled) {
    if (map.slices * T * scale > kGridThreads) return IPV_ERR_SHAPE;
    scales_call.part[0] = part(K_scales, rows * scale, T * scale, words ? 4 : 1);
    scales_call.part[1] = part(V_scales, rows * scale, T * scale, words ? 4 : 1);
  }
  IPV_TRY(check_word(ws, ws_bytes, kWsHeader));
  hipStream_t st = static_cast<hipStream_t>(stream);
  for (CopyCall* c : {&rows_call, &scales_call}) c->from = from, c->to = to, c->err = static_cast<uint32_t*>(ws), c->pages = pool->pages;
  for (int32_t z0 = 0; z0 < count; z0 += 65535) {
    const uint32_t nz = (uint32_t)std::min(count - z0, 65535);
    const auto grid = [&](const CopyCall& c, int n) {
      int64_t all = 0;
      for (int i = 0; i < n; ++i) all = std::max(all, c.part[i].all);
      return dim3((uint32_t)((all + kPageThreads * kCopyUnits - 1) / (kPageThreads * kCopyUnits)), (uint32_t)n, nz);
    };
    k_page_copy<U32x4><<<grid(rows_call, parts), dim3(kPageThreads), 0, st>>>(rows_call, z0);
    IPV_TRY(launched(hipGetLastError()));
    if (!scaled) continue;
    if (words) k_page_copy<uint32_t><<<grid(scales_call, 2), dim3(kPageThreads), 0, st>>>(scales_call, z0);
    else k_page_copy<uint8_t><<<grid(scales_call, 2), dim3(kPageThreads), 0, st>>>(scales_call, z0);
    IPV_TRY(launched(hipGetLastError()));
  }
  return IPV_OK;
}

}  // extern "C"
