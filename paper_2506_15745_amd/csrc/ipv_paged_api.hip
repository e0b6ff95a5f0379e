// C entry points of the paged cache: argument checks, the split of the work and
// the launches. As in the pass, every check that the host can make comes before
// the first launch, and nothing here allocates, throws or waits.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/ipv.h"
#include "ipv_attend.hpp"
#include "ipv_paged_host.hpp"

using namespace ipv;

namespace {

template <bool WRITE, int F, int X, int D>
hipError_t page_launch(const PageCall& c, dim3 grid, hipStream_t st) {
  if constexpr (WRITE) k_page_write<F, X, D><<<grid, dim3(kPageThreads), 0, st>>>(c);
  else k_page_read<F, X, D><<<grid, dim3(kPageThreads), 0, st>>>(c);
  return hipGetLastError();
}

// Workgroups along the rows of a launch whose widest stream has `rows`.
int64_t page_blocks(int D, int64_t rows) {
  const int per = kPageThreads / (D / 16);
  return (rows + per - 1) / per;
}

template <bool WRITE, int F, int X>
hipError_t page_launch_d(int D, const PageCall& c, int32_t rows, hipStream_t st, int32_t streams) {
  const dim3 grid((uint32_t)page_blocks(D, rows), (uint32_t)(2 * ((c.LH + kPageSlices - 1) / kPageSlices)), (uint32_t)streams);
  switch (D) {
    case 32: return page_launch<WRITE, F, X, 32>(c, grid, st);
    case 64: return page_launch<WRITE, F, X, 64>(c, grid, st);
    case 128: return page_launch<WRITE, F, X, 128>(c, grid, st);
    default: return page_launch<WRITE, F, X, 256>(c, grid, st);
  }
}

template <bool WRITE, int F>
hipError_t page_launch_f(int dtype, int D, const PageCall& c, int32_t rows, hipStream_t st, int32_t streams) {
  return dtype == IPV_BF16 ? page_launch_d<WRITE, F, kFmtBf16>(D, c, rows, st, streams)
                           : page_launch_d<WRITE, F, kFmtF32>(D, c, rows, st, streams);
}

// ipv_page_write and ipv_page_read: the same checks, the same split.
template <bool WRITE>
ipv_status page_rows(const ipv_page_shape* s, const void* K_pages, const void* V_pages, const uint8_t* Ks, const uint8_t* Vs,
                     const int32_t* table, int32_t cols, int32_t streams, const int32_t* first, const int32_t* rows,
                     int32_t first_layer, int32_t layers, const void* K, const void* V, int32_t dtype,
                     const int64_t* strides, const float* rotary, int32_t rotary_rows, void* ws, size_t ws_bytes,
                     void* stream) {
  PageCall c;
  IPV_TRY(check_pool(s, K_pages, V_pages, Ks, Vs, table, cols, streams, &c.pool));
  if (!first || !rows || !K || !V) return IPV_ERR_NULL;
  if (dtype != IPV_BF16 && dtype != IPV_F32) return IPV_ERR_DTYPE;
  if (!aligned(K, 16) || !aligned(V, 16) || (rotary && !aligned(rotary, 16))) return IPV_ERR_ALIGN;
  IPV_TRY(check_strides(strides, 4));
  if (first_layer < 0 || layers < 1 || layers > s->layers - first_layer) return IPV_ERR_SHAPE;
  const int64_t slices = (int64_t)layers * s->kv_heads, groups = (slices + kPageSlices - 1) / kPageSlices;
  if (2 * groups > 65535) return IPV_ERR_SHAPE;  // a grid's second dimension
  for (int32_t b = 0; b < streams; ++b) {
    if (rows[b] < 0 || first[b] < 0) return IPV_ERR_SHAPE;
    const int64_t end = (int64_t)first[b] + rows[b];
    if (rows[b] > 0 && end > table_rows(s, cols)) return IPV_ERR_SHAPE;
    if (page_blocks(s->head_dim, rows[b]) * kPageThreads > kGridThreads) return IPV_ERR_SHAPE;
    if (rows[b] > 0 && rotary && end > rotary_rows) return IPV_ERR_ARG;
  }
  IPV_TRY(check_word(ws, ws_bytes, kWsHeader));
  c.K = static_cast<char*>(const_cast<void*>(K));
  c.V = static_cast<char*>(const_cast<void*>(V));
  c.sb = strides[0], c.sl = strides[1], c.sh = strides[2], c.sr = strides[3];
  c.rotary = rotary;
  c.err = static_cast<uint32_t*>(ws);
  c.H = s->kv_heads;
  c.LH = (int32_t)slices;
  c.first_slice = (int64_t)first_layer * c.pool.layer_rows;
  c.H_div = make_fastdiv((uint32_t)s->kv_heads);
  hipStream_t st = static_cast<hipStream_t>(stream);
  for (int32_t b0 = 0; b0 < streams; b0 += kPageStreams) {
    const int32_t nb = std::min(kPageStreams, streams - b0);
    int32_t most = 0;
    for (int32_t i = 0; i < nb; ++i) {
      c.first[i] = first[b0 + i], c.rows[i] = rows[b0 + i];
      most = std::max(most, rows[b0 + i]);
    }
    if (most == 0) continue;
    c.b0 = b0;
    hipError_t e;
    switch (s->format) {
      case IPV_PAGES_BF16: e = page_launch_f<WRITE, kFmtBf16>(dtype, s->head_dim, c, most, st, nb); break;
      case IPV_PAGES_F32: e = page_launch_f<WRITE, kFmtF32>(dtype, s->head_dim, c, most, st, nb); break;
      case IPV_PAGES_FP8: e = page_launch_f<WRITE, kFmtFp8>(dtype, s->head_dim, c, most, st, nb); break;
      default: e = page_launch_f<WRITE, kFmtFp4>(dtype, s->head_dim, c, most, st, nb); break;
    }
    IPV_TRY(launched(e));
  }
  return IPV_OK;
}

// ------------------------------------------------------------ attention
// Workgroups that the card's 256 CUs hold at once: with fewer row tiles than that,
// key ranges are split.
int32_t attend_fill(AttendKind k, int D, int format) {
  return 256 * (k == kTile ? 1 : k == kF32 ? (D <= 64 ? 2 : 1) : few_per_cu(format, D, k == kFew1 ? 1 : 2));
}

// The kernel for a call whose widest stream has `rows` rows a KV head.
AttendKind attend_kind(int format, int64_t rows) {
  if (format == IPV_PAGES_F32) return kF32;
  return rows <= 16 ? kFew1 : rows <= 32 ? kFew2 : kTile;
}

// Parts that launches of at most so many streams, and rows a KV head, can make.
int64_t max_parts(AttendKind k, int D, int32_t streams, int32_t kv_heads, int64_t rows) {
  const int64_t tiles = k == kFew1 || k == kFew2 ? 1 : (rows + attend_rows(k, D) - 1) / attend_rows(k, D);
  return std::min<int64_t>(std::min(streams, kAttendStreams) * (kv_heads * tiles) * kMaxSplits, kMaxParts);
}

size_t part_bytes(AttendKind k, int D, int64_t parts) { return (size_t)parts * attend_rows(k, D) * (size_t)(D + 2) * sizeof(float); }

// Every launch's row tiles as a grid (parts only add to it where it stays within kMaxParts).
ipv_status check_grids(const ipv_page_shape* s, int32_t streams, const int32_t* q_rows, int32_t q_heads) {
  const int64_t G = q_heads / s->kv_heads;
  for (int32_t b0 = 0; b0 < streams; b0 += kAttendStreams) {
    const int32_t* rows = q_rows + b0;
    const int32_t nb = std::min(kAttendStreams, streams - b0);
    const AttendKind kind = attend_kind(s->format, *std::max_element(rows, rows + nb) * G);
    const int32_t BM = attend_rows(kind, s->head_dim);
    int64_t tiles = 0;
    for (int32_t i = 0; i < nb; ++i) tiles += (rows[i] * G + BM - 1) / BM;
    if ((tiles * s->kv_heads + 7) / 8 * 8 * attend_threads(kind, s->head_dim) > kGridThreads) return IPV_ERR_SHAPE;
  }
  return IPV_OK;
}

// What `blocks` workgroups of `per` key tiles take, `fill` of them at once, us, as measured on bf16 and fp32
// pools. A workgroup costs its tiles and, around them, its start, the wait for its first rows and the store of its
// result or part; joining parts costs a launch and their bytes. A last round that does not fill the
// card costs a whole one, but for heads of 128: a full card lowers its clock for their products.
// Against no parts, where the row tiles do not fill the card's rounds: 300 tokens of 64 heads of 256 over
// 8192 positions 276 -> 220 us, 600 of 64 heads of 64 147 -> 124, 1100 of 64 heads of 128 385 -> 343; fp32,
// 300 tokens of 28 heads of 128 over 6272, 452 -> 332; where they leave most of it empty, 196 of those
// in bf16, 146 -> 41. Against parts that always fill a round: 400 tokens of 64 heads over 400 38 -> 21.
// Tiles of e4m3 and e2m1 take up to a seventh longer, which chooses no worse: those calls 353 -> 260 and 345 -> 252,
// 159 -> 130 and 165 -> 134, 410 -> 354 and 397 -> 348, 165 -> 43 and 158 -> 41; of heads of 128 with whole last
// rounds instead, 600 tokens of 64 heads over 8192 189 -> 193 and 185 -> 189, 1500 415 -> 408 and 403 -> 399.
double attend_us(AttendKind kind, int D, int64_t per, int64_t blocks, int32_t fill, bool parts) {
  const int size = D == 32 ? 0 : D == 64 ? 1 : D == 128 ? 2 : 3;
  static constexpr double kTileUs[4] = {0.8, 1.06, 1.8, 2.0}, kF32Us[4] = {0.67, 1.27, 1.1, 2.2};
  const int64_t whole = blocks / fill, rounds = (blocks + fill - 1) / fill;
  const double rest = (double)(blocks % fill) / fill, last = D != 128 ? 1 : whole == 0 ? 0.6 + 0.3 * rest : 0.5 + 0.45 * rest * rest;
  const double joins = parts ? 3.5 + 0.015 * attend_rows(kind, D) * D / 32768 * blocks : 0;
  if (kind == kF32) return rounds * (per * kF32Us[size] + 5 + D / 32.0) + joins;
  return (whole + (rest > 0 ? last : 0)) * per * kTileUs[size] + 13 + 8 * (rounds - 1) + joins;
}

// The split of one launch's streams: row tiles, parts of the key ranges, and the first workgroup of
// each. A key range is split when the row tiles alone leave the card, or its last round, unfilled.
void plan(AttendArgs* a, AttendKind kind, int D, int format) {
  const int32_t BM = attend_rows(kind, D), BN = attend_keys(kind);
  int64_t base = 0, work = 0;
  int32_t count[kAttendStreams];
  for (int32_t i = 0; i < a->streams; ++i) {
    AttendStream& s = a->s[i];
    s.tiles = (int32_t)(((int64_t)s.rows * a->G + BM - 1) / BM);
    s.splits = 1;
    // the longest of its row tiles' key ranges: the last one's, with the span of one tile
    const int32_t span = (BM + a->G - 1) / a->G + 1, p_hi = s.first + s.rows - 1;
    count[i] = s.rows > 0 ? KeyTiles(s.n, std::max(s.first, p_hi - span + 1), p_hi, a->window, a->sinks, BN).count : 0;
    base += (int64_t)a->H * s.tiles;
    work += (int64_t)a->H * s.tiles * count[i];
  }
  const int32_t fill = attend_fill(kind, D, format);
  const int32_t longest = *std::max_element(count, count + a->streams);
  const int64_t unit = kind == kTile ? 1 : kFewWaves;  // waves that share a workgroup's keys
  // splits for parts of `per` tiles; the workgroups
  const auto split = [&](int64_t per) {
    int64_t blocks = 0;
    for (int32_t i = 0; i < a->streams; ++i) {
      a->s[i].splits = (int32_t)std::min<int64_t>(std::max<int64_t>((count[i] + per - 1) / per, 1), kMaxSplits);
      blocks += (int64_t)a->H * a->s[i].tiles * a->s[i].splits;
    }
    return blocks;
  };
  if (kind == kTile || kind == kF32) {
    // Bound by computing: as many parts as the model below finds fastest.
    int64_t best = std::max(longest, 1);
    double least = 0;
    for (int64_t parts = 1; parts <= kMaxSplits && (parts == 1 || base * parts <= std::min<int64_t>(4 * fill, kMaxParts)); ++parts) {
      const int64_t per = ((std::max<int64_t>(longest, 1) + parts - 1) / parts + unit - 1) / unit * unit, blocks = split(per);
      if (parts > 1 && (per < 2 || blocks > kMaxParts)) break;
      const double us = attend_us(kind, D, per, blocks, fill, blocks > base);
      if (parts == 1 || us < least) least = parts == 1 ? 0.96 * us : us, best = per;  // (no parts for the model's error's sake)
    }
    split(best);
  } else if (base < fill) {
    // Bound by loading: parts of `per` tiles, the shortest that make no more workgroups than fit at once
    // and, where the last workgroup joins them, no shorter than a square root of the range: there a
    // step of four tiles, 0.65 us, costs what the parts it saves cost that workgroup, 0.1 us each.
    int64_t per = std::max<int64_t>({(work + fill - 1) / fill, kFewWaves, a->join_apart ? 0 : (int64_t)std::sqrt(0.6 * longest)});
    per = (per + unit - 1) / unit * unit;
    for (;; per += std::max(unit, per / 16 / unit * unit)) {
      const int64_t blocks = split(per);
      if (blocks <= fill || blocks == base) break;
    }
  }
  int64_t at = 0;
  for (int32_t i = 0; i < a->streams; ++i) {
    a->s[i].start = (int32_t)at;
    a->s[i].by_tiles = make_fastdiv((uint32_t)std::max(a->s[i].tiles, 1));
    a->s[i].by_splits = make_fastdiv((uint32_t)a->s[i].splits);
    at += (int64_t)a->H * a->s[i].tiles * a->s[i].splits;
  }
  a->blocks = (int32_t)at;
}

int32_t most_splits(const AttendArgs& a) {
  int32_t most = 1;
  for (int32_t i = 0; i < a.streams; ++i) most = std::max(most, a.s[i].splits);
  return most;
}

// Trips to other workgroups' parts, over a microsecond each, that the last workgroup of a row tile would
// make to join them: four elements a thread, 16 parts at a time. A launch that joins them a wave a row
// costs as much as two to three: one token of 28 heads of 128 over 1000 positions (one trip) 7.5 us
// joined by the last workgroup and 10.1 by a launch, four tokens over 6272 (eight trips) 20.4 and 14.1,
// of heads of 256 34.7 and 20.5.
int64_t join_trips(const AttendArgs& a, AttendKind kind, int D, int32_t most_rows) {
  const int32_t splits = most_splits(a);
  if (splits == 1) return 0;
  const int64_t rows = std::min<int64_t>((int64_t)most_rows * a.G, attend_rows(kind, D));
  return join_rounds(rows, D) * ((splits + 15) / 16);
}

}  // namespace

template <bool F32OUT>
static void launch_join_t(int D, dim3 grid, int32_t BM, const AttendArgs& a, hipStream_t st) {
  const dim3 block(256);
  switch (D) {
    case 32: k_attend_join<32, F32OUT><<<grid, block, 0, st>>>(a, BM); break;
    case 64: k_attend_join<64, F32OUT><<<grid, block, 0, st>>>(a, BM); break;
    case 128: k_attend_join<128, F32OUT><<<grid, block, 0, st>>>(a, BM); break;
    default: k_attend_join<256, F32OUT><<<grid, block, 0, st>>>(a, BM); break;
  }
}

static hipError_t launch_join(int D, bool f32, uint32_t rows, int32_t BM, const AttendArgs& a, hipStream_t st) {
  const dim3 grid((rows + 3) / 4, (uint32_t)a.streams);
  if (f32) launch_join_t<true>(D, grid, BM, a, st);
  else launch_join_t<false>(D, grid, BM, a, st);
  return hipGetLastError();
}

extern "C" {

ipv_status ipv_page_write(const ipv_page_shape* pool, void* K_pages, void* V_pages, uint8_t* K_scales,
                          uint8_t* V_scales, const int32_t* page_table, int32_t table_cols, int32_t streams,
                          const int32_t* first_row, const int32_t* rows, int32_t first_layer, int32_t layers,
                          const void* K, const void* V, int32_t dtype, const int64_t* strides, const float* rotary,
                          int32_t rotary_rows, void* ws, size_t ws_bytes, void* stream) {
  return page_rows<true>(pool, K_pages, V_pages, K_scales, V_scales, page_table, table_cols, streams, first_row, rows,
                         first_layer, layers, K, V, dtype, strides, rotary, rotary_rows, ws, ws_bytes, stream);
}

ipv_status ipv_page_read(const ipv_page_shape* pool, const void* K_pages, const void* V_pages, const uint8_t* K_scales,
                         const uint8_t* V_scales, const int32_t* page_table, int32_t table_cols, int32_t streams,
                         const int32_t* first_row, const int32_t* rows, int32_t first_layer, int32_t layers, void* K,
                         void* V, int32_t dtype, const int64_t* strides, const float* rotary, int32_t rotary_rows,
                         void* ws, size_t ws_bytes, void* stream) {
  return page_rows<false>(pool, K_pages, V_pages, K_scales, V_scales, page_table, table_cols, streams, first_row, rows,
                          first_layer, layers, K, V, dtype, strides, rotary, rotary_rows, ws, ws_bytes, stream);
}

ipv_status ipv_attend_workspace_bytes(const ipv_page_shape* pool, int32_t streams, int32_t q_heads, int32_t max_rows,
                                      size_t* bytes) {
  if (!bytes) return IPV_ERR_NULL;
  IPV_TRY(check_pool_shape(pool));
  IPV_TRY(check_heads(pool, streams, q_heads, max_rows));
  // a call of fewer rows may take a kernel of narrower tiles
  const int64_t rows = (int64_t)max_rows * (q_heads / pool->kv_heads);
  const AttendKind widest = attend_kind(pool->format, rows);
  const int D = pool->head_dim;
  size_t parts = 0;
  for (AttendKind k : {kFew1, kFew2, kTile, kF32})
    if (k <= widest && (k == kF32) == (widest == kF32))
      parts = std::max(parts, part_bytes(k, D, max_parts(k, D, streams, pool->kv_heads, rows)));
  *bytes = kZeroed + parts;
  return IPV_OK;
}

ipv_status ipv_attend(const ipv_page_shape* pool, const void* K_pages, const void* V_pages, const uint8_t* K_scales,
                      const uint8_t* V_scales, const int32_t* page_table, int32_t table_cols, int32_t streams,
                      const int32_t* n_tokens, const int32_t* q_first, const int32_t* q_rows, int32_t layer,
                      const void* q, const int64_t* q_strides, int32_t q_heads, int32_t max_rows, double scale,
                      int32_t window, int32_t sinks, void* out, const int64_t* out_strides, float* lse, void* ws,
                      size_t ws_bytes, void* stream) {
  AttendArgs a;
  IPV_TRY(check_pool(pool, K_pages, V_pages, K_scales, V_scales, page_table, table_cols, streams, &a.pool));
  if (!n_tokens || !q_first || !q_rows || !q || !out) return IPV_ERR_NULL;
  IPV_TRY(check_heads(pool, streams, q_heads, max_rows));
  if (!aligned(q, 16) || !aligned(out, 16) || (lse && !aligned(lse, 4))) return IPV_ERR_ALIGN;
  IPV_TRY(check_strides(q_strides, 3));
  IPV_TRY(check_strides(out_strides, 3));
  if (layer < 0 || layer >= pool->layers) return IPV_ERR_SHAPE;
  if (!(scale > 0) || !std::isfinite(scale) || !std::isnormal((float)(scale * 1.4426950408889634)) || window < 0 ||
      sinks < 0)
    return IPV_ERR_ARG;
  for (int32_t b = 0; b < streams; ++b) {
    if (n_tokens[b] < 0 || n_tokens[b] > table_rows(pool, table_cols)) return IPV_ERR_SHAPE;
    if (q_rows[b] < 0 || q_rows[b] > max_rows || q_first[b] < 0 || q_first[b] > kMaxPosition - q_rows[b]) return IPV_ERR_SHAPE;
  }
  IPV_TRY(check_grids(pool, streams, q_rows, q_heads));
  size_t need = 0;
  IPV_TRY(ipv_attend_workspace_bytes(pool, streams, q_heads, max_rows, &need));
  IPV_TRY(check_word(ws, ws_bytes, need));

  a.layer_row = (int64_t)layer * a.pool.layer_rows;
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.q_b = q_strides[0], a.q_h = q_strides[1], a.q_m = q_strides[2];
  a.o_b = out_strides[0], a.o_h = out_strides[1], a.o_m = out_strides[2];
  a.H = pool->kv_heads;
  a.G = q_heads / pool->kv_heads;
  a.max_rows = max_rows;
  a.G_div = make_fastdiv((uint32_t)a.G);
  a.c = (float)(scale * 1.4426950408889634);
  a.window = window > kMaxPosition ? 0 : window;  // (wider than any range: none, and sums with it stay in 32 bits)
  a.sinks = std::min(sinks, kMaxPosition);
  a.err = static_cast<uint32_t*>(ws);
  hipStream_t st = static_cast<hipStream_t>(stream);
  for (int32_t b0 = 0; b0 < streams; b0 += kAttendStreams) {
    a.b0 = b0;
    a.streams = std::min(kAttendStreams, streams - b0);
    int32_t most = 0;
    for (int32_t i = 0; i < a.streams; ++i) {
      a.s[i].n = n_tokens[b0 + i], a.s[i].first = q_first[b0 + i], a.s[i].rows = q_rows[b0 + i];
      most = std::max(most, q_rows[b0 + i]);
    }
    if (most == 0) continue;
    const AttendKind kind = attend_kind(pool->format, (int64_t)most * a.G);
    a.join_apart = kind == kTile;
    plan(&a, kind, pool->head_dim, pool->format);
    if (!a.join_apart && join_trips(a, kind, pool->head_dim, most) > kJoinTrips) {
      a.join_apart = 1;
      if (kind != kF32) plan(&a, kind, pool->head_dim, pool->format);  // (parts may be shorter then)
    }
    a.arrived = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + kWsHeader);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + kZeroed);
    a.part = a.part_ml + (size_t)a.blocks * attend_rows(kind, pool->head_dim) * 2;  // (a launch that splits has at most max_parts)
    const uint32_t grid = (uint32_t)(a.blocks + 7) / 8u * 8u;
    hipError_t e;
    switch (pool->format) {
      case IPV_PAGES_BF16: e = launch_attend<kFmtBf16>(pool->head_dim, kind, grid, a, st); break;
      case IPV_PAGES_F32: e = launch_attend<kFmtF32>(pool->head_dim, kind, grid, a, st); break;
      case IPV_PAGES_FP8: e = launch_attend<kFmtFp8>(pool->head_dim, kind, grid, a, st); break;
      default: e = launch_attend<kFmtFp4>(pool->head_dim, kind, grid, a, st); break;
    }
    IPV_TRY(launched(e));
    if (a.join_apart && most_splits(a) > 1)
      IPV_TRY(launched(launch_join(pool->head_dim, kind == kF32, (uint32_t)most * (uint32_t)q_heads,
                                   attend_rows(kind, pool->head_dim), a, st)));
  }
  return IPV_OK;
}

}  // extern "C"
