// C entry points of attention over chosen blocks: argument checks, the split of the work and
// the launches. Every check that the host can make comes before the first launch, and nothing
// here allocates, throws or waits.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/ipv.h"
#include "ipv_blocks.hpp"
#include "ipv_paged_host.hpp"

using namespace ipv;

namespace {

constexpr int32_t kMaxTop = 4096;
// Tiles of queries from which on a workgroup takes all blocks of its own: 128 of them over 64 blocks 12.8 us so and 18.6
// shared out among four, over 512 33.5 and 33.7; 64 over 512 33.0 and 26.4.
constexpr int32_t kOwnBlocks = 128;
// Whether each query of a launch has a workgroup of its own: for up to 2048 blocks (its scores are in LDS), where the
// times that the two ways take, as they were measured, say so. A workgroup: what it takes for all blocks, or what all
// workgroups take on the card, by the bounds' bytes. Tiles of 16 queries: what they take at least, and the matrix
// unit's time, by the tiles. E. g. us alone and in tiles (captured runs of calls), 8 KV heads of 128 in bf16: 16 tokens over
// 64 blocks 7.0 and 15, over 512 14 and 18; 64 over 256 15 and 20, over 512 21 and 22; 128 over 64 12 and 15, over 256 27 (512 threads) and
// 21; 512 over 64 50 and 14, over 512 142 and 36; one token of 64 streams over 256 18 and 32, of one over 512 13 and 9.
// Heads of 256: 64 over 64 10 and 19, 512 over 256 151 and 36; of 32: 256 over 256 18 and 21, 512 over 64 15 and 11.
bool select_alone(int64_t queries, int32_t of_stream, int32_t units, int32_t padded, int32_t D, int32_t block_bytes) {
  if (padded > 32 * kWave) return false;
  const double bytes = block_bytes, blocks = padded, all = (double)queries * bytes;
  const double alone = std::max(6000.0 + blocks * bytes / 32, 3000.0 + (double)queries + all * (155 + blocks) * 0.65e-4);  // ns
  const double tiles = 10000.0 + (units < kOwnBlocks ? 300 * std::min(of_stream, kScoreTile) : 1000) + (double)units * blocks * D / 850;
  return alone < tiles;
}
constexpr int64_t kScoreBytes = 128ll << 20;  // of scores at a time, where 16 queries of each stream need no more

int32_t padded_blocks(int32_t n, int32_t block_rows) {
  const int64_t blocks = ((int64_t)n + block_rows - 1) / block_rows;
  return (int32_t)((blocks + kScoreTile - 1) / kScoreTile * kScoreTile);
}

// Bytes of the scores of one query of each stream of a launch.
int64_t score_bytes(int32_t streams, int32_t kv_heads, int64_t padded) {
  return std::min(streams, kAttendStreams) * (int64_t)kv_heads * padded * (int64_t)sizeof(double);
}

ipv_status check_lists(const ipv_page_shape* s, int32_t block_rows, int32_t top, BlockMap* map) {
  IPV_TRY(check_block_rows(s, block_rows, map));
  if (top < 1 || top > kMaxTop || (int64_t)top * block_rows > kMaxPosition) return IPV_ERR_SHAPE;
  return IPV_OK;
}

// Query heads of a workgroup.
int32_t block_heads(const ipv_page_shape* s, int32_t G) { return s->format != IPV_PAGES_F32 && G > 16 ? 32 : 16; }

struct Counts {
  int32_t streams, cols;
  const int32_t *n, *first, *rows;
};
ipv_status check_counts(const ipv_page_shape* s, const Counts& c, int32_t max_rows) {
  for (int32_t b = 0; b < c.streams; ++b) {
    if (c.n[b] < 0 || c.n[b] > table_rows(s, c.cols)) return IPV_ERR_SHAPE;
    if (c.rows[b] < 0 || c.rows[b] > max_rows || c.first[b] < 0 || c.first[b] > kMaxPosition - c.rows[b]) return IPV_ERR_SHAPE;
  }
  return IPV_OK;
}

// Least bytes for scores that a call can do with: 16 queries of each stream at a time, or all.
int64_t least_scores(const ipv_page_shape* s, int32_t streams, int32_t max_rows, int32_t n, int32_t block_rows) {
  return score_bytes(streams, s->kv_heads, padded_blocks(n, block_rows)) * std::min(max_rows, kScoreTile);
}

struct Select {
  SelectArgs a;
  const ipv_page_shape* pool;
  int64_t room;  // bytes for scores
};

template <int FB, int D, bool SPLIT>
void launch_select_n(dim3 grid, const SelectArgs& a, hipStream_t st) {
  const dim3 block(select_threads(FB, D, SPLIT));
  if (a.padded <= 8 * kWave) k_block_select<FB, D, 8, SPLIT><<<grid, block, 0, st>>>(a);
  else if (a.padded <= 32 * kWave) k_block_select<FB, D, 32, SPLIT><<<grid, block, 0, st>>>(a);
  else k_block_select<FB, D, 0, SPLIT><<<grid, block, 0, st>>>(a);
}
template <bool SPLIT>
void launch_select(const ipv_page_shape* s, dim3 grid, const SelectArgs& a, hipStream_t st) {
  const bool f32 = s->format == IPV_PAGES_F32;
  switch (s->head_dim) {
    case 32: f32 ? launch_select_n<kFmtF32, 32, SPLIT>(grid, a, st) : launch_select_n<kFmtBf16, 32, SPLIT>(grid, a, st); break;
    case 64: f32 ? launch_select_n<kFmtF32, 64, SPLIT>(grid, a, st) : launch_select_n<kFmtBf16, 64, SPLIT>(grid, a, st); break;
    case 128: f32 ? launch_select_n<kFmtF32, 128, SPLIT>(grid, a, st) : launch_select_n<kFmtBf16, 128, SPLIT>(grid, a, st); break;
    default: f32 ? launch_select_n<kFmtF32, 256, SPLIT>(grid, a, st) : launch_select_n<kFmtBf16, 256, SPLIT>(grid, a, st); break;
  }
}

template <int FB, int D>
void launch_one_d(dim3 grid, const SelectArgs& a, hipStream_t st) {
  const bool few = (int64_t)grid.x * grid.y * grid.z <= 256;
  if (a.padded <= 8 * kWave && few) k_block_select_one<FB, D, 8, 512><<<grid, dim3(512), 0, st>>>(a);
  else if (a.padded <= 8 * kWave) k_block_select_one<FB, D, 8, 256><<<grid, dim3(256), 0, st>>>(a);
  else if (few) k_block_select_one<FB, D, 32, 512><<<grid, dim3(512), 0, st>>>(a);
  else k_block_select_one<FB, D, 32, 256><<<grid, dim3(256), 0, st>>>(a);
}
void launch_one(const ipv_page_shape* s, dim3 grid, const SelectArgs& a, hipStream_t st) {
  const bool f32 = s->format == IPV_PAGES_F32;
  switch (s->head_dim) {
    case 32: f32 ? launch_one_d<kFmtF32, 32>(grid, a, st) : launch_one_d<kFmtBf16, 32>(grid, a, st); break;
    case 64: f32 ? launch_one_d<kFmtF32, 64>(grid, a, st) : launch_one_d<kFmtBf16, 64>(grid, a, st); break;
    case 128: f32 ? launch_one_d<kFmtF32, 128>(grid, a, st) : launch_one_d<kFmtBf16, 128>(grid, a, st); break;
    default: f32 ? launch_one_d<kFmtF32, 256>(grid, a, st) : launch_one_d<kFmtBf16, 256>(grid, a, st); break;
  }
}

// The lists of every stream's queries.
ipv_status select_blocks(Select* s, const Counts& c, hipStream_t st) {
  SelectArgs& a = s->a;
  for (int32_t b0 = 0; b0 < c.streams; b0 += kAttendStreams) {
    const int32_t nb = std::min(kAttendStreams, c.streams - b0);
    int32_t most = 0, n = 0;
    for (int32_t i = 0; i < nb; ++i) {
      a.n[i] = c.n[b0 + i], a.first[i] = c.first[b0 + i], a.rows[i] = c.rows[b0 + i];
      most = std::max(most, a.rows[i]);
      if (a.rows[i] > 0) n = std::max(n, std::min(a.n[i], a.first[i] + a.rows[i]));
    }
    if (most == 0) continue;
    a.b0 = b0;
    a.padded = padded_blocks(n, (int32_t)a.map.R.d);
    // as many queries at a time as there is room for, and as a grid's second dimension takes
    const int64_t one = score_bytes(nb, a.H, a.padded);
    int64_t fit = one > 0 ? s->room / one : most;
    if (fit < most) fit = fit / kScoreTile * kScoreTile;
    fit = std::min<int64_t>(fit, std::max(65535 / a.H, 1) * (int64_t)kScoreTile);
    const int32_t step = (int32_t)std::min<int64_t>(std::max<int64_t>(fit, 1), most);
    for (a.m0 = 0; a.m0 < most; a.m0 += step) {
      a.mq = std::min(step, most - a.m0);
      const int32_t y = a.H * ((a.mq + kScoreTile - 1) / kScoreTile);
      // several workgroups share the blocks where tiles of queries alone leave the card empty: two a CU, if LDS takes them
      const int32_t D = s->pool->head_dim, most_wg = D <= 128 ? 512 : 256;
      const int32_t units = y * nb, x = units >= kOwnBlocks ? 1 : std::max(1, std::min(a.padded / kScoreTile, most_wg / units));
      if (select_alone((int64_t)nb * a.H * a.mq, a.mq, units, a.padded, D, 2 * D * (s->pool->format == IPV_PAGES_F32 ? 4 : 2))) {
        launch_one(s->pool, dim3((uint32_t)a.mq, (uint32_t)a.H, (uint32_t)nb), a, st);
        IPV_TRY(launched(hipGetLastError()));
        continue;
      }
      a.spread = std::max(kMaxParts / units, 1);
      const dim3 grid((uint32_t)x, (uint32_t)y, (uint32_t)nb);
      if (units >= kOwnBlocks) launch_select<false>(s->pool, grid, a, st);
      else launch_select<true>(s->pool, grid, a, st);
      IPV_TRY(launched(hipGetLastError()));
    }
  }
  return IPV_OK;
}

// What ipv_block_select and ipv_attend_blocks with bounds check of a selection, and its arguments.
ipv_status prepare_select(const ipv_page_shape* pool, const Pool& p, const BlockMap& map, const void* bounds, const Counts& c,
                          int32_t layer, const void* q, const int64_t* q_strides, int32_t q_heads, int32_t max_rows,
                          int32_t first_blocks, int32_t last_blocks, int32_t top, int32_t* blocks, void* ws, size_t ws_bytes,
                          Select* s) {
  if (!aligned(bounds, 16)) return IPV_ERR_ALIGN;
  if (first_blocks < 0 || last_blocks < 0 || (int64_t)first_blocks + last_blocks > top) return IPV_ERR_ARG;
  if (pool->kv_heads > 65535) return IPV_ERR_SHAPE;  // a grid's second dimension
  int32_t n = 0;
  for (int32_t b = 0; b < c.streams; ++b) n = std::max(n, c.n[b]);
  const int64_t least = least_scores(pool, c.streams, max_rows, n, (int32_t)map.R.d);
  IPV_TRY(check_word(ws, ws_bytes, kZeroed + (size_t)least));
  SelectArgs& a = s->a;
  a.table = p.table, a.cols = p.cols, a.pages = p.pages, a.T = p.T;
  a.map = map;
  a.bounds = static_cast<const char*>(bounds);
  a.q = static_cast<const char*>(q);
  a.q_b = q_strides[0], a.q_h = q_strides[1], a.q_m = q_strides[2];
  a.H = pool->kv_heads, a.G = q_heads / pool->kv_heads, a.layer = layer;
  a.max_rows = max_rows;
  a.first_blocks = first_blocks, a.last_blocks = last_blocks, a.top = top;
  a.scores = reinterpret_cast<double*>(static_cast<char*>(ws) + kZeroed);
  a.arrived = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + kWsHeader);
  a.blocks = blocks;
  a.err = static_cast<uint32_t*>(ws);
  s->pool = pool;
  s->room = (int64_t)(ws_bytes - kZeroed);
  return IPV_OK;
}

// Whether a query is one wave's, not a workgroup's: by the rounds that either makes on the card, in the times of a key
// tile; a round's start and end take 2.5 of them, and a wave with fewer others beside it takes less time a tile. us by
// waves and by workgroups, 64 heads of 128 in bf16, 4, 16 and 64 blocks of 64: 512 queries 14 and 10, 35 and 20, 115 and 56;
// 1024 14 and 16, 37 and 35, 120 and 105; 2048 19 and 27, 55 and 63, 200 and 210; 8192 59 and 91, 192 and 224, 698 and 744.
bool wave_a_query(int64_t queries, int32_t fill, int64_t count) {
  constexpr int SIMDS = 1024;
  const double waves = std::ceil((double)queries / SIMDS) / ((double)fill * kFewWaves / SIMDS);  // of a SIMD, of those that it can hold
  const double alone = waves <= 1 ? 2.5 + count * (0.2 + 0.8 * waves) : (double)queries / (fill * kFewWaves) * (2.5 + count);
  const double shared = std::max(1.0, (double)queries / fill) * (2.5 + std::ceil((double)count / kFewWaves));
  return alone < shared;
}

// Workgroups that the card holds at once: with fewer queries than that, lists are split.
int32_t blocks_fill(const ipv_page_shape* s, int32_t G) {
  return 256 * blocks_per_cu(s->format, s->head_dim, block_heads(s, G) / 16);
}

size_t part_bytes(const ipv_page_shape* s, int32_t G, int64_t parts) {
  return (size_t)parts * block_heads(s, G) * (size_t)(s->head_dim + 2) * sizeof(float);
}

}  // namespace

extern "C" {

ipv_status ipv_blocks_workspace_bytes(const ipv_page_shape* pool, int32_t block_rows, int32_t streams, int32_t q_heads,
                                      int32_t max_rows, int32_t top, int32_t max_tokens, size_t* bytes) {
  if (!bytes) return IPV_ERR_NULL;
  BlockMap map;
  IPV_TRY(check_pool_shape(pool));
  IPV_TRY(check_heads(pool, streams, q_heads, max_rows));
  IPV_TRY(check_lists(pool, block_rows, top, &map));
  if (max_tokens < 0 || max_tokens > kMaxPosition) return IPV_ERR_SHAPE;
  const int32_t G = q_heads / pool->kv_heads, BM = block_heads(pool, G);
  const int64_t one = score_bytes(streams, pool->kv_heads, padded_blocks(max_tokens, block_rows));
  const int64_t scores = std::max(least_scores(pool, streams, max_rows, max_tokens, block_rows), std::min(one * max_rows, kScoreBytes));
  const int64_t units = (int64_t)std::min(streams, kAttendStreams) * pool->kv_heads * max_rows * ((G + BM - 1) / BM);
  const int64_t parts = std::min<int64_t>(units * kMaxSplits, kMaxParts);
  *bytes = kZeroed + std::max((size_t)scores, part_bytes(pool, G, parts));
  return IPV_OK;
}

ipv_status ipv_block_select(const ipv_page_shape* pool, const void* bounds, int32_t block_rows, const int32_t* page_table,
                            int32_t table_cols, int32_t streams, const int32_t* n_tokens, const int32_t* q_first,
                            const int32_t* q_rows, int32_t layer, const void* q, const int64_t* q_strides, int32_t q_heads,
                            int32_t max_rows, int32_t first_blocks, int32_t last_blocks, int32_t top, int32_t* blocks,
                            void* ws, size_t ws_bytes, void* stream) {
  Pool p;
  BlockMap map;
  Select s;
  IPV_TRY(check_pool_shape(pool));
  if (!bounds || !n_tokens || !q_first || !q_rows || !q || !blocks) return IPV_ERR_NULL;
  // (the pool's rows are not read: any aligned pointer stands for them)
  IPV_TRY(check_pool(pool, bounds, bounds, static_cast<const uint8_t*>(bounds), static_cast<const uint8_t*>(bounds), page_table,
                     table_cols, streams, &p));
  IPV_TRY(check_heads(pool, streams, q_heads, max_rows));
  IPV_TRY(check_lists(pool, block_rows, top, &map));
  if (!aligned(q, 16) || !aligned(blocks, 4)) return IPV_ERR_ALIGN;
  IPV_TRY(check_strides(q_strides, 3));
  if (layer < 0 || layer >= pool->layers) return IPV_ERR_SHAPE;
  const Counts c{streams, table_cols, n_tokens, q_first, q_rows};
  IPV_TRY(check_counts(pool, c, max_rows));
  IPV_TRY(prepare_select(pool, p, map, bounds, c, layer, q, q_strides, q_heads, max_rows, first_blocks, last_blocks, top, blocks,
                         ws, ws_bytes, &s));
  return select_blocks(&s, c, static_cast<hipStream_t>(stream));
}

ipv_status ipv_attend_blocks(const ipv_page_shape* pool, const void* K_pages, const void* V_pages, const uint8_t* K_scales,
                             const uint8_t* V_scales, const void* bounds, int32_t block_rows, const int32_t* page_table,
                             int32_t table_cols, int32_t streams, const int32_t* n_tokens, const int32_t* q_first,
                             const int32_t* q_rows, int32_t layer, const void* q, const int64_t* q_strides, int32_t q_heads,
                             int32_t max_rows, double scale, int32_t first_blocks, int32_t last_blocks, int32_t top,
                             int32_t* blocks, void* out, const int64_t* out_strides, float* lse, void* ws, size_t ws_bytes,
                             void* stream) {
  BlocksArgs a;
  BlockMap map;
  IPV_TRY(check_pool(pool, K_pages, V_pages, K_scales, V_scales, page_table, table_cols, streams, &a.pool));
  if (!n_tokens || !q_first || !q_rows || !q || !out || !blocks) return IPV_ERR_NULL;
  IPV_TRY(check_heads(pool, streams, q_heads, max_rows));
  IPV_TRY(check_lists(pool, block_rows, top, &map));
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(blocks, 4) || (lse && !aligned(lse, 4))) return IPV_ERR_ALIGN;
  IPV_TRY(check_strides(q_strides, 3));
  IPV_TRY(check_strides(out_strides, 3));
  if (layer < 0 || layer >= pool->layers) return IPV_ERR_SHAPE;
  if (!(scale > 0) || !std::isfinite(scale) || !std::isnormal((float)(scale * 1.4426950408889634))) return IPV_ERR_ARG;
  const Counts c{streams, table_cols, n_tokens, q_first, q_rows};
  IPV_TRY(check_counts(pool, c, max_rows));
  const int32_t H = pool->kv_heads, G = q_heads / H, BM = block_heads(pool, G), tiles = (G + BM - 1) / BM;
  for (int32_t b0 = 0; b0 < streams; b0 += kAttendStreams) {  // every launch's queries as a grid
    int64_t units = 0;
    for (int32_t i = b0; i < std::min(streams, b0 + kAttendStreams); ++i) units += (int64_t)q_rows[i] * H * tiles;
    if ((units + 7) / 8 * 8 * (64 * kFewWaves) > kGridThreads) return IPV_ERR_SHAPE;
  }
  const int64_t units = (int64_t)std::min(streams, kAttendStreams) * H * max_rows * tiles;
  IPV_TRY(check_word(ws, ws_bytes, kZeroed + part_bytes(pool, G, std::min<int64_t>(units * kMaxSplits, kMaxParts))));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (bounds) {
    Select s;
    IPV_TRY(prepare_select(pool, a.pool, map, bounds, c, layer, q, q_strides, q_heads, max_rows, first_blocks, last_blocks, top, blocks,
                           ws, ws_bytes, &s));
    IPV_TRY(select_blocks(&s, c, st));
  }
  a.layer_row = (int64_t)layer * a.pool.layer_rows;
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.q_b = q_strides[0], a.q_h = q_strides[1], a.q_m = q_strides[2];
  a.o_b = out_strides[0], a.o_h = out_strides[1], a.o_m = out_strides[2];
  a.H = H, a.G = G;
  a.max_rows = max_rows;
  a.G_div = make_fastdiv((uint32_t)G);
  a.c = (float)(scale * 1.4426950408889634);
  a.blocks = blocks;
  a.top = top;
  a.R = map.R;
  a.halves = make_fastdiv((uint32_t)block_rows / 16u);
  a.err = static_cast<uint32_t*>(ws);
  a.arrived = reinterpret_cast<uint32_t*>(static_cast<char*>(ws) + kWsHeader);
  a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + kZeroed);
  a.tiles = tiles;
  a.by_tiles = make_fastdiv((uint32_t)tiles);
  for (int32_t b0 = 0; b0 < streams; b0 += kAttendStreams) {
    a.b0 = b0;
    a.streams = std::min(kAttendStreams, streams - b0);
    int64_t queries = 0;
    int32_t n = 0;
    for (int32_t i = 0; i < a.streams; ++i) {
      a.s[i].n = n_tokens[b0 + i], a.s[i].first = q_first[b0 + i], a.s[i].rows = q_rows[b0 + i];
      a.s[i].by_rows = make_fastdiv((uint32_t)std::max(q_rows[b0 + i], 1));
      queries += (int64_t)q_rows[b0 + i] * H * tiles;
      if (q_rows[b0 + i] > 0) n = std::max(n, std::min(a.s[i].n, a.s[i].first + a.s[i].rows));
    }
    if (queries == 0) continue;
    // lists made here hold their blocks first
    a.entries = bounds ? (int32_t)std::min<int64_t>(top, ((int64_t)n + block_rows - 1) / block_rows) : top;
    // Parts of `per` key tiles of 32 rows, the shortest that make no more workgroups than fit at once, no shorter
    // than a square root of the list: the last workgroup joins them.
    a.splits = 1;
    const int32_t fill = blocks_fill(pool, G);
    const int64_t count = ((int64_t)a.entries * a.halves.d + 1) / 2;
    if (queries < fill && count > kFewWaves) {
      int64_t per = std::max<int64_t>({(count * queries + fill - 1) / fill, kFewWaves, (int64_t)std::sqrt(0.6 * (double)count)});
      per = (per + kFewWaves - 1) / kFewWaves * kFewWaves;
      a.splits = (int32_t)std::min<int64_t>({(count + per - 1) / per, kMaxSplits, fill / queries});
    }
    a.by_splits = make_fastdiv((uint32_t)a.splits);
    int64_t at = 0;
    for (int32_t i = 0; i < a.streams; ++i) {
      a.s[i].start = (int32_t)at;
      at += (int64_t)a.s[i].rows * H * tiles * a.splits;
    }
    a.slots = (int32_t)at;
    a.part = a.part_ml + (size_t)a.slots * BM * 2;  // (a launch that splits has at most kMaxParts)
    const bool solo = a.splits == 1 && wave_a_query(queries, fill, count);
    hipError_t e;
    switch (pool->format) {
      case IPV_PAGES_BF16: e = launch_attend_blocks<kFmtBf16>(pool->head_dim, BM == 32, solo, a, st); break;
      case IPV_PAGES_F32: e = launch_attend_blocks<kFmtF32>(pool->head_dim, false, solo, a, st); break;
      case IPV_PAGES_FP8: e = launch_attend_blocks<kFmtFp8>(pool->head_dim, BM == 32, solo, a, st); break;
      default: e = launch_attend_blocks<kFmtFp4>(pool->head_dim, BM == 32, solo, a, st); break;
    }
    IPV_TRY(launched(e));
  }
  return IPV_OK;
}

}  // extern "C"
