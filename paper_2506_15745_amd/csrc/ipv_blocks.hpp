// Attention over the blocks of a paged cache that can score highest for a query.
//
// A block's score for a query's group of heads is the sum over the heads a and the channels d of
// max(q_a[d] lo[d], q_a[d] hi[d]), lo and hi the bounds of its keys: with
// Q+[d] = sum_a max(q_a[d], 0) and Q-[d] = sum_a min(q_a[d], 0) that is Q+ . hi + Q- . lo, one product of
// 2 D terms whatever the number of heads. It is taken in 64 bits by the matrix unit: equal bounds give
// equal scores, and no rounding decides between blocks that differ.
#pragma once

#include "ipv_attend.hpp"

namespace ipv {

typedef double F64x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------ scores
constexpr int kSelectThreads = 256;
constexpr int kScoreTile = 16;  // queries, and blocks, of a product

struct SelectArgs {
  const int32_t* table;
  int32_t cols, pages;
  FastDiv T;
  BlockMap map;
  const char* bounds;
  const char* q;
  int64_t q_b, q_h, q_m;
  int32_t b0, H, G, layer;
  int32_t max_rows, m0, mq;  // queries of a stream in all; the first one of this launch, and how many
  int32_t first_blocks, last_blocks, top;
  int32_t padded;  // blocks from one query's scores to the next's
  double* scores;  // [stream][head][query of the launch][padded]
  int32_t* blocks;
  uint32_t* err;
  int32_t n[kAttendStreams], first[kAttendStreams], rows[kAttendStreams];
};

// Blocks that query i of stream b can pick among.
__device__ __forceinline__ int32_t candidates(const SelectArgs& a, int b, int i) {
  const int32_t held = min(a.n[b], a.first[b] + i + 1);
  return (int32_t)fast_div((uint32_t)held + a.map.R.d - 1u, a.map.R);
}

// blockIdx.x: tiles of blocks, a wave each in turn; .y: head and tile of queries; .z: stream. Q+ and Q- of
// the tile's queries are made in LDS in the order in which the product takes them: step 8 c + e has channel
// 8 (4 c + k) + e in its place k, so that a lane's 16 bytes of bounds are operands of eight steps.
template <int FB, int D>
__global__ __launch_bounds__(kSelectThreads) void k_block_scores(SelectArgs a) {
  constexpr int STEPS = D / 2, CHUNKS = D / 16;  // of four terms; of eight steps
  __shared__ double lds[STEPS * kWave];
  const int b = blockIdx.z, q_tiles = (a.mq + kScoreTile - 1) / kScoreTile;
  const int h = blockIdx.y / q_tiles, i0 = a.m0 + blockIdx.y % q_tiles * kScoreTile;
  const int i1 = min(min(i0 + kScoreTile, a.m0 + a.mq), a.rows[b]);
  if (i0 >= i1) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int32_t most = candidates(a, b, i1 - 1), tiles = (most + kScoreTile - 1) / kScoreTile;
  if ((int)blockIdx.x * (kSelectThreads / kWave) >= tiles) return;  // the whole workgroup
  for (int x = threadIdx.x; x < kScoreTile * (D / 8); x += kSelectThreads) {
    const int col = x % kScoreTile, piece = x / kScoreTile;
    const int64_t at = (int64_t)(a.b0 + b) * a.q_b + (int64_t)h * a.G * a.q_h + (int64_t)min(i0 + col, i1 - 1) * a.q_m + piece * 8;
    double plus[8], minus[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) plus[e] = minus[e] = 0;
    for (int g = 0; g < a.G; ++g) {
      float f[8];
      load_row8<FB>(a.q, at + g * a.q_h, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {  // (a NaN reaches both)
        plus[e] += (double)(f[e] < 0.f ? 0.f : f[e]);
        minus[e] += (double)(f[e] > 0.f ? 0.f : f[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {  // the bounds' first D channels are the lowest elements
      lds[((piece / 4 * 8 + e) * 4 + piece % 4) * kScoreTile + col] = minus[e];
      lds[(((piece + D / 8) / 4 * 8 + e) * 4 + (piece + D / 8) % 4) * kScoreTile + col] = plus[e];
    }
  }
  __syncthreads();
  const int row = lane % kScoreTile, k = lane / kScoreTile;
  bool bad = false;
  for (int tile = blockIdx.x * (kSelectThreads / kWave) + wave; tile < tiles; tile += gridDim.x * (kSelectThreads / kWave)) {
    const uint32_t j = (uint32_t)min(tile * kScoreTile + row, most - 1), p = j * a.map.R.d;
    int32_t page = a.table ? a.table[(int64_t)(a.b0 + b) * a.cols + fast_div(p, a.T)] : a.b0 + b;
    if ((uint32_t)page >= (uint32_t)a.pages) page = 0, bad = true;
    const char* at = a.bounds + a.map.block(page, (uint32_t)(a.layer * a.H + h), p, a.T) * (2 * D * (FB == kFmtF32 ? 4 : 2));
    F64x4 s[2] = {};
    float f[CHUNKS][8];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) load_row8<FB>(at, (c * 4 + k) * 8, f[c]);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        s[e % 2] = __builtin_amdgcn_mfma_f64_16x16x4f64((double)f[c][e], lds[(c * 8 + e) * kWave + lane], s[e % 2], 0, 0, 0);
    // a lane has the scores of its query (lane % 16) and of the tile's blocks 4 e + lane / 16
    const int i = i0 + row;
    if (i >= i1) continue;
    double* to = a.scores + (((int64_t)b * a.H + h) * a.mq + (i - a.m0)) * a.padded + tile * kScoreTile + k;
#pragma unroll
    for (int e = 0; e < 4; ++e) to[4 * e] = s[0][e] + s[1][e];
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, kDevBadPage);
}

// ------------------------------------------------------------ the highest scores
// A score as 64 bits whose order as a whole number is the scores' (-0 as +0): 0 for what cannot be picked,
// all ones for what always is, and NaN just below that.
__device__ __forceinline__ uint64_t score_key(double s, bool candidate, bool always) {
  uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
  u = (int64_t)u < 0 ? ~u : u | 1ull << 63;
  if (s != s) u = ~0ull - 1;
  return !candidate ? 0 : always ? ~0ull : u;
}

__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// A wave a query: the k-th highest key bit by bit, its upper half first, until as many keys as wanted are
// at least the bits so far; then the keys above it and, of those equal to it, the lowest blocks'. NR: a lane's
// keys, in registers (0: any number, read again for every bit).
template <int NR>
__global__ __launch_bounds__(kSelectThreads) void k_block_pick(SelectArgs a) {
  const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x % kWave;
  const int i = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kSelectThreads / kWave) + threadIdx.x / kWave)) + a.m0;
  if (i >= min(a.m0 + a.mq, a.rows[b])) return;
  const int32_t count = candidates(a, b, i), want = min(a.top, count);
  const double* scores = a.scores + (((int64_t)b * a.H + h) * a.mq + (i - a.m0)) * a.padded;
  int32_t* to = a.blocks + (((int64_t)(a.b0 + b) * a.H + h) * a.max_rows + i) * a.top;
  const int turns = (count + kWave - 1) / kWave;
  const auto load_key = [&](int r) __attribute__((always_inline)) {
    const int j = r * kWave + lane;
    const double s = scores[min(j, count - 1)];
    return score_key(s, j < count, (j < a.first_blocks) | (j >= count - a.last_blocks));
  };
  constexpr int N = NR > 0 ? NR : 1;
  uint64_t key[N];
  if constexpr (NR > 0) {
#pragma unroll
    for (int r = 0; r < NR; ++r) key[r] = r < turns ? load_key(r) : 0;
  }
  const auto each = [&](auto&& what) __attribute__((always_inline)) {
    if constexpr (NR > 0) {
#pragma unroll
      for (int r = 0; r < NR; ++r) what(r, key[r]);
    } else {
      for (int r = 0; r < turns; ++r) what(r, load_key(r));
    }
  };
  const auto at_least = [&](uint64_t x) __attribute__((always_inline)) {
    int c = 0;
    each([&](int, uint64_t y) __attribute__((always_inline)) { c += __builtin_popcountll(__ballot(y >= x)); });
    return c;
  };
  uint64_t limit = 1;  // the least key that is picked
  int equal = 0;       // of those equal to it, as many (all, if `all`)
  bool all = true;
  if (want < count) {
    limit = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t x = limit | 1ull << bit;
      const int c = at_least(x);
      if (c < want) continue;
      limit = x;
      if (c == want) break;
    }
    const int above = limit == ~0ull ? 0 : at_least(limit + 1);
    all = at_least(limit) == want;
    equal = want - above;
  }
  int pos = 0;
  each([&](int r, uint64_t y) __attribute__((always_inline)) {
    bool in = y >= limit && y != 0;
    if (!all) {
      const uint64_t same = __ballot(y == limit);
      in = in && (y != limit || lanes_below(same) < equal);
      equal = max(equal - __builtin_popcountll(same), 0);
    }
    const uint64_t mask = __ballot(in);
    if (in) to[pos + lanes_below(mask)] = r * kWave + lane;
    pos += __builtin_popcountll(mask);
  });
  for (int x = pos + lane; x < a.top; x += kWave) to[x] = -1;
}

// ------------------------------------------------------------ attention over lists
struct BlockStream {
  int32_t n, first, rows;
  int32_t start;  // its first workgroup
  FastDiv by_rows;
};

struct BlocksArgs {
  static constexpr bool kApart = false;  // parts are joined by the last workgroup to come
  Pool pool;
  int64_t layer_row;
  const char* q;
  char* out;
  float* lse;
  int64_t q_b, q_h, q_m, o_b, o_h, o_m;  // strides, elements
  int32_t b0, H, G, max_rows;
  FastDiv G_div;
  float c;  // scale * log2(e)
  const int32_t* blocks;
  int32_t top, entries;  // of a query's list; of those, how many can hold blocks
  FastDiv R, halves;     // rows of a block; runs of 16 of them
  float* part;
  float* part_ml;
  uint32_t* err;
  uint32_t* arrived;
  int32_t streams, slots;
  int32_t tiles, splits;  // tiles of a KV head's query heads; parts of a list
  FastDiv by_tiles, by_splits;
  BlockStream s[kAttendStreams];
};

// A workgroup's query and part: tokens of a head follow each other on an XCD, since their lists are often alike.
struct BlockPlace : Place {
  int32_t token;
};
__device__ __forceinline__ BlockPlace block_place(const BlocksArgs& a) {
  const uint32_t per = (uint32_t)(a.slots + 7) / 8u;
  BlockPlace p;
  p.slot = (int32_t)((blockIdx.x % 8u) * per + blockIdx.x / 8u);
  p.b = 0;
  if (p.slot >= a.slots) {
    p.slot = -1;
    return p;
  }
  int lo = 0, hi = a.streams - 1;  // the last stream that starts at or before the slot
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.s[mid].start <= p.slot) lo = mid;
    else hi = mid - 1;
  }
  p.b = lo;
  const BlockStream& s = a.s[lo];
  const uint32_t x = (uint32_t)(p.slot - s.start), y = fast_div(x, a.by_splits), z = fast_div(y, a.by_tiles);
  p.split = (int32_t)(x - y * (uint32_t)a.splits);
  p.first = p.slot - p.split;
  p.tile = (int32_t)(y - z * (uint32_t)a.tiles);
  p.h = (int32_t)fast_div(z, s.by_rows);
  p.token = (int32_t)(z - (uint32_t)p.h * (uint32_t)s.rows);
  return p;
}

// The rows of a wave's next 32 key tiles, two runs of 16 rows each, a run a lane: looked up at once, so
// that a tile's rows wait for no list and no table.
struct Runs {
  int64_t row;   // of the pool (of page 0 where the run has no row that is seen)
  int32_t seen;  // of its rows
  uint64_t some; // by even lane: tiles that have a row that is seen
  __device__ __forceinline__ void look_up(const BlocksArgs& a, const int32_t* list, int b, int64_t head_row, int32_t held, int32_t t,
                                          int32_t step, int32_t t_end, bool& bad) {
    const int lane = threadIdx.x % kWave;
    t += lane / 2 * step;
    const uint32_t x = 2u * (uint32_t)t + (lane & 1), e = fast_div(x, a.halves);
    const int32_t block = t < t_end && e < (uint32_t)a.entries ? list[e] : -1;
    const int32_t count = (int32_t)fast_div((uint32_t)held + a.R.d - 1u, a.R);
    const bool in = (uint32_t)block < (uint32_t)count;
    const int32_t p = in ? block * (int32_t)a.R.d + (int32_t)(x - e * a.halves.d) * 16 : held;
    seen = min(max(held - p, 0), 16);
    row = 0;
    if (seen > 0) {
      bool none;
      row = pool_row(a.pool, pool_page(a.pool, b, (uint32_t)p), (uint32_t)p, &none) + head_row;
      bad |= none;
    }
    const uint64_t m = __ballot(seen > 0);
    some = (m | m >> 1) & 0x5555555555555555ull;
  }
  __device__ __forceinline__ int64_t row_at(int lane_) const {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)row, lane_);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)row >> 32), lane_);
    return (int64_t)((uint64_t)hi << 32 | lo);
  }
  __device__ __forceinline__ int32_t seen_at(int lane_) const { return __builtin_amdgcn_readlane(seen, lane_); }
};

// As k_attend_few, but that the keys are those of a list, and all rows of the workgroup are one token's: a
// row of the cache is seen by all of them or by none.
template <int F, int D, int NB>
__global__ __launch_bounds__(64 * kFewWaves, few_per_cu(F, D, NB)) void k_attend_blocks(BlocksArgs a) {
  using C = FewCfg<F, D>;
  __shared__ __attribute__((aligned(16))) char lds[kFewWaves][few_wave_lds<F, D, NB>()];
  __shared__ float lds_ml[kFewWaves][16 * NB][2];
  __shared__ uint32_t lds_last;
  const BlockPlace pl = block_place(a);
  if (pl.slot < 0) return;  // the whole workgroup
  const int lane = threadIdx.x % kWave, g = lane / 16, l16 = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int b = a.b0 + pl.b;
  const int64_t head_row = a.layer_row + (int64_t)pl.h * a.pool.T.d;
  const int32_t held = min(a.s[pl.b].n, a.s[pl.b].first + pl.token + 1);
  const int32_t* list = a.blocks + (((int64_t)b * a.H + pl.h) * a.max_rows + pl.token) * a.top;
  const int32_t count = (int32_t)(((int64_t)a.entries * a.halves.d + 1) / 2);  // key tiles of the list
  const int32_t t_end = (int32_t)((int64_t)count * (pl.split + 1) / a.splits);
  const int32_t t_begin = (int32_t)((int64_t)count * pl.split / a.splits) + wave;
  const int heads = min(a.G - pl.tile * 16 * NB, 16 * NB);  // of the workgroup

  F32x4 o[NB][D / 16];
  float m[NB], l[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = -INFINITY, l[nb] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[nb][i] = F32x4{0.f, 0.f, 0.f, 0.f};
  }
  Bf16x8 q[NB][D / 32];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int head = pl.h * a.G + pl.tile * 16 * NB + min(nb * 16 + l16, heads - 1);
    const char* at = a.q + 2 * ((int64_t)b * a.q_b + (int64_t)head * a.q_h + (int64_t)pl.token * a.q_m);
#pragma unroll
    for (int c = 0; c < C::KN; ++c)
#pragma unroll
      for (int s = 0; s < C::KE / 8; ++s)
        q[nb][c * (C::KE / 8) + s] = __builtin_bit_cast(Bf16x8, load16(at + 2 * ((c * 4 + g) * C::KE + 8 * s)));
  }

  constexpr bool COPY = F == kFmtBf16;
  constexpr int VTILE = kFewKeys * D * 2;
  uint32_t kr[2][C::KQ / 4], vr[COPY ? 1 : C::NV][4];
  uint64_t ks[2], vs[COPY ? 1 : C::NV];
  char* tile = lds[wave];
  int vbuf = 0;
  bool bad = false;
  // the rows of both runs set out
  const auto fetch = [&](int64_t r0, int64_t r1, char* v_tile) __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int64_t row = kb ? r1 : r0;
      const char* p = a.pool.K + row * C::RB;
#pragma unroll
      for (int c = 0; c < C::KN; ++c)
        load_piece<C::KB>(p + c * 4 * C::KB + (uint32_t)(l16 * C::RB + g * C::KB), kr[kb] + c * (C::KB / 4));
      if (fmt_scaled(F)) ks[kb] = load_scales<D>(a.pool.Ks + row * (D / kScaleBlock), l16);
    }
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      const int key = (i * kWave + lane) / C::CPR % kFewKeys;  // (a piece too many is the first ones' again)
      constexpr int PER = kWave / C::CPR;                      // rows a load
      if constexpr (COPY) {
        const char* p = a.pool.V + (i * PER < 16 ? r0 + i * PER : r1 + (i * PER - 16)) * C::RB;
        const int ch = lane % C::CPR ^ C::swz(key);  // the source column makes up for the place
        copy_to_lds(p, (uint32_t)(lane / C::CPR * C::RB + ch * 16), __builtin_amdgcn_readfirstlane(lds_address(v_tile) + i * 1024));
      } else if constexpr (PER <= 16) {
        const int64_t row = i * PER < 16 ? r0 + i * PER : r1 + (i * PER - 16);
        load_piece<16>(a.pool.V + row * C::RB + (uint32_t)(lane / C::CPR * C::RB + lane % C::CPR * 16), vr[i]);
        if (fmt_scaled(F)) vs[i] = load_scales<D>(a.pool.Vs + row * (D / kScaleBlock), lane / C::CPR);
      } else {
        const int64_t row = (key < 16 ? r0 : r1) + key % 16;
        load_piece<16>(a.pool.V + row * C::RB + lane % C::CPR * 16, vr[i]);
        if (fmt_scaled(F)) vs[i] = load_scales<D>(a.pool.Vs, row);
      }
    }
  };
  for (int32_t t0 = t_begin; t0 < t_end; t0 += 32 * kFewWaves) {
    Runs runs;
    runs.look_up(a, list, b, head_row, held, t0, kFewWaves, t_end, bad);
    uint64_t todo = runs.some;
    if (todo == 0) continue;
    int at = __builtin_ctzll(todo);
    fetch(runs.row_at(at), runs.row_at(at + 1), tile + vbuf * VTILE);
    while (todo != 0) {
      todo &= todo - 1;
      if constexpr (COPY) copies_done();
      const int32_t seen0 = runs.seen_at(at), seen1 = runs.seen_at(at + 1);
      const bool full = (seen0 == 16) & (seen1 == 16);
      F32x4 sc[NB][2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) sc[nb][kb] = F32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C::KN; ++c)
#pragma unroll
          for (int s = 0; s < C::KE / 8; ++s) {
            const float scale = fmt_scaled(F) ? scale_at(ks[kb], ((c * 4 + g) * C::KE + 8 * s) / kScaleBlock) : 0.f;
            const Bf16x8 k = __builtin_bit_cast(Bf16x8, piece8<F>(kr[kb] + c * (C::KB / 4), s, scale));
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
              sc[nb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[nb][c * (C::KE / 8) + s], sc[nb][kb], 0, 0, 0);
          }
      }
      // V into LDS as bf16, rows that are not seen as zeros
      if (!full) {
#pragma unroll
        for (int i = 0; i < C::NV; ++i) {
          const int x = i * kWave + lane, key = x / C::CPR % kFewKeys;
          if (key % 16 < (key < 16 ? seen0 : seen1)) continue;
          if constexpr (COPY) {
            *reinterpret_cast<Raw16*>(tile + vbuf * VTILE + x * 16) = Raw16{0, 0, 0, 0};  // as this lane copied it
          } else {
            vr[i][0] = vr[i][1] = vr[i][2] = vr[i][3] = 0;
            vs[i] = 0;
          }
        }
      }
      if constexpr (!COPY)
#pragma unroll
        for (int i = 0; i < C::NV; ++i) {
          const int x = i * kWave + lane, key = x / C::CPR, col = x % C::CPR;
          if (C::CPR == 1 && x >= kFewKeys) continue;
          const float scale = scale_at(vs[i], col * C::VE / kScaleBlock);
#pragma unroll
          for (int e = 0; e < C::VE / 8; ++e)
            *reinterpret_cast<Raw16*>(tile + key * (D * 2) + 16 * ((col * (C::VE / 8) + e) ^ C::swz(key))) = piece8<F>(vr[i], e, scale);
        }
      if (todo != 0) {
        at = __builtin_ctzll(todo);
        fetch(runs.row_at(at), runs.row_at(at + 1), tile + (COPY ? (vbuf ^ 1) * VTILE : 0));
      }
      Bf16x8 w[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if (!full) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (4 * g + i >= seen0) sc[nb][0][i] = -INFINITY;
            if (4 * g + i >= seen1) sc[nb][1][i] = -INFINITY;
          }
        }
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(fmaxf(top, sc[nb][0][i]), sc[nb][1][i]);
        top = lanes_max<4>(top) * a.c;
        if (__ballot(top > m[nb]) != 0) {
          rare();
          top = fmaxf(top, m[nb]);
          const float old = exp2_hw(m[nb] - shift_of(top));
          m[nb] = top;
          l[nb] *= old;
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            if constexpr (NB * D > 256) in_acc(o[nb][i]);
            o[nb][i] *= old;
            if constexpr (NB * D > 256) in_acc(o[nb][i]);
          }
        }
        const float shift = shift_of(m[nb]);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float e = exp2_hw(__builtin_fmaf(sc[nb][kb][i], a.c, -shift));
            l[nb] += e;
            w[nb][kb * 4 + i] = (__bf16)e;
          }
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int db = 0; db < D / 16; ++db) {
        const int k0 = 4 * g + l16 / 4, ch = 2 * db + (l16 % 4) / 2, in = 8 * (l16 & 1);
        const char* from = tile + (COPY ? vbuf * VTILE : 0);
        const U32x2 x = lds_column4(from + k0 * (D * 2) + 16 * (ch ^ C::swz(k0)) + in);
        const U32x2 y = lds_column4(from + (k0 + 16) * (D * 2) + 16 * (ch ^ C::swz(k0 + 16)) + in);
        const Raw16 r = {x.x, x.y, y.x, y.y};
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
          o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf16x8, r), w[nb], o[nb][db], 0, 0, 0);
      }
      __builtin_amdgcn_wave_barrier();
      if (COPY) vbuf ^= 1;
    }
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, kDevBadPage);

  // join the waves: each scales its sums to the largest maximum
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    l[nb] = lanes_sum<4>(l[nb]);
    if (lane < 16) lds_ml[wave][nb * 16 + lane][0] = m[nb], lds_ml[wave][nb * 16 + lane][1] = l[nb];
  }
  __syncthreads();
  constexpr int STRIDE = JoinLds<D, 16 * NB>::STRIDE;
  float* mine = reinterpret_cast<float*>(lds[wave]);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, lds_ml[w][nb * 16 + l16][0]);
    const float f = exp2_hw(m[nb] - shift_of(top));
#pragma unroll
    for (int db = 0; db < D / 16; ++db)
      *reinterpret_cast<F32x4*>(mine + (nb * 16 + l16) * STRIDE + 16 * db + 4 * g) = o[nb][db] * f;
  }
  __syncthreads();
  AttendStream st;
  st.splits = a.splits;
  join_parts<D, 16 * NB, false>(a, st, pl, b, pl.token * a.G + pl.tile * 16 * NB, heads, lds, lds_ml, &lds_last);
}

// As k_attend_f32: fp32 pools, up to 32 query heads of a token.
template <int D>
__global__ __launch_bounds__(64 * kFewWaves, D <= 64 ? 2 : 1) void k_attend_blocks_f32(BlocksArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[kFewWaves][JoinLds<D, 32>::kWaveBytes];
  __shared__ float lds_ml[kFewWaves][32][2];
  __shared__ uint32_t lds_last;
  const BlockPlace pl = block_place(a);
  if (pl.slot < 0) return;
  const int lane = threadIdx.x % kWave, h = lane / 32, l32 = lane % 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int b = a.b0 + pl.b;
  const int64_t head_row = a.layer_row + (int64_t)pl.h * a.pool.T.d;
  const int32_t held = min(a.s[pl.b].n, a.s[pl.b].first + pl.token + 1);
  const int32_t* list = a.blocks + (((int64_t)b * a.H + pl.h) * a.max_rows + pl.token) * a.top;
  const int32_t count = (int32_t)(((int64_t)a.entries * a.halves.d + 1) / 2);
  const int32_t t_end = (int32_t)((int64_t)count * (pl.split + 1) / a.splits);
  const int32_t t_begin = (int32_t)((int64_t)count * pl.split / a.splits) + wave;
  const int heads = min(a.G - pl.tile * 32, 32);
  float q[D / 2];
  const char* qa = a.q + 4 * ((int64_t)b * a.q_b + (int64_t)(pl.h * a.G + pl.tile * 32 + min(l32, heads - 1)) * a.q_h +
                              (int64_t)pl.token * a.q_m + 4 * h);
#pragma unroll
  for (int k = 0; k < D / 2; k += 4) {
    const F32x4 v = *reinterpret_cast<const F32x4*>(qa + 8 * k);
    q[k] = v.x, q[k + 1] = v.y, q[k + 2] = v.z, q[k + 3] = v.w;
  }
  F32x16 o[D / 32];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = F32x16{};
  bool bad = false;
  constexpr int KA = D <= 128 ? D / 8 : 8;  // pieces of a K row in registers
  F32x4 kx[KA];
  constexpr int VA = D <= 128 ? 16 : 4;  // keys of V
  float vx[VA][D / 32];
  for (int32_t t0 = t_begin; t0 < t_end; t0 += 32 * kFewWaves) {
    Runs runs;
    runs.look_up(a, list, b, head_row, held, t0, kFewWaves, t_end, bad);
    for (uint64_t todo = runs.some; todo != 0; todo &= todo - 1) {
      const int at = __builtin_ctzll(todo);
      const int64_t r0 = runs.row_at(at), r1 = runs.row_at(at + 1);
      const int32_t seen0 = runs.seen_at(at), seen1 = runs.seen_at(at + 1);
      const bool full = (seen0 == 16) & (seen1 == 16);
      const float* kp = reinterpret_cast<const float*>(a.pool.K) + ((l32 < 16 ? r0 : r1) + l32 % 16) * D + 4 * h;
      const auto load_k = [&](int k) __attribute__((always_inline)) { kx[k % KA] = *reinterpret_cast<const F32x4*>(kp + 8 * k); };
      const auto load_v = [&](int i) __attribute__((always_inline)) {
        const int key = 8 * (i / 4) + i % 4;  // (+ 4 h)
        const float* p = reinterpret_cast<const float*>(a.pool.V) + (i < 8 ? r0 + key : r1 + (key - 16)) * D;
#pragma unroll
        for (int db = 0; db < D / 32; ++db) vx[i % VA][db] = p[32 * db + (uint32_t)(4 * h * D + l32)];
      };
#pragma unroll
      for (int k = 0; k < KA; ++k) load_k(k);
#pragma unroll
      for (int i = 0; i < VA; ++i) load_v(i);
      F32x16 s = {};
#pragma unroll
      for (int k = 0; k < D / 8; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kx[k % KA][i], q[4 * k + i], s, 0, 0, 0);
        if (k + KA < D / 8) load_k(k + KA);
      }
      if (!full) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if ((8 * (i / 4) + i % 4) % 16 + 4 * h >= (i < 8 ? seen0 : seen1)) s[i] = -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[i]);
      top = lanes_max<2>(top) * a.c;
      if (__ballot(top > m + kLazy) != 0) {
        rare();
        top = fmaxf(top, m);
        const float old = exp2_hw(m - shift_of(top));
        m = top;
        l *= old;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          if constexpr (D > 64) in_acc(o[i]);
          o[i] *= old;
          if constexpr (D > 64) in_acc(o[i]);
        }
      }
      const float shift = shift_of(m);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = exp2_hw(__builtin_fmaf(s[i], a.c, -shift));
        l += e;
        float(&v)[D / 32] = vx[i % VA];
        if (!full) {
          const bool some = (8 * (i / 4) + i % 4) % 16 + 4 * h < (i < 8 ? seen0 : seen1);
#pragma unroll
          for (int db = 0; db < D / 32; ++db)
            if (!some) v[db] = 0.f;
        }
#pragma unroll
        for (int db = 0; db < D / 32; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[db], e, o[db], 0, 0, 0);
        if (i + VA < 16) load_v(i + VA);
      }
    }
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, kDevBadPage);

  l = lanes_sum<2>(l);
  if (h == 0) lds_ml[wave][l32][0] = m, lds_ml[wave][l32][1] = l;
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, lds_ml[w][l32][0]);
  const float f = exp2_hw(m - shift_of(top));
  float* mine = reinterpret_cast<float*>(lds[wave]) + l32 * JoinLds<D, 32>::STRIDE;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<F32x4*>(mine + 32 * db + 8 * i + 4 * h) =
          F32x4{o[db][4 * i] * f, o[db][4 * i + 1] * f, o[db][4 * i + 2] * f, o[db][4 * i + 3] * f};
  __syncthreads();
  AttendStream st;
  st.splits = a.splits;
  join_parts<D, 32, true>(a, st, pl, b, pl.token * a.G + pl.tile * 32, heads, lds, lds_ml, &lds_last);
}

// What a format's translation unit offers.
template <int F>
hipError_t launch_attend_blocks(int D, bool wide, uint32_t grid, const BlocksArgs& a, hipStream_t st);

}  // namespace ipv
