// Attention over the blocks of a paged cache that can score highest for a query.
//
// A block's score for a query's group of heads is the sum over the heads a and the channels d of
// max(q_a[d] lo[d], q_a[d] hi[d]), lo and hi the bounds of its keys: with
// Q+[d] = sum_a max(q_a[d], 0) and Q-[d] = sum_a min(q_a[d], 0) that is Q+ . hi + Q- . lo, one product of
// 2 D terms whatever the number of heads. It is taken in 64 bits, by the vector or the matrix unit: within a call bounds of the
// same bits give scores of the same bits, and scores that differ by more than the rounding of a 64-bit sum of 2 D terms
// are ordered as they are. Closer ones may be ordered either way, and otherwise in a call of other sizes, whose sums run in
// another order.
#pragma once

#include "ipv_attend.hpp"

namespace ipv {

typedef double F64x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------ selection
// Threads of a workgroup, and waves of a SIMD at least: as many as the registers that a tile of blocks takes leave.
constexpr int select_threads(int FB, int D, bool split) { return split || (FB == kFmtF32 && D > 128) ? 256 : 512; }
constexpr int select_waves(int FB, int D, bool split) { return split || D * (FB == kFmtF32 ? 2 : 1) > 128 ? 1 : 4; }
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
  uint32_t* arrived;  // workgroups of a tile of queries that have left their scores: zero before and after a call
  int32_t spread;     // counters from one to the next: apart, since one line takes them one after the other (up to 32 tiles of
                      // queries have a line each, 127 of them 32 bytes)
  int32_t n[kAttendStreams], first[kAttendStreams], rows[kAttendStreams];
};

// Blocks that query i of stream b can pick among.
__device__ __forceinline__ int32_t candidates(const SelectArgs& a, int b, int i) {
  const int32_t held = min(a.n[b], a.first[b] + i + 1);
  return (int32_t)fast_div((uint32_t)held + a.map.R.d - 1u, a.map.R);
}

// A score as 64 bits whose order as a whole number is the scores' (-0 as +0): 0 for what cannot be picked,
// all ones for what always is, and NaN just below that.
__device__ __forceinline__ uint64_t score_key(double s, bool candidate, bool always) {
  uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
  u = (int64_t)u < 0 ? ~u : u | 1ull << 63;
  if (s != s) u = ~0ull - 1;
  return !candidate ? 0 : always ? ~0ull : u;
}

__device__ __forceinline__ uint64_t readlane64(uint64_t x, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}

__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// A wave's scores of one query. NR: a lane's, in registers (0: any number, read again each time); cross: other
// workgroups wrote some of them.
template <int NR>
struct Scores {
  double s[NR > 0 ? NR : 1];
  // block r * 64 + lane's score (past the last one's: the last)
  static __device__ __forceinline__ double at(double* scores, int32_t count, int r, bool cross) {
    double* p = scores + min(r * kWave + (int)threadIdx.x % kWave, count - 1);
    return cross ? __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT))
                 : *p;
  }
  __device__ __forceinline__ void load(double* scores, int32_t count, bool cross) {
#pragma unroll
    for (int r = 0; r < NR; ++r) s[r] = r * kWave < count ? at(scores, count, r, cross) : 0;
  }
};
__device__ __forceinline__ double* scores_of(const SelectArgs& a, int b, int h, int i) {
  return a.scores + (((int64_t)b * a.H + h) * a.mq + (i - a.m0)) * a.padded;
}
// A wave's list for query i: a histogram of 256 equal parts of the keys' range (of their upper words) says which part holds
// the k-th highest. Up to 64 keys there, a key a lane, count those above them; among more it is found bit by bit, until
// as many keys as wanted are at least the bits so far. Then the keys above it and, of those equal to it, the lowest
// blocks'. hist: 256 words of LDS.
template <int NR>
__device__ __forceinline__ void pick_blocks(const SelectArgs& a, const Scores<NR>& held, double* scores, int b, int h, int i, bool cross,
                                            uint32_t* hist) {
  const int lane = threadIdx.x % kWave;
  const int32_t count = candidates(a, b, i), want = min(a.top, count);
  int32_t* to = a.blocks + (((int64_t)(a.b0 + b) * a.H + h) * a.max_rows + i) * a.top;
  const int turns = (count + kWave - 1) / kWave;
  const auto key_of = [&](int r, double s) __attribute__((always_inline)) {
    const int j = r * kWave + lane;
    return score_key(s, j < count, (j < a.first_blocks) | (j >= count - a.last_blocks));
  };
  constexpr int N = NR > 0 ? NR : 1;
  uint64_t key[N];
  if constexpr (NR > 0) {
#pragma unroll
    for (int r = 0; r < NR; ++r) key[r] = key_of(r, held.s[r]);
  }
  const auto each = [&](auto&& what) __attribute__((always_inline)) {
    if constexpr (NR > 0) {
#pragma unroll
      for (int r = 0; r < NR; ++r) what(r, key[r]);
    } else {
      constexpr int AHEAD = 8;  // on their way at once (past the last ones: keys of 0)
      for (int r0 = 0; r0 < turns; r0 += AHEAD) {
        double s[AHEAD];
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) s[r] = Scores<NR>::at(scores, count, r0 + r, cross);
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) what(r0 + r, key_of(r0 + r, s[r]));
      }
    }
  };
  const auto at_least = [&](uint64_t x) __attribute__((always_inline)) {
    int c = 0;
    each([&](int, uint64_t y) __attribute__((always_inline)) { c += __builtin_popcountll(__ballot(y >= x)); });
    return c;
  };
  const auto upper_at_least = [&](uint32_t x) __attribute__((always_inline)) {
    int c = 0;
    each([&](int, uint64_t y) __attribute__((always_inline)) { c += __builtin_popcountll(__ballot((uint32_t)(y >> 32) >= x)); });
    return c;
  };
  uint64_t limit = 1;  // the least key that is picked
  int equal = 0;       // of those equal to it, as many (all, if `all`)
  bool all = true, found = false;
  const int forced = a.first_blocks + a.last_blocks;  // (of which there are as many where there are more blocks than wanted)
  if (want < count && want == forced) {
    limit = ~0ull;
  } else if (want < count) {
    // the range of the others' upper words, from `from` on
    uint32_t least, most;
    const auto range = [&](uint32_t from, uint32_t size) __attribute__((always_inline)) {
      least = ~0u, most = 0;
      each([&](int, uint64_t y) __attribute__((always_inline)) {
        const uint32_t u = (uint32_t)(y >> 32);
        const bool in = (y != 0) & (y != ~0ull) & (u - from <= size);
        least = in ? min(least, u) : least, most = in ? max(most, u) : most;
      });
      wave_min_max(least, most);
    };
    range(0, ~0u);
    all = false;
    limit = (uint64_t)least << 32;
    if (least < most) {
      const int shift = max(24 - __builtin_clz(most - least), 0);
      U32x4* bins = reinterpret_cast<U32x4*>(hist);
      bins[lane] = U32x4{0, 0, 0, 0};
      asm volatile("" ::: "memory");
      each([&](int, uint64_t y) __attribute__((always_inline)) {
        if ((y != 0) & (y != ~0ull)) atomicAdd(&hist[((uint32_t)(y >> 32) - least) >> shift], 1u);
      });
      asm volatile("" ::: "memory");
      // lane 0 has the four highest parts: keys of them and of all before
      const U32x4 c = bins[kWave - 1 - lane];
      const int32_t sum = (int32_t)(c[0] + c[1] + c[2] + c[3]), upto = wave_inclusive_scan(sum), rest = want - forced;
      const int32_t before = upto - sum, a3 = before + (int32_t)c[3], a2 = a3 + (int32_t)c[2], a1 = a2 + (int32_t)c[1];
      const int part = a3 >= rest ? 3 : a2 >= rest ? 2 : a1 >= rest ? 1 : 0;
      const int32_t above = part == 3 ? before : part == 2 ? a3 : part == 1 ? a2 : a1;  // keys above that part, and with it
      const int32_t reached = part == 3 ? a3 : part == 2 ? a2 : part == 1 ? a1 : upto;
      const int at = __builtin_ctzll(__ballot(upto >= rest));
      const uint32_t from = least + ((uint32_t)((kWave - 1 - at) * 4 + __builtin_amdgcn_readlane(part, at)) << shift);
      all = __builtin_amdgcn_readlane(reached, at) == rest;
      limit = (uint64_t)from << 32;
      const int32_t over = __builtin_amdgcn_readlane(above, at), inside = __builtin_amdgcn_readlane(reached, at) - over, need = rest - over;
      if (!all && inside <= kWave) {
        uint64_t* few = reinterpret_cast<uint64_t*>(hist);
        int put = 0;
        each([&](int, uint64_t y) __attribute__((always_inline)) {
          const bool in = (y != 0) & (y != ~0ull) & (((uint32_t)(y >> 32) - from) >> shift == 0);
          const uint64_t mask = __ballot(in);
          if (in) few[put + lanes_below(mask)] = y;
          put += __builtin_popcountll(mask);
        });
        asm volatile("" ::: "memory");
        const uint64_t mine = lane < inside ? few[lane] : 0;
        int higher = 0, no_less = 0;
        for (int x = 0; x < inside; ++x) {
          const uint64_t y = readlane64(mine, x);
          higher += y > mine, no_less += y >= mine;
        }
        const int it = __builtin_ctzll(__ballot((lane < inside) & (higher < need) & (no_less >= need)));
        limit = readlane64(mine, it);
        equal = need - __builtin_amdgcn_readlane(higher, it);
        all = __builtin_amdgcn_readlane(no_less, it) == need;
        found = true;
      } else if (!all && shift > 0) {
        range(from, (1u << shift) - 1u);
        const int top_bit = least < most ? 31 - __builtin_clz(least ^ most) : -1;
        uint32_t upper = top_bit < 0 ? least : least >> top_bit >> 1 << top_bit << 1;
        for (int bit = top_bit; bit >= 0 && !all; --bit) {
          const uint32_t x = upper | 1u << bit;
          const int n = upper_at_least(x);
          if (n >= want) upper = x;
          all = n == want;
        }
        limit = (uint64_t)upper << 32;
      }
    }
    for (int bit = 31; bit >= 0 && !all && !found; --bit) {
      const uint64_t x = limit | 1ull << bit;
      const int n = at_least(x);
      if (n >= want) limit = x;
      all = n == want;
    }
    if (!all && !found) equal = want - at_least(limit + 1);
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

// Q+ and Q- of four channels: sums over the group's heads, the first one's elements at `at`.
template <int FB>
__device__ __forceinline__ void group_queries(const SelectArgs& a, int64_t at, double (&plus)[4], double (&minus)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) plus[e] = minus[e] = 0;
  constexpr int HEADS = 8;  // on their way at once
  for (int g0 = 0; g0 < a.G; g0 += HEADS) {
    float f[HEADS][4];
#pragma unroll
    for (int g = 0; g < HEADS; ++g) {
      const int64_t from = at + min(g0 + g, a.G - 1) * a.q_h;
      if constexpr (FB == kFmtF32) {
        Lane<float>::decode(load16(a.q + from * 4), f[g]);
      } else {
        const U32x2 w = *reinterpret_cast<const U32x2*>(a.q + from * 2);
        f[g][0] = __uint_as_float(w.x << 16), f[g][1] = __uint_as_float(w.x & 0xffff0000u);
        f[g][2] = __uint_as_float(w.y << 16), f[g][3] = __uint_as_float(w.y & 0xffff0000u);
      }
    }
#pragma unroll
    for (int g = 0; g < HEADS; ++g) {
      if (g0 + g >= a.G) break;
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // (a NaN reaches both)
        plus[e] += (double)(f[g][e] < 0.f ? 0.f : f[g][e]);
        minus[e] += (double)(f[g][e] > 0.f ? 0.f : f[g][e]);
      }
    }
  }
}

// A term of a score where the product form came out as NaN: 0 times an infinity counts as 0, as on a side to which no query adds
// against that side's infinite bound (a group's sum is 0 only if each of its parts is). Such scores, and no others, are made
// again so after the loops over the blocks; a NaN bound or query stays one. Bounds that are finite pay the comparison (1024 tokens
// over 512 blocks 61.4 and 61.8 us, 256 over 256 of heads of 32 16.9 and 18.1); with a NaN in every block or query those 1024 take
// 0.4 ms (made again a score at a time by a whole wave: 4.2).
__device__ __forceinline__ double score_term(double q, float bound) {
  const double p = q * (double)bound;
  return p != p && q == q && bound == bound ? 0.0 : p;
}

// The list of one query of a head. blockIdx.x: query; .y: head; .z: stream. Eight lanes have a block's bounds, eight blocks
// a wave at a time, and add up their products in the vector unit: the matrix unit would take 16 queries' time for one.
// Scores stay in LDS, and no workgroup waits for another. For few queries over up to 64 NR blocks. 512 threads where each has
// a CU of its own, else 256, of which a CU holds more: one token of 16 streams of four heads over 512 blocks of 128 15 us
// by trace (and 19; 12.3 in a captured run of calls), of 196 tokens over 98 16 (and 22): the way to the bounds, and the
// products (64 bits a channel).
template <int FB, int D, int NR, int THREADS>
__global__ __launch_bounds__(THREADS) void k_block_select_one(SelectArgs a) {
  constexpr int E = FB == kFmtF32 ? 4 : 2, PER = 16 / E, PIECES = 2 * D / 8 / PER;  // bytes of an element; elements of 16 bytes; of these, a lane's
  constexpr bool HELD = D <= 128;  // the lane's part of the queries in registers
  constexpr int WAVES = THREADS / kWave, AHEAD = PIECES <= 4 ? 4 : PIECES <= 8 ? 2 : 1;  // eights of blocks on their way
  __shared__ __attribute__((aligned(16))) double lds_q[2 * D];
  __shared__ double lds_scores[NR * kWave];
  __shared__ __attribute__((aligned(16))) uint32_t hist[256];
  const int b = blockIdx.z, h = blockIdx.y, i = a.m0 + (int)blockIdx.x;
  if (i >= min(a.m0 + a.mq, a.rows[b])) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t count = candidates(a, b, i);
  const int own = lane / 8, part = lane % 8;
  bool bad = false;
  struct Piece {
    Raw16 r[PIECES];
  };
  // the page of the lane's block, and its part of the bounds there (blocks past the last: the last one again)
  const auto page_of = [&](int j0) __attribute__((always_inline)) {
    const uint32_t p = (uint32_t)min(j0 + own, count - 1) * a.map.R.d;
    return a.table ? a.table[(int64_t)(a.b0 + b) * a.cols + fast_div(p, a.T)] : a.b0 + b;
  };
  const auto bounds_of = [&](int j0, int32_t page) __attribute__((always_inline)) {
    const uint32_t p = (uint32_t)min(j0 + own, count - 1) * a.map.R.d;
    if ((uint32_t)page >= (uint32_t)a.pages) page = 0, bad = true;
    return a.bounds + a.map.block(page, (uint32_t)(a.layer * a.H + h), p, a.T) * (2 * D * E) + part * 16;
  };
  const auto load_block = [&](int j0, int32_t page) __attribute__((always_inline)) {
    const char* at = bounds_of(j0, page);
    Piece x;
#pragma unroll
    for (int c = 0; c < PIECES; ++c) x.r[c] = load16(at + c * 128);
    return x;
  };
  Piece ahead[AHEAD] = {};
  int j0 = wave * 8;
  constexpr int STEP = WAVES * 8;
  int32_t page = 0;  // of the blocks after those on their way
  if (j0 < count) {
    int32_t pages[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) pages[u] = page_of(j0 + u * STEP);
    page = page_of(j0 + AHEAD * STEP);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (j0 + u * STEP < count) ahead[u] = load_block(j0 + u * STEP, pages[u]);
  }
  if (threadIdx.x < D / 4) {
    const int channel = threadIdx.x * 4;
    double plus[4], minus[4];
    group_queries<FB>(a, (int64_t)(a.b0 + b) * a.q_b + (int64_t)h * a.G * a.q_h + (int64_t)i * a.q_m + channel, plus, minus);
#pragma unroll
    for (int e = 0; e < 4; ++e) lds_q[channel + e] = minus[e], lds_q[D + channel + e] = plus[e];
  }
  __syncthreads();
  const auto query = [&](int c, int e) __attribute__((always_inline)) { return lds_q[(c * 8 + part) * PER + e]; };
  double q[HELD ? PIECES : 1][HELD ? PER : 1];
  if constexpr (HELD) {
#pragma unroll
    for (int c = 0; c < PIECES; ++c)
#pragma unroll
      for (int e = 0; e < PER; ++e) q[c][e] = query(c, e);
  }
  bool odd = false;  // a score of NaN
  for (; j0 < count; j0 += STEP) {
    const Piece x = ahead[0];
#pragma unroll
    for (int u = 0; u + 1 < AHEAD; ++u) ahead[u] = ahead[u + 1];
    if (j0 + AHEAD * STEP < count) {
      ahead[AHEAD - 1] = load_block(j0 + AHEAD * STEP, page);
      page = page_of(j0 + (AHEAD + 1) * STEP);
    }
    double s = 0, s1 = 0;
#pragma unroll
    for (int c = 0; c < PIECES; ++c) {
      float f[PER];
      if constexpr (FB == kFmtF32) Lane<float>::decode(x.r[c], f);
      else Lane<uint16_t>::decode(x.r[c], f);
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const double v = HELD ? q[HELD ? c : 0][HELD ? e : 0] : query(c, e);
        if (e % 2) s1 = __builtin_fma((double)f[e], v, s1);
        else s = __builtin_fma((double)f[e], v, s);
      }
    }
    s = group_sum64<8>(s + s1);
    odd |= s != s;
    if (part == 0 && j0 + own < count) lds_scores[j0 + own] = s;
  }
  if (__ballot(odd) != 0) {  // the wave's blocks once more
    for (int j1 = wave * 8; j1 < count; j1 += STEP) {
      const char* at = bounds_of(j1, page_of(j1));
      double s = 0;
#pragma unroll 1
      for (int c = 0; c < PIECES; ++c) {
        float f[PER];
        Lane<std::conditional_t<FB == kFmtF32, float, uint16_t>>::decode(load16(at + c * 128), f);
#pragma unroll
        for (int e = 0; e < PER; ++e) s += score_term(query(c, e), f[e]);
      }
      s = group_sum64<8>(s);
      if (part == 0 && j1 + own < count && lds_scores[j1 + own] != lds_scores[j1 + own]) lds_scores[j1 + own] = s;
    }
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, kDevBadPage);
  __syncthreads();
  if (wave != 0) return;
  Scores<NR> scores;
  scores.load(lds_scores, count, false);
  pick_blocks<NR>(a, scores, lds_scores, b, h, i, false, hist);
}

// Where channel ch (of 2 D) of query col is: step 8 (ch / 32) + ch % 8, place ch / 8 % 4, and the queries of a place in an
// order by which the channels that a wave writes together lie in different banks.
__device__ __forceinline__ int select_place(int ch, int col) {
  const int c = ch / 32, k = ch / 8 % 4;
  return (c * 8 + ch % 8) * kWave + k * kScoreTile + (col ^ (k * 4 + c % 4));
}

// The lists of up to 16 queries of a head. blockIdx.x: tiles of 16 blocks, in turn; .y: head and tile of queries; .z:
// stream. Q+ and Q- of the queries are made in LDS in the order in which the product takes them: step 8 c + e has channel
// 8 (4 c + k) + e in its place k, so that a lane's 16 bytes of bounds are operands of eight steps. A wave takes a tile
// of blocks or, where there are few queries (SPLIT), a quarter of its steps, added up through LDS: then the way through
// all of them is what a tile costs. The scores go to memory; the workgroup, the last one to come where several share the
// blocks, picks from them. Bound by the 64-bit products where there are many queries (1024 tokens of 8 KV heads over 512
// blocks: 62 us in a captured run of such calls, 63 to 76 by trace, 33 of them the products at the rate of a large one; the matrix
// unit is busy for 48% of the cycles); for one by the trips to table, bounds, scores, counter and scores again (9, and 10 to 13).
template <int FB, int D, int NR, bool SPLIT>
__global__ __launch_bounds__(select_threads(FB, D, SPLIT), select_waves(FB, D, SPLIT)) void k_block_select(SelectArgs a) {
  constexpr int THREADS = select_threads(FB, D, SPLIT), SELECT_WAVES = THREADS / kWave;
  constexpr int STEPS = D / 2, PART = SPLIT ? STEPS / SELECT_WAVES : STEPS;  // of four terms; of a wave
  constexpr int CHUNKS = PART < 8 ? 1 : PART / 8;                            // of eight steps, that a wave loads
  constexpr int WAVES = SPLIT ? 1 : SELECT_WAVES;                            // tiles at a time
  __shared__ double lds[STEPS * kWave];
  __shared__ double sums[SPLIT ? 2 : 1][SPLIT ? SELECT_WAVES : 1][kScoreTile * kScoreTile];
  __shared__ bool lds_last;
  const int b = blockIdx.z, q_tiles = (a.mq + kScoreTile - 1) / kScoreTile;
  const int h = blockIdx.y / q_tiles, i0 = a.m0 + blockIdx.y % q_tiles * kScoreTile;
  const int i1 = min(min(i0 + kScoreTile, a.m0 + a.mq), a.rows[b]);
  if (i0 >= i1) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int row = lane % kScoreTile, k = lane / kScoreTile;
  const int32_t most = candidates(a, b, i1 - 1), tiles = (most + kScoreTile - 1) / kScoreTile;
  const int sharing = max(min((int)gridDim.x, tiles), 1);
  if ((int)blockIdx.x >= sharing) return;  // the whole workgroup
  const int c0 = SPLIT ? wave * PART / 8 : 0, e0 = SPLIT ? wave * PART % 8 : 0;  // the wave's first chunk and step there
  bool bad = false;
  // the page of the lane's block of a tile (a tile past the last: the last block); its bounds, in the wave's channels
  const auto page_of = [&](int tile) __attribute__((always_inline)) {
    const uint32_t p = (uint32_t)min(tile * kScoreTile + row, most - 1) * a.map.R.d;
    return a.table ? a.table[(int64_t)(a.b0 + b) * a.cols + fast_div(p, a.T)] : a.b0 + b;
  };
  struct Piece {
    Raw16 r[CHUNKS * (FB == kFmtF32 ? 2 : 1)];
  };
  const auto load_tile = [&](int tile, int32_t page) __attribute__((always_inline)) {
    const uint32_t p = (uint32_t)min(tile * kScoreTile + row, most - 1) * a.map.R.d;
    if ((uint32_t)page >= (uint32_t)a.pages) page = 0, bad = true;
    constexpr int E = FB == kFmtF32 ? 4 : 2;
    const char* at = a.bounds + a.map.block(page, (uint32_t)(a.layer * a.H + h), p, a.T) * (2 * D * E) + (c0 * 4 + k) * 8 * E;
    Piece x;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int i = 0; i < E / 2; ++i) x.r[c * (E / 2) + i] = load16(at + c * 32 * E + 16 * i);
    return x;
  };
  const int first = (int)blockIdx.x * WAVES + (SPLIT ? 0 : wave), step = (int)gridDim.x * WAVES;
  Piece next = {};
  int32_t page = 0;  // of the tile after the next
  if (first < tiles) {
    next = load_tile(first, page_of(first));
    page = page_of(first + step);
  }
  // four channels of a query a thread (of the queries that there are: what is in the other columns reaches no score of these)
  for (int x = threadIdx.x; x < (i1 - i0) * (D / 4); x += THREADS) {
    const int col = x / (D / 4), channel = x % (D / 4) * 4;
    double plus[4], minus[4];
    group_queries<FB>(a, (int64_t)(a.b0 + b) * a.q_b + (int64_t)h * a.G * a.q_h + (int64_t)(i0 + col) * a.q_m + channel, plus, minus);
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // the bounds' first D channels are the lowest elements
      lds[select_place(channel + e, col)] = minus[e];
      lds[select_place(D + channel + e, col)] = plus[e];
    }
  }
  __syncthreads();
  // the wave's operands of the queries' side in registers, where those suffice for the waves that a CU can have then
  constexpr bool HELD = SPLIT && PART <= 64;
  double q[HELD ? PART : 1];
  const auto operand = [&](int i) __attribute__((always_inline)) {
    const int step = (SPLIT ? wave * PART : 0) + i;
    return lds[select_place(step / 8 * 32 + k * 8 + step % 8, row)];
  };
  if constexpr (HELD)
#pragma unroll
    for (int i = 0; i < PART; ++i) q[i] = operand(i);
  bool odd = false;  // a score of NaN
  const auto put = [&](double* to, double v) __attribute__((always_inline)) {
    if (sharing > 1)
      __hip_atomic_store(reinterpret_cast<uint64_t*>(to), __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    else *to = v;
  };
  int buf = 0;
  for (int tile = first; tile < tiles; tile += step, buf ^= 1) {
    const Piece x = next;
    if (tile + step < tiles) {
      next = load_tile(tile + step, page);
      page = page_of(tile + 2 * step);
    }
    float f[CHUNKS][8];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      if constexpr (FB == kFmtF32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[c][i] = __uint_as_float(x.r[2 * c].w[i]), f[c][4 + i] = __uint_as_float(x.r[2 * c + 1].w[i]);
      } else {
        Lane<uint16_t>::decode(x.r[c], f[c]);
      }
    }
    F64x4 s = {}, s1 = {};
#pragma unroll
    for (int i = 0; i < PART; ++i) {
      float v = f[i / 8][i % 8];
      if constexpr (PART < 8) v = e0 ? f[0][4 + i] : f[0][i];
      F64x4& sum = i % 2 ? s1 : s;  // (two, since each waits for its last product)
      sum = __builtin_amdgcn_mfma_f64_16x16x4f64((double)v, HELD ? q[HELD ? i : 0] : operand(i), sum, 0, 0, 0);
    }
    s += s1;
    // a lane has the scores, or their parts, of its query (lane % 16) and of the tile's blocks 4 e + lane / 16
    const auto keep = [&](int col, int i, double v) __attribute__((always_inline)) {
      if (i0 + col >= i1) return;
      odd |= v != v;
      put(scores_of(a, b, h, i0 + col) + tile * kScoreTile + i, v);
    };
    if constexpr (SPLIT) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sums[buf][wave][e * kWave + lane] = s[e];
      __syncthreads();
      double total = 0;
#pragma unroll
      for (int w = 0; w < SELECT_WAVES; ++w) total += sums[buf][w][threadIdx.x];
      keep(threadIdx.x % kScoreTile, threadIdx.x / kScoreTile, total);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) keep(row, 4 * e + k, s[e]);
    }
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, kDevBadPage);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this thread's scores are written
  if (__ballot(odd) != 0) {  // the wave's own once more
    for (int tile = first; tile < tiles; tile += step)
      for (int e = 0; e < (SPLIT ? 1 : 4); ++e) {
        const int x = SPLIT ? (int)threadIdx.x : e * kWave + lane, col = x % kScoreTile, j = tile * kScoreTile + x / kScoreTile;
        double* to = scores_of(a, b, h, min(i0 + col, i1 - 1)) + j;
        uint64_t v = 0;
        if (i0 + col < i1 && j < most) v = __hip_atomic_load(reinterpret_cast<uint64_t*>(to), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const double was = __builtin_bit_cast(double, v);
        if (__ballot(was != was) == 0) continue;
        const uint32_t p = (uint32_t)min(j, most - 1) * a.map.R.d;
        int32_t there = a.table ? a.table[(int64_t)(a.b0 + b) * a.cols + fast_div(p, a.T)] : a.b0 + b;
        if ((uint32_t)there >= (uint32_t)a.pages) there = 0;
        const int64_t at = a.map.block(there, (uint32_t)(a.layer * a.H + h), p, a.T) * (2 * D);
        double s = 0;
#pragma unroll 1
        for (int ch = 0; ch < 2 * D; ch += 8) {
          float f[8];
          load_row8<FB>(a.bounds, at + ch, f);
#pragma unroll
          for (int i = 0; i < 8; ++i) s += score_term(lds[select_place(ch + i, col)], f[i]);
        }
        if (was != was) put(to, s);
      }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  __syncthreads();
  if (sharing > 1) {
    if (threadIdx.x == 0) {
      uint32_t* count = a.arrived + (blockIdx.z * gridDim.y + blockIdx.y) * a.spread;
      const uint32_t before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      lds_last = before + 1 == (uint32_t)sharing;
      if (lds_last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!lds_last) return;
  }
  static_assert(sizeof(lds) >= SELECT_WAVES * 256 * sizeof(uint32_t), "a histogram a wave");
  uint32_t* hist = reinterpret_cast<uint32_t*>(lds) + wave * 256;
  constexpr bool NEXT = NR <= 8;  // the next query's scores on their way meanwhile: more would leave room for fewer waves
  Scores<NR> later;
  if (NEXT && i0 + wave < i1) later.load(scores_of(a, b, h, i0 + wave), candidates(a, b, i0 + wave), sharing > 1);
  for (int i = i0 + wave; i < i1; i += SELECT_WAVES) {
    if (!NEXT) later.load(scores_of(a, b, h, i), candidates(a, b, i), sharing > 1);
    const Scores<NR> scores = later;
    const int then = i + SELECT_WAVES;
    if (NEXT && then < i1) later.load(scores_of(a, b, h, then), candidates(a, b, then), sharing > 1);
    pick_blocks<NR>(a, scores, scores_of(a, b, h, i), b, h, i, sharing > 1, hist);
  }
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

// The query and part of a workgroup, or (SOLO) of a wave: tokens of a head follow each other on an XCD, since
// their lists are often alike.
struct BlockPlace : Place {
  int32_t token;
};
template <bool SOLO>
__device__ __forceinline__ BlockPlace block_place(const BlocksArgs& a, int wave) {
  constexpr uint32_t EACH = SOLO ? kFewWaves : 1;  // places of a workgroup
  const uint32_t per = ((uint32_t)a.slots + 8u * EACH - 1u) / (8u * EACH);
  BlockPlace p;
  p.slot = (int32_t)(((blockIdx.x % 8u) * per + blockIdx.x / 8u) * EACH + (SOLO ? wave : 0));
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
  __device__ __forceinline__ int64_t row_at(int lane_) const { return (int64_t)readlane64((uint64_t)row, lane_); }
  __device__ __forceinline__ int32_t seen_at(int lane_) const { return __builtin_amdgcn_readlane(seen, lane_); }
};

// Workgroups of a CU, by the registers and the LDS that they take.
constexpr int blocks_per_cu(int F, int D, int NB) {
  if (F == kFmtF32) return D <= 64 ? 3 : D <= 128 ? 2 : 1;
  return NB * D <= 64 || (fmt_scaled(F) && NB * D <= 128) ? 3 : NB * D <= 128 || (fmt_scaled(F) && D <= 128) ? 2 : 1;
}

// As k_attend_few, but that the keys are those of a list, and all rows of the workgroup are one token's: a
// row of the cache is seen by all of them or by none.
template <int F, int D, int NB, bool SOLO>
__global__ __launch_bounds__(64 * kFewWaves, blocks_per_cu(F, D, NB)) void k_attend_blocks(BlocksArgs a) {
  using C = FewCfg<F, D>;
  constexpr size_t KTILE = kFewKeys * C::RB, VTILE = kFewKeys * D * 2, JOIN = JoinLds<D, 16 * NB>::kWaveBytes;
  __shared__ __attribute__((aligned(16))) char lds[kFewWaves][SOLO || JOIN < KTILE + VTILE ? KTILE + VTILE : JOIN];
  const int lane = threadIdx.x % kWave, g = lane / 16, l16 = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const BlockPlace pl = block_place<SOLO>(a, wave);
  if (pl.slot < 0) return;  // the whole workgroup, or a wave that no other waits for
  const int b = a.b0 + pl.b;
  const int64_t head_row = a.layer_row + (int64_t)pl.h * a.pool.T.d;
  const int32_t held = min(a.s[pl.b].n, a.s[pl.b].first + pl.token + 1);
  const int32_t* list = a.blocks + (((int64_t)b * a.H + pl.h) * a.max_rows + pl.token) * a.top;
  const int32_t count = (int32_t)(((int64_t)a.entries * a.halves.d + 1) / 2);  // key tiles of the list
  const int32_t t_end = (int32_t)((int64_t)count * (pl.split + 1) / a.splits);
  const int32_t t_begin = (int32_t)((int64_t)count * pl.split / a.splits) + (SOLO ? 0 : wave);
  constexpr int STEP = SOLO ? 1 : kFewWaves;
  const int heads = min(a.G - pl.tile * 16 * NB, 16 * NB);

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

  // A tile's rows as they are stored, on their way from when they are fetched until they are used: keys as well as values
  // in the order of memory and through LDS. Keys straight into the product's operand, where neighbouring lanes have
  // different rows, cost the cache a line for each lane: 1024 tokens of 64 heads with 16 blocks of 64 of
  // 32768 positions of 128 take 304 us so and 222 through LDS.
  // (Keys lie there as they are stored, values as bf16.)
  struct Rows {
    uint32_t k[C::NV][4], v[C::NV][4];
    uint64_t ks[2], vs[C::NV];  // scales of the operand's keys, and of the values' pieces
    int32_t seen0, seen1;
  };
  char* k_tile = lds[wave];
  char* v_tile = lds[wave] + KTILE;
  // places of 16-byte chunks of a key's row: those that 16 rows' lanes read together lie in different banks
  const auto k_swz = [](int row) __attribute__((always_inline)) {
    return C::CPR >= 8 ? row & 7 : C::CPR == 4 ? (row >> 1) & 3 : C::CPR == 2 ? (row >> 2) & 1 : 0;
  };
  bool bad = false;
  const auto fetch = [&](Rows& x, const Runs& runs, int at) __attribute__((always_inline)) {
    const int64_t r0 = runs.row_at(at), r1 = runs.row_at(at + 1);
    x.seen0 = runs.seen_at(at), x.seen1 = runs.seen_at(at + 1);
    constexpr int PER = kWave / C::CPR;  // rows a load
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      if constexpr (PER <= 16) {
        const int64_t row = i * PER < 16 ? r0 + i * PER : r1 + (i * PER - 16);
        load_piece<16>(a.pool.K + row * C::RB + (uint32_t)(lane * 16), x.k[i]);
        load_piece<16>(a.pool.V + row * C::RB + (uint32_t)(lane * 16), x.v[i]);
        if (fmt_scaled(F)) x.vs[i] = load_scales<D>(a.pool.Vs + row * (D / kScaleBlock), lane / C::CPR);
      } else {
        const int key = lane / C::CPR % kFewKeys;  // (a piece too many is the first ones' again)
        const int64_t row = (key < 16 ? r0 : r1) + key % 16;
        load_piece<16>(a.pool.K + row * C::RB + lane % C::CPR * 16, x.k[i]);
        load_piece<16>(a.pool.V + row * C::RB + lane % C::CPR * 16, x.v[i]);
        if (fmt_scaled(F)) x.vs[i] = load_scales<D>(a.pool.Vs, row);
      }
    }
    if (fmt_scaled(F)) x.ks[0] = load_scales<D>(a.pool.Ks, r0 + l16), x.ks[1] = load_scales<D>(a.pool.Ks, r1 + l16);
  };
  // a tile's scores, weights and sums; `next` sets out the rows of the next one when these are in LDS
  const auto use = [&](Rows& x, auto&& next) __attribute__((always_inline)) {
    const int32_t seen0 = x.seen0, seen1 = x.seen1;
    const bool full = (seen0 == 16) & (seen1 == 16);
    if (!full) {  // values of rows that are not seen as zeros
#pragma unroll
      for (int i = 0; i < C::NV; ++i) {
        const int key = (i * kWave + lane) / C::CPR % kFewKeys;
        if (key % 16 < (key < 16 ? seen0 : seen1)) continue;
        x.v[i][0] = x.v[i][1] = x.v[i][2] = x.v[i][3] = 0;
        x.vs[i] = 0;
      }
    }
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      const int y = i * kWave + lane, key = y / C::CPR, col = y % C::CPR;
      if (C::CPR == 1 && y >= kFewKeys) continue;
      *reinterpret_cast<Raw16*>(k_tile + key * C::RB + 16 * (col ^ k_swz(key))) = Raw16{x.k[i][0], x.k[i][1], x.k[i][2], x.k[i][3]};
      const float scale = fmt_scaled(F) ? scale_at(x.vs[i], col * C::VE / kScaleBlock) : 0.f;
#pragma unroll
      for (int e = 0; e < C::VE / 8; ++e)
        *reinterpret_cast<Raw16*>(v_tile + key * (D * 2) + 16 * ((col * (C::VE / 8) + e) ^ C::swz(key))) = piece8<F>(x.v[i], e, scale);
    }
    __builtin_amdgcn_wave_barrier();
    const uint64_t ks[2] = {x.ks[0], x.ks[1]};
    const bool more = next(x);
    F32x4 sc[NB][2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) sc[nb][kb] = F32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < C::KN; ++c) {
        const int byte = (c * 4 + g) * C::KB;
        uint32_t kr[4];
        load_piece<C::KB>(k_tile + (kb * 16 + l16) * C::RB + 16 * ((byte / 16) ^ k_swz(l16)) + byte % 16, kr);
#pragma unroll
        for (int s = 0; s < C::KE / 8; ++s) {
          const float scale = fmt_scaled(F) ? scale_at(ks[kb], ((c * 4 + g) * C::KE + 8 * s) / kScaleBlock) : 0.f;
          const Bf16x8 k = __builtin_bit_cast(Bf16x8, piece8<F>(kr, s, scale));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            sc[nb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[nb][c * (C::KE / 8) + s], sc[nb][kb], 0, 0, 0);
        }
      }
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
      const U32x2 v0 = lds_column4(v_tile + k0 * (D * 2) + 16 * (ch ^ C::swz(k0)) + in);
      const U32x2 v1 = lds_column4(v_tile + (k0 + 16) * (D * 2) + 16 * (ch ^ C::swz(k0 + 16)) + in);
      const Raw16 r = {v0.x, v0.y, v1.x, v1.y};
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf16x8, r), w[nb], o[nb][db], 0, 0, 0);
    }
    __builtin_amdgcn_wave_barrier();
    return more;
  };
  for (int32_t t0 = t_begin; t0 < t_end; t0 += 32 * STEP) {
    Runs runs;
    runs.look_up(a, list, b, head_row, held, t0, STEP, t_end, bad);
    uint64_t todo = runs.some;
    // the next tile's rows set out (if there is one)
    const auto next = [&](Rows& x) __attribute__((always_inline)) {
      if (todo == 0) return false;
      const int at = __builtin_ctzll(todo);
      todo &= todo - 1;
      fetch(x, runs, at);
      return true;
    };
    Rows x;
    bool more = next(x);
    while (more) more = use(x, next);
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, kDevBadPage);

  if constexpr (SOLO) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float sum = lanes_sum<4>(l[nb]);
      const int r = nb * 16 + l16;
      if (r >= heads) continue;
#pragma unroll
      for (int db = 0; db < D / 16; ++db)
        row_out<D, false>(a, b, pl.h, pl.token * a.G + pl.tile * 16 * NB + r, 16 * db + 4 * g, o[nb][db], m[nb], sum);
    }
    return;
  }
  // join the waves: each scales its sums to the largest maximum
  __shared__ float lds_ml[kFewWaves][16 * NB][2];
  __shared__ uint32_t lds_last;
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
  if constexpr (!SOLO) join_parts<D, 16 * NB, false>(a, st, pl, b, pl.token * a.G + pl.tile * 16 * NB, heads, lds, lds_ml, &lds_last);
}

// fp32 pools: as k_attend_blocks, up to 16 query heads of a token, with the fp32 matrix instruction. Keys go through LDS as
// there; values straight into the product's operand, where 16 lanes have a key's 64 (32) channels: it is its channels
// that a lane has four of side by side, so that sum 4 j + e has channels 64 j + 4 r + e in its rows r. Tiles of 16 rows, since
// a token has few: 512 tokens of 64 heads of 128 over 16 blocks of 64 take 383 us (90 TFLOP/s of half filled tiles), with the
// 32-row instruction and keys straight into its operand 724; one token of four streams over 2048 rows 20 and 23. Bound by
// the matrix instruction, single tokens by the way to the rows.
template <int D, bool SOLO>
__global__ __launch_bounds__(64 * kFewWaves, blocks_per_cu(kFmtF32, D, 1)) void k_attend_blocks_f32(BlocksArgs a) {
  constexpr size_t RB = D * 4, KTILE = kFewKeys * RB, JOIN = JoinLds<D, 16>::kWaveBytes;
  constexpr int NP = (int)(KTILE / 1024), RP = 1024 / RB;  // loads of a tile's keys; rows of one
  constexpr int VE = D >= 64 ? 4 : 1, VN = D / 16 / VE;    // channels side by side; of these, a lane's of a key
  constexpr int SUMS = D <= 32 ? 1 : D <= 64 ? 2 : 4;      // of a score: with one, heads of 256 are off by 1.4e-6 of their norm, so by 5.4e-7
  __shared__ __attribute__((aligned(16))) char lds[kFewWaves][SOLO || JOIN < KTILE ? KTILE : JOIN];
  const int lane = threadIdx.x % kWave, g = lane / 16, l16 = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const BlockPlace pl = block_place<SOLO>(a, wave);
  if (pl.slot < 0) return;  // the whole workgroup, or a wave that no other waits for
  const int b = a.b0 + pl.b;
  const int64_t head_row = a.layer_row + (int64_t)pl.h * a.pool.T.d;
  const int32_t held = min(a.s[pl.b].n, a.s[pl.b].first + pl.token + 1);
  const int32_t* list = a.blocks + (((int64_t)b * a.H + pl.h) * a.max_rows + pl.token) * a.top;
  const int32_t count = (int32_t)(((int64_t)a.entries * a.halves.d + 1) / 2);  // key tiles of the list
  const int32_t t_end = (int32_t)((int64_t)count * (pl.split + 1) / a.splits);
  const int32_t t_begin = (int32_t)((int64_t)count * pl.split / a.splits) + (SOLO ? 0 : wave);
  constexpr int STEP = SOLO ? 1 : kFewWaves;
  const int heads = min(a.G - pl.tile * 16, 16);

  F32x4 q[D / 16];
  const char* qa = a.q + 4 * ((int64_t)b * a.q_b + (int64_t)(pl.h * a.G + pl.tile * 16 + min(l16, heads - 1)) * a.q_h +
                              (int64_t)pl.token * a.q_m + 4 * g);
#pragma unroll
  for (int c = 0; c < D / 16; ++c) q[c] = *reinterpret_cast<const F32x4*>(qa + 64 * c);
  F32x4 o[D / 16];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) o[i] = F32x4{0.f, 0.f, 0.f, 0.f};

  typedef float Channels __attribute__((ext_vector_type(VE)));
  struct Rows {
    F32x4 k[NP];
    Channels v[8][VN];  // of keys 4 g + i and 16 + 4 g + i
    int32_t seen0, seen1;
  };
  char* tile = lds[wave];
  const auto swz = [](int row) __attribute__((always_inline)) { return row & 7; };  // rows that lanes read together: other banks
  bool bad = false;
  const auto fetch_k = [&](Rows& x, int64_t r0, int64_t r1) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int64_t row = i * RP < 16 ? r0 + i * RP : r1 + (i * RP - 16);
      x.k[i] = *reinterpret_cast<const F32x4*>(a.pool.K + row * (int64_t)RB + (uint32_t)(lane * 16));
    }
  };
  const auto fetch_v = [&](Rows& x, int64_t r0, int64_t r1) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const char* at = a.pool.V + (i < 4 ? r0 + i : r1 + (i - 4)) * (int64_t)RB + (uint32_t)(4 * g * (int)RB + l16 * VE * 4);
#pragma unroll
      for (int j = 0; j < VN; ++j) x.v[i][j] = *reinterpret_cast<const Channels*>(at + j * 64 * VE);
    }
  };
  // a tile's scores, weights and sums; the next one's rows set out as soon as their places are free
  const auto use = [&](Rows& x, bool more, int64_t n0, int64_t n1) __attribute__((always_inline)) {
    const int32_t seen0 = x.seen0, seen1 = x.seen1;
    const bool full = (seen0 == 16) & (seen1 == 16);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int y = i * kWave + lane, key = y / (D / 4), col = y % (D / 4);
      *reinterpret_cast<F32x4*>(tile + key * (int)RB + 16 * (col ^ swz(key))) = x.k[i];
    }
    __builtin_amdgcn_wave_barrier();
    if (more) fetch_k(x, n0, n1);
    F32x4 sc[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      F32x4 sums[SUMS];
#pragma unroll
      for (int i = 0; i < SUMS; ++i) sums[i] = F32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        const F32x4 k = *reinterpret_cast<const F32x4*>(tile + (kb * 16 + l16) * (int)RB + 16 * ((c * 4 + g) ^ swz(l16)));
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[i % SUMS] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i], q[c][i], sums[i % SUMS], 0, 0, 0);
      }
      sc[kb] = sums[0];
      if constexpr (SUMS == 2) sc[kb] += sums[1];
      if constexpr (SUMS == 4) sc[kb] = (sc[kb] + sums[1]) + (sums[2] + sums[3]);
    }
    __builtin_amdgcn_wave_barrier();
    if (!full) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (4 * g + i >= seen0) sc[0][i] = -INFINITY;
        if (4 * g + i >= seen1) sc[1][i] = -INFINITY;
#pragma unroll
        for (int j = 0; j < VN; ++j) {  // values of rows that are not seen as zeros
          if (4 * g + i >= seen0) x.v[i][j] = (Channels)(0.f);
          if (4 * g + i >= seen1) x.v[4 + i][j] = (Channels)(0.f);
        }
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(fmaxf(top, sc[0][i]), sc[1][i]);
    top = lanes_max<4>(top) * a.c;
    if (__ballot(top > m) != 0) {
      rare();
      top = fmaxf(top, m);
      const float old = exp2_hw(m - shift_of(top));
      m = top;
      l *= old;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[i] *= old;
    }
    const float shift = shift_of(m);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float e = exp2_hw(__builtin_fmaf(sc[i / 4][i % 4], a.c, -shift));
      l += e;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) {
        float v;
        if constexpr (VE == 1) v = x.v[i][db][0];
        else v = x.v[i][db / VE][db % VE];
        o[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, e, o[db], 0, 0, 0);
      }
    }
    if (more) fetch_v(x, n0, n1);
  };
  // what a lane has of the result: four channels from `d` on
  const auto each_part = [&](auto&& what) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      if constexpr (VE == 1) what(16 * x + 4 * g, o[x]);
      else what(64 * (x / 4) + 16 * g + 4 * (x % 4),
                F32x4{o[x / 4 * 4][x % 4], o[x / 4 * 4 + 1][x % 4], o[x / 4 * 4 + 2][x % 4], o[x / 4 * 4 + 3][x % 4]});
    }
  };
  for (int32_t t0 = t_begin; t0 < t_end; t0 += 32 * STEP) {
    Runs runs;
    runs.look_up(a, list, b, head_row, held, t0, STEP, t_end, bad);
    uint64_t todo = runs.some;
    if (todo == 0) continue;
    Rows x;
    int at = __builtin_ctzll(todo);
    fetch_k(x, runs.row_at(at), runs.row_at(at + 1));
    fetch_v(x, runs.row_at(at), runs.row_at(at + 1));
    while (todo != 0) {
      x.seen0 = runs.seen_at(at), x.seen1 = runs.seen_at(at + 1);
      todo &= todo - 1;
      at = todo != 0 ? __builtin_ctzll(todo) : 0;
      use(x, todo != 0, runs.row_at(at), runs.row_at(at + 1));
    }
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, kDevBadPage);

  l = lanes_sum<4>(l);
  if constexpr (SOLO) {
    if (l16 < heads)
      each_part([&](int d, const F32x4& v) __attribute__((always_inline)) {
        row_out<D, true>(a, b, pl.h, pl.token * a.G + pl.tile * 16 + l16, d, v, m, l);
      });
    return;
  }
  __shared__ float lds_ml[kFewWaves][16][2];
  __shared__ uint32_t lds_last;
  if (lane < 16) lds_ml[wave][lane][0] = m, lds_ml[wave][lane][1] = l;
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, lds_ml[w][l16][0]);
  const float f = exp2_hw(m - shift_of(top));
  float* mine = reinterpret_cast<float*>(lds[wave]) + l16 * JoinLds<D, 16>::STRIDE;
  each_part([&](int d, const F32x4& v) __attribute__((always_inline)) { *reinterpret_cast<F32x4*>(mine + d) = v * f; });
  __syncthreads();
  AttendStream st;
  st.splits = a.splits;
  if constexpr (!SOLO) join_parts<D, 16, true>(a, st, pl, b, pl.token * a.G + pl.tile * 16, heads, lds, lds_ml, &lds_last);
}

// What a format's translation unit offers.
template <int F>
hipError_t launch_attend_blocks(int D, bool wide, bool solo, const BlocksArgs& a, hipStream_t st);

}  // namespace ipv
