// Attention of new tokens over a paged cache.
//
// For a query q at position p, x_j = scale * (q . K_j) over the rows j it sees,
// out = sum_j 2^(c x_j - m) V_j / sum_j 2^(c x_j - m), c = log2 e: one pass over
// the rows with a running maximum m, the running sum and the running weighted
// sum of V rescaled when m grows. The rows of a split or of a wave are done
// apart and joined by the same rule.
//
// Scores are computed transposed, S^T = K Q^T, and so is O^T = V^T P^T: the
// matrix instruction leaves in each lane scores of one query, so a softmax
// reduces within a lane and across two or four of them, and the same registers,
// rounded to bf16, are the second product's operand as they stand: its keys are
// taken in the order in which the first product left them, and the transposing
// LDS read brings V's elements in that order.
//
// All query heads of a KV head are rows of one operand (row r: token r / G, head
// r % G), so the cache is read once for them.
#pragma once

#include <type_traits>

#include "ipv_pages.hpp"

namespace ipv {

constexpr int kAttendStreams = 64;  // streams of one launch (their counts travel in its arguments)
constexpr int kMaxSplits = 64;      // parts of a key range that are joined: a lane each
// The last workgroup of a row tile takes a trip for 1024 elements of up to 16 parts; beyond kJoinTrips
// of them a launch joins the parts.
constexpr int kJoinTrips = 2;
constexpr int64_t join_rounds(int64_t rows, int D) { return (rows * D + 1023) / 1024; }

struct AttendStream {
  int32_t n, first, rows;  // rows of the cache; position of the first query; queries
  int32_t start;           // its first workgroup
  int32_t tiles, splits;   // row tiles of a KV head; parts of a tile's keys
  FastDiv by_tiles, by_splits;
};

struct AttendArgs {
  static constexpr bool kApart = true;  // (a launch of its own can join parts)
  Pool pool;
  int64_t layer_row;  // rows of a page before the layer's first head
  const char* q;
  char* out;
  float* lse;
  int64_t q_b, q_h, q_m, o_b, o_h, o_m;  // strides, elements
  int32_t b0, H, G, max_rows;
  FastDiv G_div;
  float c;  // scale * log2(e)
  int32_t window, sinks;
  float* part;     // unnormalised sums of a split's rows, [workgroup][row][D]
  float* part_ml;  // their maxima and sums of weights, [workgroup][row][2]
  uint32_t* err;
  uint32_t* arrived;  // workgroups of a row tile that have left their part: zero before and after a call
  int32_t streams, blocks;
  int32_t join_apart;  // parts are joined by a launch of its own, not by the last workgroup
  AttendStream s[kAttendStreams];
};

// The key tiles of a range of queries: those that hold one of the first rows
// that stay visible, then those from the oldest row seen to the newest.
struct KeyTiles {
  int32_t sink_tiles, main_first, count;
  int32_t lo, hi, sink_end;  // rows [0, sink_end) and [lo, hi) are seen by some query
  __host__ __device__ KeyTiles(int32_t n, int32_t p_lo, int32_t p_hi, int32_t window, int32_t sinks, int32_t BN) {
    hi = p_hi < n ? p_hi + 1 : n;
    lo = window > 0 && p_lo >= window ? p_lo - window + 1 : 0;
    sink_end = window > 0 ? (sinks < lo ? sinks : lo) : 0;
    if (sink_end > hi) sink_end = hi;
    main_first = lo / BN;
    const int32_t sink = (sink_end + BN - 1) / BN, main_last = (hi + BN - 1) / BN;
    sink_tiles = sink < main_first ? sink : main_first;
    count = sink_tiles + (main_last > main_first ? main_last - main_first : 0);
  }
  __device__ int32_t tile(int32_t t) const { return t < sink_tiles ? t : main_first + t - sink_tiles; }
  __device__ bool some(int32_t j) const { return (j < hi) & ((j >= lo) | (j < sink_end)); }
};

// Whether a query at p sees row j of n.
__device__ __forceinline__ bool sees(int32_t j, int32_t p, int32_t n, int32_t window, int32_t sinks) {
  return (j <= p) & (j < n) & ((window <= 0) | (j > p - window) | (j < sinks));
}
// Whether every query of [p_lo, p_hi] sees all rows of [j0, j1).
__device__ __forceinline__ bool all_see(int32_t j0, int32_t j1, int32_t p_lo, int32_t p_hi, int32_t n, int32_t window,
                                        int32_t sinks) {
  return (j1 - 1 <= p_lo) & (j1 <= n) & ((window <= 0) | (j0 > p_hi - window) | (j1 <= sinks));
}

// The rows of a tile from j0 on that a query sees, as limits on the row's place x
// in the tile: x <= hi and (x > lo or x < first), without branches. The asm keeps
// the limits, and with them the comparisons, in the branch that needs them.
struct Limits {
  int32_t hi, lo, first;
  __device__ __forceinline__ Limits(int32_t j0, int32_t p, int32_t n, int32_t window, int32_t sinks) {
    hi = min(p, n - 1) - j0;
    lo = window > 0 ? p - window - j0 : -1;
    first = sinks - j0;
    asm volatile("" : "+v"(hi), "+v"(lo), "+v"(first));
  }
  __device__ __forceinline__ bool operator()(int32_t x) const { return (x <= hi) & ((x > lo) | (x < first)); }
};

// The same for 64 places as bits: a score is kept or made -inf by two instructions (its bit spread over a
// word, a choice by bits) instead of three comparisons and what joins them.
struct SeenBits {
  uint32_t w[2];
  __device__ __forceinline__ explicit SeenBits(const Limits& in) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      w[i] = below(in.hi + 1 - 32 * i) & (~below(in.lo + 1 - 32 * i) | below(in.first - 32 * i));
  }
  // bits x < k of a word
  static __device__ __forceinline__ uint32_t below(int32_t k) { return k >= 32 ? ~0u : (1u << max(k, 0)) - 1u; }
  __device__ __forceinline__ float operator()(int32_t x, float score) const {
    const uint32_t all = (uint32_t)__builtin_amdgcn_sbfe((int32_t)w[x / 32], x % 32, 1);
    return __uint_as_float((__float_as_uint(score) & all) | (__float_as_uint(-INFINITY) & ~all));
  }
};

// Keeps a rare branch a branch: its body is not computed ahead and selected.
__device__ __forceinline__ void rare() { asm volatile("" ::: "memory"); }

// How far a maximum may grow before the sums are rescaled to it, in the kernel of many rows and that of
// fp32 pools: weights stay below 2^8, which costs the fp32 sums nothing. Weights in bf16 it costs the largest
// one's exactness: rescaled at once that is 1, lazily it is rounded like the others (by up to 2^-8 of it), and
// since it often has the largest part in a result, the error against 64 bits grows, of a frame of 196 tokens of 28
// heads over 6272 positions from 0.0018 to 0.0022 of the result's norm (0.0017 of it the result's own rounding).
// At once costs time: that frame 39.0 -> 40.7 us, its windowed prompt 130 -> 136, 2048 tokens of 64 heads over 32768
// positions 1823 -> 1868, of heads of 256 4475 -> 4775, 1568 tokens over themselves 47.8 -> 52.3.
constexpr float kLazy = 8.f;

// Keeps a value in accumulation registers, which only the matrix unit reads, where the others do not
// suffice: left to itself the compiler moves such values there and back in every step (900 tokens of 64
// heads of 256 over 8192 positions 612 us, 546 without that).
__device__ __forceinline__ void in_acc(F32x16& x) { asm volatile("" : "+a"(x)); }
__device__ __forceinline__ void in_acc(F32x4& x) { asm volatile("" : "+a"(x)); }
__device__ __forceinline__ void in_acc(Bf16x8& x) {
  U32x4 w = __builtin_bit_cast(U32x4, x);
  asm volatile("" : "+a"(w));
  x = __builtin_bit_cast(Bf16x8, w);
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_hw(float x) { return __builtin_amdgcn_logf(x); }
constexpr float kLn2 = 0.693147180559945309f;

// A maximum as the exponent's shift: a query that has seen nothing has -inf,
// and nothing to shift.
__device__ __forceinline__ float shift_of(float m) { return m == -INFINITY ? 0.f : m; }

// Maximum and sum over the lanes that hold the same query: 32 apart (two
// halves of a 32-wide tile), or 16 and 32 apart.
template <int N>
__device__ __forceinline__ float lanes_max(float v) {
  if (N == 4) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <int N>
__device__ __forceinline__ float lanes_sum(float v) {
  if (N == 4) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Maximum and sum over the wave, in all lanes.
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp_f32<kDppXor1>(v));
  v = fmaxf(v, dpp_f32<kDppXor2>(v));
  v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
  v = fmaxf(v, dpp_f32<kDppRowMirror>(v));
  return lanes_max<4>(v);
}
__device__ __forceinline__ float wave_sum(float v) { return lanes_sum<4>(group_sum<16>(v)); }

// Four bf16 of one column from four rows of LDS: the 16 lanes of a group give
// the addresses of a 4 x 16 block, row by row, 8 bytes each; lane i receives
// column i.
typedef short S16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ U32x2 lds_column4(const char* p) {
  return __builtin_bit_cast(U32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((S16x4 __attribute__((address_space(3)))*)p));
}

// The block's place: its stream, KV head, row tile and part of the keys.
// Workgroups go to the eight XCDs in turn; each XCD takes a run of consecutive
// places, so the tiles and parts that read one head's rows share its L2.
struct Place {
  int32_t slot, b, h, tile, split;
  int32_t first;  // slot of the row tile's first part
};
__device__ __forceinline__ Place place_of(const AttendArgs& a) {
  // the arguments that the first loads wait for, all on their way at once
  asm volatile("" ::"s"(a.blocks), "s"(a.streams), "s"(a.pool.K), "s"(a.pool.V), "s"(a.pool.table), "s"(a.pool.T.m), "s"(a.q),
               "s"(a.G_div.m), "s"(a.window), "s"(a.s[0].n), "s"(a.s[0].by_splits.m), "s"(a.layer_row), "s"(a.pool.page_rows_all));
  const uint32_t per = (uint32_t)(a.blocks + 7) / 8u;
  Place p;
  p.slot = (int32_t)((blockIdx.x % 8u) * per + blockIdx.x / 8u);
  p.b = 0;
  if (p.slot >= a.blocks) {
    p.slot = -1;
    return p;
  }
  int lo = 0, hi = a.streams - 1;  // the last stream that starts at or before the slot (empty ones hold no slot)
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.s[mid].start <= p.slot) lo = mid;
    else hi = mid - 1;
  }
  p.b = lo;
  const AttendStream& s = a.s[lo];
  const uint32_t x = (uint32_t)(p.slot - s.start), y = fast_div(x, s.by_splits);
  p.split = (int32_t)(x - y * (uint32_t)s.splits);
  p.first = p.slot - p.split;
  p.h = (int32_t)fast_div(y, s.by_tiles);
  // the last row tile first: under a causal mask it has the most keys
  p.tile = s.tiles - 1 - (int32_t)(y - (uint32_t)p.h * (uint32_t)s.tiles);
  return p;
}

// Stored elements of a row that some query does not see: nothing of them if none
// does, else without infinities (in bf16) and NaN (a product with a weight of zero would
// be NaN). Whether any were taken out of a row that some see.
template <int F>
__device__ __forceinline__ bool clean(uint32_t (&x)[4], uint64_t& scales, int block, bool some) {
  bool special = false, nan = false;
  asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));  // nothing of this outside the branch that needs it
  if constexpr (fmt_scaled(F)) {
    // values of 2^128 and more, infinite in bf16, need a scale of 2^120 (e4m3) or 2^126 (e2m1) at least
    constexpr uint32_t large = F == kFmtFp8 ? 247u : 253u;
    const uint32_t byte = (uint32_t)(scales >> (8 * block)) & 255u;
    nan = byte == 255u;
    special = nan && some;
    if (nan) scales = 0;
    if (byte >= large && !nan) {  // all elements of a word at once, by their exponents
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t over;
        if constexpr (F == kFmtFp8) over = (((x[e] >> 3) & 0x0f0f0f0fu) + (byte - 246u) * 0x01010101u) >> 4 & 0x01010101u;
        else over = x[e] >> 2 & (byte == large ? x[e] >> 1 : ~0u) & 0x11111111u;
        x[e] &= ~(over * (F == kFmtFp8 ? 255u : 15u));
        special |= some & (over != 0);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (!some || nan) x[e] = 0;
    if constexpr (F == kFmtBf16) {
      if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u, special = true;
      if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu, special = true;
    } else if constexpr (F == kFmtFp8) {
#pragma unroll
      for (int k = 0; k < 32; k += 8)
        if (((x[e] >> k) & 0x7fu) == 0x7fu) x[e] &= ~(0xffu << k), special = true;
    }
  }
  return special;
}

// Parts that another workgroup, maybe on another XCD, will read: stored and loaded
// past this XCD's L2 (the cache policy of agent scope), 16 and 8 bytes at a time.
constexpr int kAgentScope = 16;  // the sc1 bit of a buffer instruction
__device__ __forceinline__ void store_part(__amdgpu_buffer_rsrc_t parts, uint32_t offset, const F32x4& v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(U32x4, v), parts, (int)offset, 0, kAgentScope);
}
__device__ __forceinline__ F32x4 load_part(__amdgpu_buffer_rsrc_t parts, uint32_t offset) {
  return __builtin_bit_cast(F32x4, __builtin_amdgcn_raw_buffer_load_b128(parts, (int)offset, 0, kAgentScope));
}
__device__ __forceinline__ void store_pair(float* p, float a, float b) {
  const uint64_t v = ((uint64_t)__float_as_uint(b) << 32) | __float_as_uint(a);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void load_pair(const float* p, float& a, float& b) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  a = __uint_as_float((uint32_t)v), b = __uint_as_float((uint32_t)(v >> 32));
}

// One element of V, for the rare rows that need care.
template <int F, int D>
__device__ __forceinline__ float v_element(const Pool& p, int64_t row, int d) {
  float f[8];
  decode_row8<F, D>(p.V, p.Vs, row, d & ~7, f);
  float v = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i == (d & 7)) v = f[i];
  return v;
}

// Eight elements at 8 * s of a 16-byte (or shorter) piece of stored bytes, as bf16.
template <int F>
__device__ __forceinline__ Raw16 piece8(const uint32_t* w, int s, float scale) {
  if (F == kFmtFp8) return fp8_to_bf16(w[2 * s], w[2 * s + 1], scale);
  if (F == kFmtFp4) return fp4_to_bf16(w[s], scale);
  return Raw16{w[0], w[1], w[2], w[3]};
}

// Sixteen bytes a lane from memory straight into LDS: lane i's to `at` + 16 i, `at` the
// same in all lanes. No register waits for them: copies_done() does, for all of the wave's.
__device__ __forceinline__ void copy_to_lds(const char* from, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(from) : "memory", "m0");
}
// From `base`, the same in all lanes, + offset.
__device__ __forceinline__ void copy_to_lds(const char* base, uint32_t offset, uint32_t at) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void copies_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const char* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}

// ---------------------------------------------------------------- few rows
// Up to 16 * NB rows a KV head (single tokens of grouped heads): bound by the
// bytes of the cache. Each wave takes key tiles of its own (32 rows), K straight
// into the matrix operand's layout, V through an LDS tile that only this wave
// uses (bf16: copied there, two tiles in turn); the next tile's rows are in flight
// while one is computed. The four waves join through LDS; parts of a key range through
// memory, by the last workgroup to come or, where that takes it long, by k_attend_join.
// One token of 8 streams over 32768 positions of 8 heads of 128: 184 us in bf16 (5.8 TB/s),
// 106 in fp8 (5.2), 53 in fp4 (5.4); of one stream, where the start, the first rows' way and
// the join weigh, 28 us (4.8 TB/s) in bf16 and 16 in fp4.
constexpr int kFewWaves = 4;
constexpr int kFewKeys = 32;

template <int F, int D>
struct FewCfg {
  static constexpr int RB = fmt_row_bytes(F, D);
  static constexpr int KQ = RB / 4;                   // bytes of a K row that a lane holds
  static constexpr int KB = KQ < 16 ? KQ : 16;        // bytes a load
  static constexpr int KN = KQ / KB;
  static constexpr int KE = KB * 8 / fmt_bits(F);     // elements a load
  static constexpr int CPR = RB / 16;                 // 16-byte chunks of a V row
  static constexpr int NV = CPR >= 2 ? CPR / 2 : 1;   // chunks a lane loads
  static constexpr int VE = 128 / fmt_bits(F);        // elements a chunk
  // V's 16-byte chunks of bf16 are stored at ch ^ swizzle(row): eight rows of a
  // transposing read then lie in different banks
  static __device__ int swz(int row) {
    return D >= 128 ? 2 * (row & 7) : D == 64 ? 2 * ((row >> 1) & 3) : 2 * ((row >> 2) & 1);
  }
};

// LDS of the joining: each wave's sums of its keys, [row][D + 4] a wave, relative to
// the workgroup's maximum of the row; their maxima and sums of weights.
template <int D, int NR>
struct JoinLds {
  static constexpr int STRIDE = D + 4;
  static constexpr size_t kWaveBytes = (size_t)NR * STRIDE * 4;
};

// Workgroups of a CU, by registers and LDS.
constexpr int few_per_cu(int F, int D, int NB) {
  return NB * D > 256 || (F == kFmtBf16 && D > 128) ? 1 : fmt_scaled(F) && NB * D <= 128 ? 3 : 2;  // (D = 256: by its bf16 tiles)
}

template <int F, int D, int NB>
constexpr size_t few_wave_lds() {
  constexpr size_t tile = (size_t)kFewKeys * D * 2 * (F == kFmtBf16 ? 2 : 1), join = JoinLds<D, 16 * NB>::kWaveBytes;
  return tile > join ? tile : join;
}

// Four elements of row r's result, and its lse: v, sum and top are the weighted
// sum, the sum of the weights and the maximum they are relative to.
template <int D, bool F32OUT, class ARGS>
__device__ __forceinline__ void row_out(const ARGS& a, int b, int h, int r, int d, const F32x4& v, float top, float sum) {
  const int tok = (int)fast_div((uint32_t)r, a.G_div), head = h * a.G + r - tok * a.G;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int64_t at = (int64_t)b * a.o_b + (int64_t)head * a.o_h + (int64_t)tok * a.o_m + d;
  if (F32OUT) *reinterpret_cast<F32x4*>(a.out + 4 * at) = v * inv;
  else *reinterpret_cast<U32x2*>(a.out + 2 * at) = U32x2{pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv)};
  if (d == 0 && a.lse)
    a.lse[((int64_t)b * (a.H * a.G) + head) * a.max_rows + tok] = sum == 0.f ? -INFINITY : (top + log2_hw(sum)) * kLn2;
}

// The waves' sums are in LDS: their total is the result of the first `rows` rows of the
// row tile (rows r0, ... of the stream) or, where the keys are split, a part of it. The row
// tile's last workgroup to come joins its parts, in their order.
template <int D, int NR, bool F32OUT, size_t BYTES, class ARGS>
__device__ __forceinline__ void join_parts(const ARGS& a, const AttendStream& st, const Place& pl, int b, int r0, int rows,
                                           char (&lds)[kFewWaves][BYTES], float (&lds_ml)[kFewWaves][NR][2], uint32_t* lds_last) {
  constexpr int STRIDE = JoinLds<D, NR>::STRIDE;
  static_assert(BYTES >= JoinLds<D, NR>::kWaveBytes && kFewWaves * BYTES >= sizeof(float) * NR * kMaxSplits, "LDS of the joining");
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  // the row tile's parts, [part][row][D]
  const __amdgpu_buffer_rsrc_t parts = buffer_rsrc(a.part + (int64_t)pl.first * NR * D, (uint32_t)(st.splits * NR * D * 4));
  for (int x = threadIdx.x; x < rows * (D / 4); x += 64 * kFewWaves) {
    const int r = x / (D / 4), d = x % (D / 4) * 4;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, lds_ml[w][r][0]);
    F32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      sum += lds_ml[w][r][1] * exp2_hw(lds_ml[w][r][0] - shift_of(top));
      v += *reinterpret_cast<const F32x4*>(reinterpret_cast<const float*>(lds[w]) + r * STRIDE + d);
    }
    if (st.splits > 1) {
      store_part(parts, (uint32_t)((pl.split * NR + r) * D + d) * 4, v);
      if (d == 0) store_pair(a.part_ml + ((int64_t)pl.slot * NR + r) * 2, top, sum);
    } else {
      row_out<D, F32OUT>(a, b, pl.h, r0 + r, d, v, top, sum);
    }
  }
  if (st.splits <= 1) return;
  if constexpr (ARGS::kApart) {
    if (a.join_apart) return;
    if (!F32OUT && NR > 16 && join_rounds(17, D) > kJoinTrips) return;  // (as many rows always are)
  }

  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this thread's parts are written
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t* count = a.arrived + pl.first;
    const uint32_t before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *lds_last = before + 1 == (uint32_t)st.splits;
    if (*lds_last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!*lds_last) return;
  // Each thread has four elements of a row and takes 16 parts at a time, the first
  // ones on their way while the parts' weights are made (a trip to another XCD's
  // data takes over a microsecond).
  constexpr int ROUND = 16;
  F32x4 y[ROUND];
  const auto load_round = [&](int x, int k0) __attribute__((always_inline)) {
    const uint32_t at = (uint32_t)(min(x / (D / 4), rows - 1) * D + x % (D / 4) * 4) * 4;
#pragma unroll
    for (int k = 0; k < ROUND; ++k) y[k] = load_part(parts, at + (uint32_t)((k0 + k) * NR * D * 4));  // (zeros past the last)
  };
  load_round(threadIdx.x, 0);
  // weights of the parts, by row: lane s has part s
  float(*weight)[kMaxSplits] = reinterpret_cast<float(*)[kMaxSplits]>(&lds[0][0]);
  constexpr int RW = NR / kFewWaves;  // rows of a wave, all on their way at once
  float pm[RW], ps[RW];
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    const int r = i * kFewWaves + wave;
    pm[i] = -INFINITY, ps[i] = 0.f;
    if (r < rows && lane < st.splits) load_pair(a.part_ml + ((int64_t)(pl.first + lane) * NR + r) * 2, pm[i], ps[i]);
  }
#pragma unroll
  for (int i = 0; i < RW; ++i) {
    const int r = i * kFewWaves + wave;
    const float top = wave_max(pm[i]), f = exp2_hw(pm[i] - shift_of(top)), sum = wave_sum(ps[i] * f);
    weight[r][lane] = f;
    if (lane == 0) lds_ml[0][r][0] = top, lds_ml[0][r][1] = sum;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < rows * (D / 4); x += 64 * kFewWaves) {
    const int r = x / (D / 4), d = x % (D / 4) * 4;
    if (x != (int)threadIdx.x) load_round(x, 0);
    F32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0;;) {
#pragma unroll
      for (int k = 0; k < ROUND; ++k)
        if (k0 + k < st.splits) v += y[k] * weight[r][k0 + k];
      k0 += ROUND;
      if (k0 >= st.splits) break;
      load_round(x, k0);
    }
    row_out<D, F32OUT>(a, b, pl.h, r0 + r, d, v, lds_ml[0][r][0], lds_ml[0][r][1]);
  }
}

// WHOLE: pages hold whole tiles (their rows are a multiple of a tile's), so a tile's rows follow
// each other: one page to look up, by a scalar load, and one scalar base with 32-bit offsets that
// stay the same, where otherwise each lane has a 64-bit address a row. For D = 256 that is also
// what makes its registers suffice: one token of fp8 over 16384 positions of 8 heads takes 22.1 us
// with it and 28.5 without, four tokens of bf16 49.4 and 64.5.
template <int F, int D, int NB, bool WHOLE>
__global__ __launch_bounds__(64 * kFewWaves, few_per_cu(F, D, NB)) void k_attend_few(AttendArgs a) {
  using C = FewCfg<F, D>;
  __shared__ __attribute__((aligned(16))) char lds[kFewWaves][few_wave_lds<F, D, NB>()];
  __shared__ float lds_ml[kFewWaves][16 * NB][2];
  __shared__ uint32_t lds_last;
  const Place pl = place_of(a);
  if (pl.slot < 0) return;  // the whole workgroup
  const AttendStream st = a.s[pl.b];
  const int lane = threadIdx.x % kWave, g = lane / 16, l16 = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t n = st.n, p_lo = st.first, p_hi = st.first + st.rows - 1, R = st.rows * a.G;
  const int b = a.b0 + pl.b;
  const int64_t head_row = a.layer_row + (int64_t)pl.h * a.pool.T.d;
  const KeyTiles kt(n, p_lo, p_hi, a.window, a.sinks, kFewKeys);
  const int32_t t_end = (int32_t)((int64_t)kt.count * (pl.split + 1) / st.splits);
  int32_t t = (int32_t)((int64_t)kt.count * pl.split / st.splits) + wave;

  // queries: lane's row and, in its pieces' order, its elements
  Bf16x8 q[NB][D / 32];
  int32_t pos[NB];
  const char* q_at[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = min(nb * 16 + l16, R - 1), tok = (int)fast_div((uint32_t)r, a.G_div);
    pos[nb] = p_lo + tok;
    q_at[nb] = a.q + 2 * ((int64_t)b * a.q_b + (int64_t)(pl.h * a.G + r - tok * a.G) * a.q_h + (int64_t)tok * a.q_m);
  }

  F32x4 o[NB][D / 16];
  float m[NB], l[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = -INFINITY, l[nb] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[nb][i] = F32x4{0.f, 0.f, 0.f, 0.f};
  }

  // Whether a row that some query sees has no page: a tile of other rows than a whole page's may
  // also hold rows that none sees, whose entries say nothing (every tile has one that is seen).
  bool bad = false;
  // the tile's key lane % 32, or its first; a key past the last is the last; its page, and its row in the pool
  const auto key_of = [&](int32_t tt) __attribute__((always_inline)) {
    return min(kt.tile(min(tt, kt.count - 1)) * kFewKeys + (WHOLE ? 0 : lane % 32), n - 1);
  };
  const auto page_of = [&](int32_t tt) __attribute__((always_inline)) {
    return WHOLE ? pool_page_uniform(a.pool, b, (uint32_t)key_of(tt)) : pool_page(a.pool, b, (uint32_t)key_of(tt));
  };
  const auto row_of = [&](int32_t page, int32_t tt) __attribute__((always_inline)) {
    bool x;
    const int32_t j = key_of(tt);
    const int64_t r = pool_row(a.pool, page, (uint32_t)j, &x) + head_row;
    bad |= x & (WHOLE | kt.some(j));
    return r;
  };
  constexpr bool COPY = F == kFmtBf16;
  uint32_t kr[2][C::KQ / 4], vr[COPY ? 1 : C::NV][4];
  uint64_t ks[2], vs[COPY ? 1 : C::NV];
  char* tile = lds[wave];
  auto fetch = [&](int64_t row, char* v_tile) __attribute__((always_inline)) {
    // rows from the tile's first one on (WHOLE: base and 32-bit offset), or each in the pool
    using At = std::conditional_t<WHOLE, uint32_t, int64_t>;
    const int64_t base = WHOLE ? row : 0;
    const char* kp = a.pool.K + base * C::RB;
    const char* vp = a.pool.V + base * C::RB;
    const uint8_t* ksp = a.pool.Ks + base * (D / kScaleBlock);
    const uint8_t* vsp = a.pool.Vs + base * (D / kScaleBlock);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const At r = WHOLE ? l16 : shfl64(row, kb * 16 + l16);
      constexpr int up = WHOLE ? 16 : 0;
#pragma unroll
      for (int c = 0; c < C::KN; ++c)
        load_piece<C::KB>(kp + (kb * up * C::RB + c * 4 * C::KB) + (At)(r * C::RB + g * C::KB), kr[kb] + c * (C::KB / 4));
      if (fmt_scaled(F)) ks[kb] = load_scales<D>(ksp + kb * up * (D / kScaleBlock), r);
    }
#pragma unroll
    for (int i = 0; i < C::NV; ++i) {
      const int key = (i * kWave + lane) / C::CPR % kFewKeys;  // (a piece too many is the first ones' again)
      constexpr int step = WHOLE ? kWave / C::CPR : 0;
      const At r = WHOLE ? (lane / C::CPR) % kFewKeys : shfl64(row, key);
      if constexpr (COPY) {  // the source column makes up for the place
        const int ch = lane % C::CPR ^ C::swz((i * kWave + lane) / C::CPR);
        const uint32_t at = __builtin_amdgcn_readfirstlane(lds_address(v_tile) + i * 1024);
        if constexpr (WHOLE) copy_to_lds(vp + i * step * C::RB, r * C::RB + ch * 16, at);
        else copy_to_lds(vp + (r * C::RB + ch * 16), at);
      } else {
        load_piece<16>(vp + i * step * C::RB + (At)(r * C::RB + lane % C::CPR * 16), vr[i]);
        if (fmt_scaled(F)) vs[i] = load_scales<D>(vsp + i * step * (D / kScaleBlock), r);
      }
    }
  };

  int32_t next = 0;      // the next tile's page
  bool special = false;  // V held infinities or NaN in rows that only some queries see
  const int32_t t_begin = t;
  if (t < t_end) {
    const int32_t page = page_of(t);
    next = page_of(t + kFewWaves);
    fetch(row_of(page, t), tile);
    // (after the rows, whose addresses took a trip to the table)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int c = 0; c < C::KN; ++c)
#pragma unroll
        for (int s = 0; s < C::KE / 8; ++s)
          q[nb][c * (C::KE / 8) + s] = __builtin_bit_cast(Bf16x8, load16(q_at[nb] + 2 * ((c * 4 + g) * C::KE + 8 * s)));
  }
  constexpr int VTILE = kFewKeys * D * 2;
  int vbuf = 0;
  for (; t < t_end; t += kFewWaves) {
    if constexpr (COPY) copies_done();
    const int32_t j0 = kt.tile(t) * kFewKeys;
    const bool full = all_see(j0, j0 + kFewKeys, p_lo, p_hi, n, a.window, a.sinks);
    // scores of this tile's keys (the operand is built from the loaded bytes)
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
    // V into LDS as bf16; rows that no query sees become zeros, and what is
    // infinite or NaN in rows that only some see is taken out and added at the end
    if (!full) {
      int32_t jv = j0;
      asm volatile("" : "+v"(jv));
#pragma unroll
      for (int i = 0; i < C::NV; ++i) {
        const int x = i * kWave + lane;
        const bool some = kt.some(jv + x / C::CPR);
        if constexpr (COPY) {
          Raw16* p = reinterpret_cast<Raw16*>(tile + vbuf * VTILE + x * 16);  // as this lane copied it
          const Raw16 v = *p;
          uint32_t e[4] = {v.w[0], v.w[1], v.w[2], v.w[3]};
          uint64_t none = 0;
          special |= clean<F>(e, none, 0, some);
          *p = Raw16{e[0], e[1], e[2], e[3]};
        } else {
          special |= clean<F>(vr[i], vs[i], x % C::CPR * C::VE / kScaleBlock, some);
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
    if (t + kFewWaves < t_end) {
      const int64_t row = row_of(next, t + kFewWaves);
      next = page_of(t + 2 * kFewWaves);  // before the rows: what waits for it need not wait for them
      fetch(row, tile + (vbuf ^ 1) * VTILE);
    }
    // softmax: weights of 8 keys a lane, keys 4 g + i and 16 + 4 g + i
    Bf16x8 w[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (!full) {
        const Limits in(j0 + 4 * g, pos[nb], n, a.window, a.sinks);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!in(kb * 16 + i)) sc[nb][kb][i] = -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(fmaxf(top, sc[nb][0][i]), sc[nb][1][i]);
      top = lanes_max<4>(top) * a.c;
      // The sums are rescaled as soon as a maximum grows, so that the largest weight is 1 and not rounded; only
      // where a maximum has grown (four tokens of 8 streams of 64 heads of 256 in e2m1 over 32768 positions 183 us,
      // in every tile 214). Rescaled lazily, as by the kernel of many rows, those would take 162 us, in e4m3 200 in
      // place of 219, in bf16 353 in place of 356, and be off by 0.0023 of the result's norm in place of 0.0019.
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
      const char* at = tile + (COPY ? vbuf * VTILE : 0);
      const U32x2 x = lds_column4(at + k0 * (D * 2) + 16 * (ch ^ C::swz(k0)) + in);
      const U32x2 y = lds_column4(at + (k0 + 16) * (D * 2) + 16 * (ch ^ C::swz(k0 + 16)) + in);
      const Raw16 r = {x.x, x.y, y.x, y.y};
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf16x8, r), w[nb], o[nb][db], 0, 0, 0);
    }
    __builtin_amdgcn_wave_barrier();
    vbuf ^= 1;
  }
  if (__ballot(special) != 0) {
#pragma unroll 1
    for (int32_t tt = t_begin; tt < t_end; tt += kFewWaves) {
      const int32_t j0 = kt.tile(tt) * kFewKeys;
      if (all_see(j0, j0 + kFewKeys, p_lo, p_hi, n, a.window, a.sinks)) continue;
      const int64_t row = row_of(page_of(tt), tt);
#pragma unroll 1
      for (int key = 0; key < kFewKeys; ++key) {
        if (!kt.some(j0 + key)) continue;
        const int64_t r = WHOLE ? row + key : shfl64(row, key);
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = v_element<F, D>(a.pool, r, 16 * db + 4 * g + i);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
              if (!(fabsf(v) < INFINITY) & sees(j0 + key, pos[nb], n, a.window, a.sinks)) o[nb][db][i] += v;
          }
      }
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
  join_parts<D, 16 * NB, false>(a, st, pl, b, 0, min(R, 16 * NB), lds, lds_ml, &lds_last);
}

// ---------------------------------------------------------------- many rows
// Row tiles of 32 rows a wave, keys in tiles of 64 through LDS, where all waves
// read them; the next tiles' rows are in flight meanwhile. Two waves a SIMD, or one
// for D = 256, whose sums and queries take 192 accumulation registers. Bound by the matrix
// unit, at a clock that its load lowers: 2048 tokens of 64 heads over 32768 positions of 8,
// D = 128, take 1790 to 1890 us, 1130 to 1190 TFLOP/s at 60% of the unit's cycles and 1.86 GHz (the library's
// product of random bf16 matrices reaches 1490); fp8 1860 to 1930. D = 64: half the products with the
// same softmax instructions, 38% of the unit's cycles, 900 TFLOP/s; D = 256, one wave a SIMD: 40%, 950.
// 128 rows a workgroup, two of them a CU: 2045 us; 64 rows a wave, one wave a SIMD: 3135.
// Short calls are bound by the way to their first rows and back: a frame of 196 tokens of 28 heads
// over 6272 positions 33 us and 7.6 for the join, of 12 at the library product's rate.
constexpr int kTileKeys = 64;
__host__ __device__ constexpr int tile_waves(int D) { return D <= 128 ? 8 : 4; }

template <int F, int D, int W>
struct TileCfg {
  static constexpr int RB = fmt_row_bytes(F, D);
  static constexpr int CPR = RB / 16;
  static constexpr int CHUNKS = kTileKeys * CPR;
  static constexpr int NL = CHUNKS >= 64 * W ? CHUNKS / (64 * W) : 1;  // chunks a thread loads
  static constexpr int E = 128 / fmt_bits(F);                          // elements a chunk
  // LDS places of 16-byte chunks of bf16: K is read 16 bytes a lane from 32
  // rows, V by transposing reads of 4 rows and 32 columns
  static __device__ int kswz(int row) { return D >= 128 ? row & 15 : D == 64 ? (row >> 1) & 7 : (row >> 2) & 3; }
  static __device__ int vswz(int row) { return D >= 128 ? 4 * (row & 3) : D == 64 ? 4 * ((row >> 1) & 1) : 0; }
};

// WHOLE: as for the kernel of few rows; 2048 tokens of 64 heads over 32768 positions of 8, D = 128,
// take 1820 us with it and 1901 without.
template <int F, int D, bool WHOLE>
__global__ __launch_bounds__(64 * tile_waves(D), tile_waves(D) / 4) void k_attend_tile(AttendArgs a) {
  constexpr int W = tile_waves(D), BM = 32 * W, BN = kTileKeys;
  using C = TileCfg<F, D, W>;
  // bf16 rows are copied straight into LDS; the others pass through registers, as bf16
  constexpr bool COPY = F == kFmtBf16;
  __shared__ __attribute__((aligned(16))) char ldsK[2][BN * D * 2];
  __shared__ __attribute__((aligned(16))) char ldsV[2][BN * D * 2];
  __shared__ int32_t lds_special;
  const Place pl = place_of(a);
  if (pl.slot < 0) return;
  const AttendStream st = a.s[pl.b];
  const int lane = threadIdx.x % kWave, h = lane / 32, l32 = lane % 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t n = st.n, R = st.rows * a.G, r0 = pl.tile * BM;
  const int b = a.b0 + pl.b;
  const int64_t head_row = a.layer_row + (int64_t)pl.h * a.pool.T.d;
  const int32_t p_lo = st.first + (int32_t)fast_div((uint32_t)r0, a.G_div);
  const int32_t p_hi = st.first + (int32_t)fast_div((uint32_t)(min(r0 + BM, R) - 1), a.G_div);
  const KeyTiles kt(n, p_lo, p_hi, a.window, a.sinks, BN);
  const int32_t t_end = (int32_t)((int64_t)kt.count * (pl.split + 1) / st.splits);
  int32_t t = (int32_t)((int64_t)kt.count * pl.split / st.splits);

  Bf16x8 q[D / 16];
  const int qr = min(r0 + wave * 32 + l32, R - 1), tok = (int)fast_div((uint32_t)qr, a.G_div);
  const int32_t pos = st.first + tok;
  // the wave's own positions
  const int32_t pw_lo = st.first + (int32_t)fast_div((uint32_t)min(r0 + wave * 32, R - 1), a.G_div);
  const int32_t pw_hi = st.first + (int32_t)fast_div((uint32_t)min(r0 + wave * 32 + 31, R - 1), a.G_div);

  F32x16 o[D / 32];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = F32x16{};
  if (threadIdx.x == 0) lds_special = 0;

  bool bad = false;
  // the tile's key `lane` (WHOLE: its first); its page, and its row in the pool
  const auto key_of = [&](int32_t tt) __attribute__((always_inline)) {
    return min(kt.tile(min(tt, kt.count - 1)) * BN + (WHOLE ? 0 : lane), n - 1);
  };
  const auto page_of = [&](int32_t tt) __attribute__((always_inline)) {
    return WHOLE ? pool_page_uniform(a.pool, b, (uint32_t)key_of(tt)) : pool_page(a.pool, b, (uint32_t)key_of(tt));
  };
  const auto row_of = [&](int32_t page, int32_t tt) __attribute__((always_inline)) {
    bool x;
    const int32_t j = key_of(tt);
    const int64_t r = pool_row(a.pool, page, (uint32_t)j, &x) + head_row;
    bad |= x & (WHOLE | kt.some(j));
    return r;
  };
  // rows on their way through registers
  constexpr int NX = COPY ? 1 : C::NL;
  uint32_t kr[NX][4], vr[NX][4];
  uint64_t ks[NX], vs[NX];
  // this thread's chunks: column threadIdx.x % CPR of rows key0 + i * 64 W / CPR
  const int key0 = threadIdx.x / C::CPR % BN;
  constexpr int STEP = 64 * W / C::CPR;
  const int col = threadIdx.x % C::CPR, block = col * C::E / kScaleBlock;
  const bool mine = C::CHUNKS >= 64 * W || (int)threadIdx.x < C::CHUNKS;  // (whole waves)
  // fetch: rows of a tile set out; stage: they are in LDS buffer `buf` when it is done
  // (copied rows set out with their buffer known; the source column makes up for the place)
  const auto fetch = [&](const char* pages, const uint8_t* scales, int64_t row, const char* buf, auto swz, auto& x, auto& xs)
      __attribute__((always_inline)) {
    using At = std::conditional_t<WHOLE, uint32_t, int64_t>;
    const int64_t base = WHOLE ? row : 0;
    const uint32_t at = __builtin_amdgcn_readfirstlane(lds_address(buf) + wave * 1024);
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const int key = key0 + i * STEP;
      const char* p = pages + (base + (WHOLE ? i * STEP : 0)) * C::RB;
      const At r = WHOLE ? key0 : shfl64(row, key);
      if constexpr (COPY) {
        const int ch = col ^ swz(key);
        if (!mine) continue;
        if constexpr (WHOLE) copy_to_lds(p, r * C::RB + 16 * ch, at + i * 1024 * W);
        else copy_to_lds(p + (r * C::RB + 16 * ch), at + i * 1024 * W);
      } else {
        load_piece<16>(p + (At)(r * C::RB + col * 16), x[i]);
        if (fmt_scaled(F)) xs[i] = load_scales<D>(scales + (base + (WHOLE ? i * STEP : 0)) * (D / kScaleBlock), r);
      }
    }
  };
  const auto fetch_k = [&](int64_t row, int buf) __attribute__((always_inline)) {
    fetch(a.pool.K, a.pool.Ks, row, ldsK[buf], [](int key) { return C::kswz(key); }, kr, ks);
  };
  const auto fetch_v = [&](int64_t row, int buf) __attribute__((always_inline)) {
    fetch(a.pool.V, a.pool.Vs, row, ldsV[buf], [](int key) { return C::vswz(key); }, vr, vs);
  };
  const auto stage_k = [&](int buf) __attribute__((always_inline)) {
    if constexpr (!COPY) {
      if (!mine) return;
#pragma unroll
      for (int i = 0; i < C::NL; ++i) {
        const int key = key0 + i * STEP;
#pragma unroll
        for (int e = 0; e < C::E / 8; ++e)
          *reinterpret_cast<Raw16*>(ldsK[buf] + key * (D * 2) + 16 * ((col * (C::E / 8) + e) ^ C::kswz(key))) =
              piece8<F>(kr[i], e, scale_at(ks[i], block));
      }
    }
  };
  // After the wave's copies are done. Where some query does not see all of the tile, rows that no
  // query sees become zeros, and what is infinite or NaN in rows that only some see is
  // taken out here and added at the end.
  const auto stage_v = [&](int32_t tt, int buf) __attribute__((always_inline)) {
    if constexpr (COPY) copies_done();
    if (!mine) return;
    const int32_t j0 = kt.tile(tt) * BN;
    if (!all_see(j0, j0 + BN, p_lo, p_hi, n, a.window, a.sinks)) {
      int32_t jv = j0;
      asm volatile("" : "+v"(jv));
      bool special = false;
#pragma unroll
      for (int i = 0; i < C::NL; ++i) {
        const bool some = kt.some(jv + key0 + i * STEP);
        if constexpr (COPY) {
          Raw16* p = reinterpret_cast<Raw16*>(ldsV[buf] + (threadIdx.x + i * 64 * W) * 16);  // as this thread copied it
          const Raw16 v = *p;
          uint32_t x[4] = {v.w[0], v.w[1], v.w[2], v.w[3]};
          uint64_t none = 0;
          special |= clean<F>(x, none, 0, some);
          *p = Raw16{x[0], x[1], x[2], x[3]};
        } else {
          special |= clean<F>(vr[i], vs[i], block, some);
        }
      }
      if (special) lds_special = 1;
    }
    if constexpr (!COPY)
#pragma unroll
      for (int i = 0; i < C::NL; ++i) {
        const int key = key0 + i * STEP;
#pragma unroll
        for (int e = 0; e < C::E / 8; ++e)
          *reinterpret_cast<Raw16*>(ldsV[buf] + key * (D * 2) + 16 * ((col * (C::E / 8) + e) ^ C::vswz(key))) =
              piece8<F>(vr[i], e, scale_at(vs[i], block));
      }
  };

  // LDS addresses of a lane's operands: the rest is the same for all lanes
  int kat[D / 16], vat[D / 32];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) kat[kk] = l32 * (D * 2) + 16 * ((2 * kk + h) ^ C::kswz(l32));
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    const int k0 = 4 * h + (lane % 16) / 4, ch = 4 * db + 2 * ((lane / 16) % 2) + (lane % 4) / 2;
    vat[db] = k0 * (D * 2) + 16 * (ch ^ C::vswz(k0)) + 8 * (lane & 1);
  }
  // A tile's scores, a lane's largest of them, and the weights made from them.
  F32x16 s[2];
  float most = -INFINITY;
  const auto k_operand = [&](int kbuf, int i) __attribute__((always_inline)) {  // of the i-th product of a tile's scores
    return __builtin_bit_cast(Bf16x8, load16(ldsK[kbuf] + i / (D / 16) * 32 * (D * 2) + kat[i % (D / 16)]));
  };
  const auto v_operand = [&](int vbuf, int i) __attribute__((always_inline)) {  // of the i-th product with the weights
    const char* at = ldsV[vbuf] + i / (D / 32) * 16 * (D * 2) + vat[i % (D / 32)];
    const U32x2 x = lds_column4(at), y = lds_column4(at + 8 * (D * 2));
    return __builtin_bit_cast(Bf16x8, Raw16{x.x, x.y, y.x, y.y});
  };
  const auto largest = [&](const F32x16 (&x)[2], int i0, int i1, float v) __attribute__((always_inline)) {
#pragma unroll
    for (int i = i0; i < i1; ++i) v = fmaxf(fmaxf(v, x[0][i]), x[1][i]);
    return v;
  };
  // Tile t: its scores are there, its V is in buffer BUF. The scores of tile
  // t + 1 are computed beside its softmax. A product takes the matrix unit 32 cycles
  // in which the vector unit is free: the source has between two products what
  // fits there, and their operands' reads two or three products ahead.
  int64_t rows;      // of tile t + 1
  int32_t page = 0;  // of the tile after it
  const int32_t t_begin = t;
  constexpr int NS = D / 8, NP = D / 8, HALF = NP / 2;  // products for the scores, and with the weights
  // operands in flight: KA products ahead of the first kind's, VA of the second's
  constexpr int KA = NS < 5 ? NS : 5, VA = NP < 4 ? NP : 4;
  Bf16x8 kf[KA + 1];
  auto step = [&](auto bufc) __attribute__((always_inline)) {
    constexpr int BUF = decltype(bufc)::value, NEXT = BUF ^ 1;  // tile t's buffers, and t + 1's
    // Tile t + 1's K and t's V are in LDS, and no wave reads what is written below.
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KA; ++i) kf[i] = k_operand(NEXT, i);
    F32x16 ahead[2];
    const auto score = [&](int i) __attribute__((always_inline)) {  // the i-th product of tile t + 1's scores
      const int kb = i / (D / 16), kk = i % (D / 16);
      ahead[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % (KA + 1)], q[kk], kk == 0 ? F32x16{} : ahead[kb], 0, 0, 0);
    };
    Bf16x8 vf[VA + 1];
    const auto operand = [&](int i) __attribute__((always_inline)) {  // of the scores' i-th product, then of the weights' first ones
      if (i < NS) kf[i % (KA + 1)] = k_operand(NEXT, i);
      else if (i - NS < VA) vf[i - NS] = v_operand(BUF, i - NS);
    };
    // The first products need nothing of tile t: its mask, its maximum and the next
    // tiles' loads go beside them.
    constexpr int FIRST = 3;
    static_assert(FIRST < NS && FIRST <= KA, "products before the softmax");
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < FIRST; ++i) {
      operand(i + KA);
      score(i);
    }
    const int64_t later = row_of(page, t + 2);
    page = page_of(t + 3);  // a step before it is needed, and before the copies: nothing waits for it, or for them with it
    fetch_k(later, BUF);
    fetch_v(rows, NEXT);
    const int32_t j0 = kt.tile(t) * BN;
    if (!all_see(j0, j0 + BN, pw_lo, pw_hi, n, a.window, a.sinks)) {
      const SeenBits in(Limits(j0 + 4 * h, pos, n, a.window, a.sinks));
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = in(kb * 32 + 8 * (i / 4) + i % 4, s[kb][i]);
      most = largest(s, 0, 16, -INFINITY);
    }
    float top = lanes_max<2>(most) * a.c;
    if (__ballot(top > m + kLazy) != 0) {
      rare();
      top = fmaxf(top, m);
      const float old = exp2_hw(m - shift_of(top));
      m = top;
      l *= old;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        if constexpr (D > 128) in_acc(o[i]);
        o[i] *= old;
        if constexpr (D > 128) in_acc(o[i]);
      }
    }
    const float shift = shift_of(m);
    Bf16x8 w[4];
    // pairs [p0, p1) of block kb's 16 weights
    const auto weights = [&](int kb, int p0, int p1) __attribute__((always_inline)) {
#pragma unroll
      for (int p = p0; p < p1; ++p) {
        const float x = exp2_hw(__builtin_fmaf(s[kb][2 * p], a.c, -shift));
        const float y = exp2_hw(__builtin_fmaf(s[kb][2 * p + 1], a.c, -shift));
        w[kb * 2 + p / 4][p % 4 * 2] = (__bf16)x;
        w[kb * 2 + p / 4][p % 4 * 2 + 1] = (__bf16)y;
        l += x + y;  // (as fp32: the sum also gives the lse)
      }
    };
    __builtin_amdgcn_s_setprio(1);  // of two waves, the one among its products first (2% of a long prompt)
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = FIRST; i < NS; ++i) {
      operand(i + KA);
      score(i);
      weights(0, 8 * (i - FIRST) / (NS - FIRST), 8 * (i - FIRST + 1) / (NS - FIRST));
      __builtin_amdgcn_sched_barrier(0);
    }
    float biggest = -INFINITY;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (i + VA < NP) vf[(i + VA) % (VA + 1)] = v_operand(BUF, i + VA);
      const int ks4 = i / (D / 32), db = i % (D / 32);
      o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % (VA + 1)], w[ks4], o[db], 0, 0, 0);
      if (i < HALF) {
        weights(1, 8 * i / HALF, 8 * (i + 1) / HALF);
      } else {
        biggest = largest(ahead, 16 * (i - HALF) / HALF, 16 * (i - HALF + 1) / HALF, biggest);
        asm volatile("" : "+v"(biggest));  // here, not where it is next used
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    stage_k(BUF);
    stage_v(t + 1, NEXT);
    s[0] = ahead[0], s[1] = ahead[1];
    most = biggest;
    rows = later;
    ++t;
  };
  if (t < t_end) {
    // tiles past the last are read as the last again, and not used
    const int32_t first = page_of(t), second = page_of(t + 1);
    page = page_of(t + 2);
    const int64_t here = row_of(first, t);
    rows = row_of(second, t + 1);
    __syncthreads();  // lds_special is set
    fetch_k(here, 0);
    stage_k(0);
    fetch_k(rows, 1);
    stage_k(1);
    fetch_v(here, 0);
    const char* q_at = a.q + 2 * ((int64_t)b * a.q_b + (int64_t)(pl.h * a.G + qr - tok * a.G) * a.q_h + (int64_t)tok * a.q_m);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      q[kk] = __builtin_bit_cast(Bf16x8, load16(q_at + 2 * (16 * kk + 8 * h)));
      if constexpr (D > 128) in_acc(q[kk]);
    }
    stage_v(t, 0);
    __syncthreads();
    if (r0 + wave * 32 < R) {
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int kb = i / (D / 16), kk = i % (D / 16);
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(0, i), q[kk], kk == 0 ? F32x16{} : s[kb], 0, 0, 0);
      }
      most = largest(s, 0, 16, -INFINITY);
      for (;;) {
        step(std::integral_constant<int, 0>());
        if (t >= t_end) break;
        step(std::integral_constant<int, 1>());
        if (t >= t_end) break;
      }
    } else {  // no rows: only the other waves' keys, in the same steps (6 tokens of 32 heads, 16 streams over
              // 12000 positions: 80 us against 112 with products of the last row over again)
      for (int buf = 0; t < t_end; ++t, buf ^= 1) {
        __syncthreads();
        const int64_t later = row_of(page, t + 2);
        page = page_of(t + 3);
        fetch_k(later, buf);
        fetch_v(rows, buf ^ 1);
        stage_k(buf);
        stage_v(t + 1, buf ^ 1);
        rows = later;
      }
    }
    __syncthreads();
    if (lds_special) {
#pragma unroll 1
      for (int32_t tt = t_begin; tt < t_end; ++tt) {
        const int32_t j0 = kt.tile(tt) * BN;
        if (all_see(j0, j0 + BN, p_lo, p_hi, n, a.window, a.sinks)) continue;
        const int64_t tile_row = row_of(page_of(tt), tt);
#pragma unroll 1
        for (int key = 0; key < BN; ++key) {
          if (!kt.some(j0 + key)) continue;
          const int64_t r = WHOLE ? tile_row + key : shfl64(tile_row, key);
#pragma unroll
          for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float v = v_element<F, D>(a.pool, r, 32 * db + 8 * (i / 4) + 4 * h + i % 4);
              if (!(fabsf(v) < INFINITY) & sees(j0 + key, pos, n, a.window, a.sinks)) o[db][i] += v;
            }
        }
      }
    }
  }
  if (__ballot(bad) != 0 && lane == 0) atomicOr(a.err, kDevBadPage);

  {
    const int rr = wave * 32 + l32, r = r0 + rr;
    const float sum = lanes_sum<2>(l);
    if (r >= R) return;
    if (st.splits > 1) {
      float* at = a.part + ((int64_t)pl.slot * BM + rr) * D;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<F32x4*>(at + 32 * db + 8 * i + 4 * h) =
              F32x4{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]};
      if (h == 0) {
        float* ml = a.part_ml + ((int64_t)pl.slot * BM + rr) * 2;
        ml[0] = m, ml[1] = sum;
      }
    } else {
      const int head = pl.h * a.G + r - tok * a.G;  // (r is qr here)
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      char* at = a.out + 2 * ((int64_t)b * a.o_b + (int64_t)head * a.o_h + (int64_t)tok * a.o_m);
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<U32x2*>(at + 2 * (32 * db + 8 * i + 4 * h)) =
              U32x2{pack_bf16(o[db][4 * i] * inv, o[db][4 * i + 1] * inv),
                    pack_bf16(o[db][4 * i + 2] * inv, o[db][4 * i + 3] * inv)};
      if (h == 0 && a.lse)
        a.lse[((int64_t)b * (a.H * a.G) + head) * a.max_rows + tok] = sum == 0.f ? -INFINITY : (m + log2_hw(sum)) * kLn2;
    }
  }
}

// ---------------------------------------------------------------- fp32 pools
// Row tiles of 32 rows; the four waves share the keys, 32 at a time, with the fp32
// matrix instruction. It has a sixteenth of the bf16 one's rate, so rows are read
// straight from the caches into its operands, without LDS. Its operands take one
// element a lane: half h of the wave holds the elements 8 k + 4 h + i of a key, so that a
// load reads 32 bytes of each row, and a row's lines stay in the first cache until they
// are used up (halves of a row instead: 819 -> 860 us for 1600 tokens of 64 heads of 64 over
// 4096 positions). S^T leaves the weights as the second product's operand as they stand.
// Chunks are bound by that instruction, single tokens by the cache's bytes: 512 tokens of 64 heads over
// 4096 positions of 8, D = 128, 548 us, 117 TFLOP/s (the library's product of such sizes: 154), 106
// for D = 64, 112 for 256; one token of 8 streams over 32768 positions 370 us, 5.8 TB/s.
template <int D, bool WHOLE>
__global__ __launch_bounds__(64 * kFewWaves, D <= 64 ? 2 : 1) void k_attend_f32(AttendArgs a) {
  constexpr int BN = 32;
  __shared__ __attribute__((aligned(16))) char lds[kFewWaves][JoinLds<D, 32>::kWaveBytes];
  __shared__ float lds_ml[kFewWaves][32][2];
  __shared__ uint32_t lds_last;
  const Place pl = place_of(a);
  if (pl.slot < 0) return;
  const AttendStream st = a.s[pl.b];
  const int lane = threadIdx.x % kWave, h = lane / 32, l32 = lane % 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int32_t n = st.n, R = st.rows * a.G, r0 = pl.tile * 32;
  const int b = a.b0 + pl.b;
  const int64_t head_row = a.layer_row + (int64_t)pl.h * a.pool.T.d;
  const int32_t p_lo = st.first + (int32_t)fast_div((uint32_t)r0, a.G_div);
  const int32_t p_hi = st.first + (int32_t)fast_div((uint32_t)(min(r0 + 32, R) - 1), a.G_div);
  const KeyTiles kt(n, p_lo, p_hi, a.window, a.sinks, BN);
  const int32_t t_end = (int32_t)((int64_t)kt.count * (pl.split + 1) / st.splits);
  const int32_t t_begin = (int32_t)((int64_t)kt.count * pl.split / st.splits) + wave;
  const int32_t r = min(r0 + l32, R - 1), tok = (int32_t)fast_div((uint32_t)r, a.G_div), pos = st.first + tok;
  float q[D / 2];
  const char* qa = a.q + 4 * ((int64_t)b * a.q_b + (int64_t)(pl.h * a.G + r - tok * a.G) * a.q_h + (int64_t)tok * a.q_m + 4 * h);
#pragma unroll
  for (int k = 0; k < D / 2; k += 4) {
    const F32x4 v = *reinterpret_cast<const F32x4*>(qa + 8 * k);
    q[k] = v.x, q[k + 1] = v.y, q[k + 2] = v.z, q[k + 3] = v.w;
  }
  F32x16 o[D / 32];
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = F32x16{};
  bool bad = false, special = false;
  auto row_of = [&](int32_t t) __attribute__((always_inline)) {  // the pool's row of the tile's key l32 (WHOLE: its first)
    bool x;
    const int32_t j = min(kt.tile(min(t, kt.count - 1)) * BN + (WHOLE ? 0 : l32), n - 1);
    const int32_t page = WHOLE ? pool_page_uniform(a.pool, b, (uint32_t)j) : pool_page(a.pool, b, (uint32_t)j);
    const int64_t at = pool_row(a.pool, page, (uint32_t)j, &x) + head_row;
    bad |= x & (WHOLE | kt.some(j));
    return at;
  };
  // K in pieces of four elements, KA of them in registers: all of a row's up to D = 128. With one
  // wave a SIMD (D > 64) the next tile's are on their way while V is used: 512 tokens of 64 heads
  // over 4096 positions of 8, D = 128, take 549 us with that and 648 without. Where two share it
  // they cover for each other, and loads ahead only hold them up: 320 us with it and 297 without, D = 64.
  constexpr bool AHEAD = D > 64;
  using At = std::conditional_t<WHOLE, uint32_t, int64_t>;
  constexpr int KA = D <= 128 ? D / 8 : 8;
  F32x4 kx[KA];
  const auto load_k = [&](int64_t row, int k) __attribute__((always_inline)) {
    const char* base = a.pool.K + (WHOLE ? row * D * 4 : 0);
    kx[k % KA] = *reinterpret_cast<const F32x4*>(base + 32 * k + (At)((WHOLE ? (At)l32 : (At)row) * D * 4 + 16 * h));
  };
  // V's rows (all of them up to D = 128, else four keys ahead) are on their way while the
  // scores are computed
  constexpr int VA = D <= 128 ? 16 : 4;
  float vx[VA][D / 32];
  int64_t row = 0;
  if (t_begin < t_end) {
    row = row_of(t_begin);
    if constexpr (AHEAD)
#pragma unroll
      for (int k = 0; k < KA; ++k) load_k(row, k);
  }
  for (int32_t t = t_begin; t < t_end; t += kFewWaves) {
    const int32_t j0 = kt.tile(t) * BN;
    const int64_t next = row_of(t + kFewWaves);
    if constexpr (!AHEAD)
#pragma unroll
      for (int k = 0; k < KA; ++k) load_k(row, k);
    const bool full = all_see(j0, j0 + BN, p_lo, p_hi, n, a.window, a.sinks);
    const auto load_v = [&](int i) __attribute__((always_inline)) {
      const int key = 8 * (i / 4) + i % 4;  // (+ 4 h)
      const char* base = a.pool.V + (WHOLE ? (row + key) * D * 4 : 0);
      const At at = WHOLE ? (At)(4 * h * D * 4) : (At)(shfl64(row, key + 4 * h) * D * 4);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) vx[i % VA][db] = *reinterpret_cast<const float*>(base + 128 * db + (At)(at + 4 * l32));
    };
#pragma unroll
    for (int i = 0; i < VA; ++i) load_v(i);
    if constexpr (AHEAD) __builtin_amdgcn_sched_barrier(0);
    F32x16 s = {};
#pragma unroll
    for (int k = 0; k < D / 8; ++k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kx[k % KA][i], q[4 * k + i], s, 0, 0, 0);
      if (k + KA < D / 8) load_k(row, k + KA);
    }
    if constexpr (AHEAD) __builtin_amdgcn_sched_barrier(0);
    if (AHEAD && t + kFewWaves < t_end) {
#pragma unroll
      for (int k = 0; k < KA; ++k) load_k(next, k);
    }
    if constexpr (AHEAD) __builtin_amdgcn_sched_barrier(0);
    if (!full) {
      const Limits in(j0 + 4 * h, pos, n, a.window, a.sinks);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!in(8 * (i / 4) + i % 4)) s[i] = -INFINITY;
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
      if (!full) {  // as in the other kernels: nothing of rows that nobody sees, infinities and NaN at the end
        const bool some = kt.some(j0 + 8 * (i / 4) + 4 * h + i % 4);
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          if (!some) v[db] = 0.f;
          if (!(fabsf(v[db]) < INFINITY)) v[db] = 0.f, special = true;
        }
      }
#pragma unroll
      for (int db = 0; db < D / 32; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[db], e, o[db], 0, 0, 0);
      if (i + VA < 16) load_v(i + VA);
    }
    row = next;
  }
  if (__ballot(special) != 0) {
#pragma unroll 1
    for (int32_t t = t_begin; t < t_end; t += kFewWaves) {
      const int32_t j0 = kt.tile(t) * BN;
      if (all_see(j0, j0 + BN, p_lo, p_hi, n, a.window, a.sinks)) continue;
      const int64_t row = row_of(t);
#pragma unroll 1
      for (int key = 0; key < BN; ++key) {
        const int64_t rv = WHOLE ? row + key : shfl64(row, key);
        if (!kt.some(j0 + key)) continue;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float v = reinterpret_cast<const float*>(a.pool.V)[rv * D + 32 * db + 8 * (i / 4) + 4 * h + i % 4];
            if (!(fabsf(v) < INFINITY) & sees(j0 + key, pos, n, a.window, a.sinks)) o[db][i] += v;
          }
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
  join_parts<D, 32, true>(a, st, pl, b, r0, min(R - r0, 32), lds, lds_ml, &lds_last);
}

// ---------------------------------------------------------------- joining parts by a launch
// One wave a row: lane s has split s's maximum and sum, then every lane a part
// of the row's elements over the splits in order. Bound by the parts' bytes, which come from
// other XCDs: 28 heads of 196 rows of 128 in 10 parts (28 MB) 7.5 us, 3.8 TB/s.
template <int D, bool F32OUT>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, int32_t BM) {
  const AttendStream st = a.s[blockIdx.y];
  if (st.splits <= 1) return;
  const int lane = threadIdx.x % kWave;
  const uint32_t R = (uint32_t)(st.rows * a.G), x = blockIdx.x * 4 + threadIdx.x / kWave;
  if (x >= R * (uint32_t)a.H) return;
  const int32_t h = (int32_t)(x / R), r = (int32_t)(x % R), tile = r / BM, rr = r % BM;
  // places run over the splits, the tiles from the last, the heads
  const int64_t slot = st.start + ((int64_t)h * st.tiles + (st.tiles - 1 - tile)) * st.splits;
  // the row's elements of 16 parts at a time, the first ones on their way while the weights are made
  constexpr int E = D >= 64 ? D / 64 : 1, ROUND = 16;
  typedef float Part __attribute__((ext_vector_type(E)));
  const float* p = a.part + (slot * BM + rr) * D + (lane * E) % D;
  Part y[ROUND];
  const auto load_round = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < ROUND; ++k)  // the last again past the last, with no weight
      y[k] = *reinterpret_cast<const Part*>(p + (int64_t)min(s0 + k, st.splits - 1) * BM * D);
  };
  load_round(0);
  const float* ml = a.part_ml + (slot * BM + rr) * 2;
  float m = -INFINITY, l = 0.f;
  if (lane < st.splits) m = ml[(int64_t)lane * BM * 2], l = ml[(int64_t)lane * BM * 2 + 1];
  const float top = wave_max(m), w = exp2_hw(m - shift_of(top)), sum = wave_sum(l * w);
  Part v = 0.f;
  for (int s0 = 0;;) {
#pragma unroll
    for (int k = 0; k < ROUND; ++k) {
      const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), min(s0 + k, kWave - 1)));
      if (s0 + k < st.splits) v += y[k] * f;
    }
    s0 += ROUND;
    if (s0 >= st.splits) break;
    load_round(s0);
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int32_t tok = (int32_t)fast_div((uint32_t)r, a.G_div), head = h * a.G + r - tok * a.G;
  const int64_t b = a.b0 + blockIdx.y, at = b * a.o_b + (int64_t)head * a.o_h + (int64_t)tok * a.o_m + lane * E;
  if (lane * E < D) {
#pragma unroll
    for (int e = 0; e < E; ++e) {  // (one store)
      if constexpr (F32OUT) reinterpret_cast<float*>(a.out)[at + e] = v[e] * inv;
      else reinterpret_cast<__bf16*>(a.out)[at + e] = (__bf16)(v[e] * inv);
    }
  }
  if (lane == 0 && a.lse)
    a.lse[(b * (a.H * a.G) + head) * a.max_rows + tok] = sum == 0.f ? -INFINITY : (top + log2_hw(sum)) * kLn2;
}

// ---------------------------------------------------------------- launches
// What a format's translation unit offers: the kernel for `shape` rows.
enum AttendKind { kFew1, kFew2, kTile, kF32 };
template <int F>
hipError_t launch_attend(int D, AttendKind kind, uint32_t grid, const AttendArgs& a, hipStream_t st);
inline int attend_rows(AttendKind k, int D) { return k == kFew1 ? 16 : k == kFew2 || k == kF32 ? 32 : 32 * tile_waves(D); }
inline int attend_threads(AttendKind k, int D) { return 64 * (k == kTile ? tile_waves(D) : kFewWaves); }
inline int attend_keys(AttendKind k) { return k == kTile ? kTileKeys : 32; }

}  // namespace ipv
