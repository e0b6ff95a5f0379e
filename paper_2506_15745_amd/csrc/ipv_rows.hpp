// Rows of a paged cache beyond plain writes and reads: new tokens' queries, keys and values
// normed, rotated and written in one pass; bounds of blocks of keys; kept rows into
// new pages; pages onto pages.
#pragma once

#include "ipv_pages.hpp"

namespace ipv {

constexpr uint32_t kDevBadKeep = 8u;
constexpr int kTokenHeads = 4;  // heads of queries (or of keys, of values) that a thread takes, at one position

// ------------------------------------------------------------ bounds of a block's keys
// The lowest and highest element of each channel. Elements are compared as whole numbers:
// a bf16 or fp32 whose lower bits are inverted where its sign is set is in that order (with
// -0 below +0, and NaN beyond the infinity of its sign), two bf16 at a time.
typedef short S16x2 __attribute__((ext_vector_type(2)));

template <int F>
constexpr int kWords = F == kFmtF32 ? 8 : 4;  // words of eight elements as bf16, or as fp32

template <int F>
__device__ __forceinline__ uint32_t ordered(uint32_t w) {  // (its own inverse)
  if constexpr (F == kFmtF32) {
    const int32_t x = (int32_t)w;
    return (uint32_t)(x ^ ((x >> 31) & 0x7fffffff));
  } else {
    const S16x2 x = __builtin_bit_cast(S16x2, w);
    return __builtin_bit_cast(uint32_t, (S16x2)(x ^ ((x >> (short)15) & (short)0x7fff)));
  }
}
template <int F>
__device__ __forceinline__ uint32_t lower(uint32_t a, uint32_t b) {
  if constexpr (F == kFmtF32) return (uint32_t)min((int32_t)a, (int32_t)b);
  else return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(S16x2, a), __builtin_bit_cast(S16x2, b)));
}
template <int F>
__device__ __forceinline__ uint32_t higher(uint32_t a, uint32_t b) {
  if constexpr (F == kFmtF32) return (uint32_t)max((int32_t)a, (int32_t)b);
  else return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(S16x2, a), __builtin_bit_cast(S16x2, b)));
}

// Eight elements of a stored row as bf16 (exact) or fp32.
template <int F, int D>
__device__ __forceinline__ void stored8(const char* pages, const uint8_t* scales, int64_t row, int d, uint32_t (&w)[kWords<F>]) {
  const char* at = pages + row * fmt_row_bytes(F, D);
  if constexpr (F == kFmtF32) {
    const Raw16 a = load16(at + 4 * d), b = load16(at + 4 * d + 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = a.w[i], w[4 + i] = b.w[i];
  } else {
    Raw16 r;
    if constexpr (F == kFmtBf16) {
      r = load16(at + 2 * d);
    } else {
      const float scale = scale_of(scales[row * (D / kScaleBlock) + d / kScaleBlock]);
      if constexpr (F == kFmtFp8) {
        const U32x2 x = *reinterpret_cast<const U32x2*>(at + d);
        r = fp8_to_bf16(x.x, x.y, scale);
      } else {
        r = fp4_to_bf16(*reinterpret_cast<const uint32_t*>(at + d / 2), scale);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = r.w[i];
  }
}

// The bounds of a block of keys, built by a workgroup: a thread has eight channels of either half of
// the rows that it adds, as the threads of RowSplit have them.
template <int F, int D>
struct Bounds {
  static constexpr int W = kWords<F>, kLds = (kPageThreads / kWave) * 2 * D / 8 * W;  // words of LDS
  uint32_t lo[2][W], hi[2][W];

  __device__ __forceinline__ Bounds() {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < W; ++i) {
        lo[s][i] = F == kFmtF32 ? 0x7fffffffu : 0x7fff7fffu;
        hi[s][i] = ~lo[s][i];
      }
  }
  __device__ __forceinline__ void add(const uint32_t (&first)[W], const uint32_t (&second)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const uint32_t a = ordered<F>(first[i]), b = ordered<F>(second[i]);
      lo[0][i] = lower<F>(lo[0][i], a), hi[0][i] = higher<F>(hi[0][i], a);
      lo[1][i] = lower<F>(lo[1][i], b), hi[1][i] = higher<F>(hi[1][i], b);
    }
  }
  // A row just put into the pool: as it is stored.
  __device__ __forceinline__ void add_put(const float (&fl)[8], const float (&fh)[8], const uint32_t (&wl)[2], const uint32_t (&wh)[2],
                                          uint32_t el, uint32_t eh) {
    uint32_t a[W], b[W];
    if constexpr (F == kFmtF32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = __float_as_uint(fl[i]), b[i] = __float_as_uint(fh[i]);
    } else {
      Raw16 x, y;
      if constexpr (F == kFmtBf16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x.w[i] = pack_bf16(fl[2 * i], fl[2 * i + 1]), y.w[i] = pack_bf16(fh[2 * i], fh[2 * i + 1]);
      } else if constexpr (F == kFmtFp8) {
        x = fp8_to_bf16(wl[0], wl[1], scale_of(el)), y = fp8_to_bf16(wh[0], wh[1], scale_of(eh));
      } else {
        x = fp4_to_bf16(wl[0], scale_of(el)), y = fp4_to_bf16(wh[0], scale_of(eh));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = x.w[i], b[i] = y.w[i];
    }
    add(a, b);
  }
  template <int CTRL>
  __device__ __forceinline__ void with_lane() {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < W; ++i) {
        lo[s][i] = lower<F>(lo[s][i], dpp_u32<CTRL>(lo[s][i]));
        hi[s][i] = higher<F>(hi[s][i], dpp_u32<CTRL>(hi[s][i]));
      }
  }
  // Over the wave's rows, in all of its lanes.
  __device__ __forceinline__ void over_wave() {
    constexpr int RT = RowSplit<D>::kThreads;
    // within rows of 16 lanes the lanes RT apart hold the same channels: rotations by RT, 2 RT, .. 8
    if constexpr (RT <= 2) with_lane<0x122>();
    if constexpr (RT <= 4) with_lane<0x124>();
    if constexpr (RT <= 8) with_lane<0x128>();
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < W; ++i) {
        auto a = __builtin_amdgcn_permlane16_swap(lo[s][i], lo[s][i], false, false);
        uint32_t l = lower<F>(a[0], a[1]);
        a = __builtin_amdgcn_permlane32_swap(l, l, false, false);
        lo[s][i] = lower<F>(a[0], a[1]);
        a = __builtin_amdgcn_permlane16_swap(hi[s][i], hi[s][i], false, false);
        uint32_t h = higher<F>(a[0], a[1]);
        a = __builtin_amdgcn_permlane32_swap(h, h, false, false);
        hi[s][i] = higher<F>(a[0], a[1]);
      }
  }
  // The bounds of a wave's rows to `at`.
  __device__ __forceinline__ void store_wave(char* at) {
    over_wave();
    const int lane = threadIdx.x % kWave;
    if (lane >= RowSplit<D>::kThreads) return;
    U32x4* to = reinterpret_cast<U32x4*>(at);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < W; i += 4) {
        const int piece = (s * (D / 16) + lane) * (W / 4) + i / 4;
        U32x4 l, h;
#pragma unroll
        for (int e = 0; e < 4; ++e) l[e] = ordered<F>(lo[s][i + e]), h[e] = ordered<F>(hi[s][i + e]);
        to[piece] = l, to[D / 8 * (W / 4) + piece] = h;
      }
  }
  // All threads of the workgroup: the bounds of its rows to `at`.
  __device__ __forceinline__ void store(char* at, uint32_t* lds) {
    constexpr int RT = RowSplit<D>::kThreads;
    over_wave();
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    U32x4* to = reinterpret_cast<U32x4*>(lds);  // [wave][lo, hi][piece of eight channels][W]
    if (lane < RT) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < W; i += 4) {
          const int piece = s * (D / 16) + lane;
          to[((wave * 2 + 0) * (D / 8) + piece) * (W / 4) + i / 4] = U32x4{lo[s][i], lo[s][i + 1], lo[s][i + 2], lo[s][i + 3]};
          to[((wave * 2 + 1) * (D / 8) + piece) * (W / 4) + i / 4] = U32x4{hi[s][i], hi[s][i + 1], hi[s][i + 2], hi[s][i + 3]};
        }
    }
    __syncthreads();
    const int x = threadIdx.x;  // a piece of four words: of lo first, then of hi, as they lie in memory
    constexpr int PIECES = D / 8 * (W / 4);
    if (x < 2 * PIECES) {
      U32x4 v = to[x];
#pragma unroll
      for (int w = 1; w < kPageThreads / kWave; ++w) {
        const U32x4 y = to[w * 2 * PIECES + x];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = x < PIECES ? lower<F>(v[i], y[i]) : higher<F>(v[i], y[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = ordered<F>(v[i]);
      reinterpret_cast<U32x4*>(at)[x] = v;
    }
  }
};

// Bytes of a block's bounds.
constexpr int bound_bytes(int F, int D) { return 2 * D * (F == kFmtF32 ? 4 : 2); }

// ------------------------------------------------------------ angles of a wave's rows
// The cosines and sines of a position lie in 4 D bytes, of which a thread of RowSplit needs 64. Loaded so by each, four
// neighbouring lanes ask for four lines at a time, and the cache takes them one after the other; so the wave
// loads its rows' angles in the order of memory and spreads them through LDS.
template <int D>
struct Angles {
  static constexpr int PIECES = D / 4, LOADS = 4, LDS = LOADS * kWave * 16;  // 16-byte pieces of a position; bytes of LDS a wave
  F32x4 piece[LOADS];
  // pos(r): the position of the wave's row r (of kWave / RowSplit<D>::kThreads)
  template <class POS>
  __device__ __forceinline__ void load(const float* table, const POS& pos) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int x = i * kWave + threadIdx.x % kWave;
      piece[i] = *reinterpret_cast<const F32x4*>(table + (int64_t)pos(x / PIECES) * D + x % PIECES * 4);
    }
  }
  // The thread's eight pairs. A piece's place: those that neighbouring lanes read together lie in different banks.
  __device__ __forceinline__ void spread(char* lds, float (&c)[8], float (&s)[8]) const {
    const int lane = threadIdx.x % kWave;
    F32x4* at = reinterpret_cast<F32x4*>(lds);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int x = i * kWave + lane;
      at[x ^ (x / 4 % 4)] = piece[i];
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const F32x4 v = at[lane * 4 + (i ^ lane % 4)];
      c[2 * i] = v.x, s[2 * i] = v.y, c[2 * i + 1] = v.z, s[2 * i + 1] = v.w;
    }
    __builtin_amdgcn_wave_barrier();
  }
};

// ------------------------------------------------------------ new tokens
struct TokenCall {
  Pool pool;
  const char* q;
  const char* k;
  const char* v;
  char* q_out;
  char* bounds;
  int64_t q_b, q_h, q_m, k_b, k_h, k_m, o_b, o_h, o_m;  // strides, elements
  const float* q_norm;
  const float* k_norm;
  const float* rotary;
  double eps;
  uint32_t* err;
  int32_t b0, A, H, layer;
  int32_t q_groups, v_groups;  // workgroups' heads: of queries, of values, then of keys
  BlockMap map;                // (with bounds)
  int32_t first[kPageStreams], rows[kPageStreams];
};

// x * s * norm, s = 1 / sqrt(mean x^2 + eps). The mean is in 64 bits, so that s is the same fp32 number
// whatever the order of the sum: rows are rounded to few bits next, where a last bit of 32 decides now and then.
template <int D>
__device__ __forceinline__ void normed(float (&lo)[8], float (&hi)[8], const float (&wl)[8], const float (&wh)[8], double eps) {
  double sum = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    sum = __builtin_fma((double)lo[i], (double)lo[i], sum);
    sum = __builtin_fma((double)hi[i], (double)hi[i], sum);
  }
  const float s = (float)rsqrt(group_sum64<RowSplit<D>::kThreads>(sum) * (1.0 / D) + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) {  // (products alone: nothing that could be contracted)
    lo[i] = lo[i] * s, hi[i] = hi[i] * s;
    lo[i] = lo[i] * wl[i], hi[i] = hi[i] * wh[i];
  }
}

__device__ __forceinline__ void load_norm(const float* norm, int d, int half, float (&wl)[8], float (&wh)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) wl[i] = norm[d + i], wh[i] = norm[half + d + i];
}

// blockIdx.z: stream; .y: heads, kTokenHeads of the queries, then of the values, then of the keys (with
// bounds one head of those); .x: positions (with bounds, of the keys: a block that has new rows, whose
// older rows are read for its bounds). Bound by the rows' bytes: 6272 tokens of 64 heads and 8 KV heads of 128
// with bounds, 260 MB, in 55 to 58 us (4.5 to 4.7 TB/s); one token of 16 streams of 28 and 4 heads 4.9 to 5.7 us, the way to
// the older rows and back; 196 tokens of 4 streams in e4m3 7.4, of whose five waves a CU 60% of the cycles are waits for memory.
template <int F, int SRC, int D>
__global__ __launch_bounds__(kPageThreads) void k_qkv_write(TokenCall c) {
  using S = RowSplit<D>;
  constexpr int QF = F == kFmtF32 ? kFmtF32 : kFmtBf16;
  __shared__ __attribute__((aligned(16))) uint32_t lds[Bounds<F, D>::kLds];
  const int b = blockIdx.z, rows = c.rows[b], first = c.first[b], slot = threadIdx.x / S::kThreads;
  if (rows == 0) return;
  const int d = (int)(threadIdx.x % S::kThreads) * 8;
  const int y = blockIdx.y;
  const bool isq = y < c.q_groups, isv = !isq && y < c.q_groups + c.v_groups;
  const float* norm = isq ? c.q_norm : isv ? nullptr : c.k_norm;
  const bool rot = !isv && c.rotary != nullptr;
  float wl[8], wh[8], cs[8], sn[8];
  if (norm) load_norm(norm, d, D / 2, wl, wh);

  if (!isq && !isv && c.bounds) {
    const int h = y - c.q_groups - c.v_groups;
    const uint32_t j = fast_div((uint32_t)first, c.map.R) + blockIdx.x;
    const int64_t p0 = (int64_t)j * c.map.R.d, end = (int64_t)first + rows;
    if (p0 >= end) return;  // the whole workgroup
    const int32_t held = (int32_t)(min(p0 + (int64_t)c.map.R.d, end) - p0);
    bool bad;
    const int32_t page = pool_page(c.pool, c.b0 + b, (uint32_t)p0);
    const uint32_t slice = (uint32_t)(c.layer * c.H + h);
    const int64_t row0 = pool_row(c.pool, page, (uint32_t)p0, &bad) + (int64_t)slice * c.pool.T.d;
    if (bad) {
      if (threadIdx.x == 0) atomicOr(c.err, kDevBadPage);
      return;
    }
    Bounds<F, D> got;
    const int64_t src0 = (int64_t)(c.b0 + b) * c.k_b + (int64_t)h * c.k_h + d;
    for (int r = slot; r < held; r += S::kRows) {
      const int i = (int)(p0 - first) + r;  // (of the new rows)
      if (i < 0) {
        uint32_t x[kWords<F>], z[kWords<F>];
        stored8<F, D>(c.pool.K, c.pool.Ks, row0 + r, d, x);
        stored8<F, D>(c.pool.K, c.pool.Ks, row0 + r, D / 2 + d, z);
        got.add(x, z);
      } else {
        float lo[8], hi[8];
        load_row8<SRC>(c.k, src0 + (int64_t)i * c.k_m, lo);
        load_row8<SRC>(c.k, src0 + (int64_t)i * c.k_m + D / 2, hi);
        if (rot) load_angles(c.rotary, p0 + r, D / 2, d, cs, sn);
        if (norm) normed<D>(lo, hi, wl, wh, c.eps);
        if (rot) turn(lo, hi, cs, sn, false);
        uint32_t el, eh, xl[2], xh[2];
        put_row<F, D>(c.pool.K, c.pool.Ks, row0 + r, d, lo, hi, c.err, xl, xh, el, eh);
        got.add_put(lo, hi, xl, xh, el, eh);
      }
    }
    got.store(c.bounds + c.map.block(page, slice, (uint32_t)p0, c.pool.T) * bound_bytes(F, D), lds);
    return;
  }

  const int i = (int)(blockIdx.x * S::kRows) + slot;
  if (i >= rows) return;  // whole rows' threads leave together
  const int64_t pos = (int64_t)first + i;
  const int g = isq ? y : isv ? y - c.q_groups : y - c.q_groups - c.v_groups, heads = isq ? c.A : c.H;
  int64_t row0 = 0;
  if (!isq) {
    bool bad;
    row0 = pool_row(c.pool, pool_page(c.pool, c.b0 + b, (uint32_t)pos), (uint32_t)pos, &bad) + (int64_t)c.layer * c.pool.layer_rows;
    if (bad) {
      if (d == 0) atomicOr(c.err, kDevBadPage);
      return;
    }
  }
  if (rot) load_angles(c.rotary, pos, D / 2, d, cs, sn);
  const char* src = isq ? c.q : isv ? c.v : c.k;
  const int64_t sh = isq ? c.q_h : c.k_h;
  const int64_t src0 = (int64_t)(c.b0 + b) * (isq ? c.q_b : c.k_b) + (int64_t)i * (isq ? c.q_m : c.k_m) + d;
  float lo[kTokenHeads][8], hi[kTokenHeads][8];
#pragma unroll
  for (int u = 0; u < kTokenHeads; ++u) {
    const int64_t at = src0 + (int64_t)min(g * kTokenHeads + u, heads - 1) * sh;
    load_row8<SRC>(src, at, lo[u]);
    load_row8<SRC>(src, at + D / 2, hi[u]);
  }
#pragma unroll
  for (int u = 0; u < kTokenHeads; ++u) {
    const int h = g * kTokenHeads + u;
    if (h >= heads) break;
    if (norm) normed<D>(lo[u], hi[u], wl, wh, c.eps);
    if (rot) turn(lo[u], hi[u], cs, sn, false);
    if (isq) {
      const int64_t at = (int64_t)(c.b0 + b) * c.o_b + (int64_t)h * c.o_h + (int64_t)i * c.o_m + d;
      // past the caches: the next kernel reads it on other XCDs (6272 tokens of 64 heads 58.3 us through them, 54.8 so)
      store_row8<QF, true>(c.q_out, at, lo[u]);
      store_row8<QF, true>(c.q_out, at + D / 2, hi[u]);
    } else {
      uint32_t el, eh, xl[2], xh[2];
      put_row<F, D>(isv ? c.pool.V : c.pool.K, isv ? c.pool.Vs : c.pool.Ks, row0 + (int64_t)h * c.pool.T.d, d, lo[u], hi[u], c.err,
                    xl, xh, el, eh);
    }
  }
}

// ------------------------------------------------------------ bounds of blocks as they stand
struct BoundsCall {
  Pool pool;
  char* bounds;
  uint32_t* err;
  int32_t b0;
  uint32_t first_slice;
  BlockMap map;
  int32_t first[kPageStreams], rows[kPageStreams];
};

// blockIdx.x: a block that holds one of the positions; .y: slice; .z: stream. Bound by the keys' bytes: 6272 rows of 28
// layers of 4 heads of 128 take 73 us in fp32 (371 MB, 5.1 TB/s), 28 in bf16; in e2m1 25, for whose unpacking and comparing
// the vector unit is busy throughout.
template <int F, int D>
__global__ __launch_bounds__(kPageThreads) void k_block_bounds(BoundsCall c) {
  using S = RowSplit<D>;
  __shared__ __attribute__((aligned(16))) uint32_t lds[Bounds<F, D>::kLds];
  const int b = blockIdx.z, d = (int)(threadIdx.x % S::kThreads) * 8;
  const int64_t p0 = ((int64_t)fast_div((uint32_t)c.first[b], c.map.R) + blockIdx.x) * c.map.R.d;
  const int64_t end = (int64_t)c.first[b] + c.rows[b];
  if (c.rows[b] == 0 || p0 >= end) return;
  const int32_t held = (int32_t)(min(p0 + (int64_t)c.map.R.d, end) - p0);
  const int32_t page = pool_page(c.pool, c.b0 + b, (uint32_t)p0);
  const uint32_t slice = c.first_slice + blockIdx.y;
  bool bad;
  const int64_t row0 = pool_row(c.pool, page, (uint32_t)p0, &bad) + (int64_t)slice * c.pool.T.d;
  if (bad) {
    if (threadIdx.x == 0) atomicOr(c.err, kDevBadPage);
    return;
  }
  Bounds<F, D> got;
  for (int r = threadIdx.x / S::kThreads; r < held; r += S::kRows) {
    uint32_t x[kWords<F>], z[kWords<F>];
    stored8<F, D>(c.pool.K, c.pool.Ks, row0 + r, d, x);
    stored8<F, D>(c.pool.K, c.pool.Ks, row0 + r, D / 2 + d, z);
    got.add(x, z);
  }
  got.store(c.bounds + c.map.block(page, slice, (uint32_t)p0, c.pool.T) * bound_bytes(F, D), lds);
}

// ------------------------------------------------------------ kept rows into new pages
struct CompactCall {
  Pool pool;  // with the table of the old pages
  char* bounds;
  const int32_t* new_table;
  const int32_t* keep;
  const float* rotary;
  uint32_t* err;
  int32_t b0, new_cols, C;
  BlockMap map;  // (the slices also without bounds)
  int32_t n[kPageStreams], rows[kPageStreams];
};
constexpr int kCompactWaves = kPageThreads / kWave;

// Rows that a wave takes: whole blocks where it makes their bounds.
__host__ __device__ inline int64_t compact_run(bool bounds, uint32_t R) { return !bounds ? 32 : R >= 64 ? R : 64 / R * R; }

// blockIdx.x: a run of rows of the new pages; .y: four slices, of K or of V, a wave each (side by side, so that the
// workgroups at work at one time write neighbouring rows); .z: stream. A wave looks up its next 64 rows at once, a row a
// lane (their places take two trips, to keep_idx and to the table); a block's bounds stay in the wave. Values, and keys that
// neither turn nor have bounds, are copied four steps at a time. Bound by the rows' bytes: 3136 rows of 28 layers of 4 heads
// of 128, 367 MB, take 87 us with turned keys and bounds (4.2 TB/s), 78 without bounds, 70 copied.
template <int F, int D, bool TURN, bool BOUNDS>
__global__ __launch_bounds__(kPageThreads) void k_page_compact(CompactCall c) {
  constexpr int W = kWords<F>, RB = fmt_row_bytes(F, D), RT = RowSplit<D>::kThreads, PIECE = RB / RT / 2;  // stored bytes of eight elements
  constexpr int ROWS = kWave / RT;  // of a step
  __shared__ __attribute__((aligned(16))) char lds_angles[kCompactWaves][Angles<D>::LDS];
  const int b = blockIdx.z, lane = threadIdx.x % kWave, thread = lane % RT, d = thread * 8;
  const uint32_t slice = (blockIdx.y >> 1) * kCompactWaves + threadIdx.x / kWave;
  if (slice >= (uint32_t)c.map.slices) return;  // the whole wave
  const bool isv = blockIdx.y & 1, block = BOUNDS && !isv;
  const int64_t run = compact_run(block, c.map.R.d);
  const int64_t begin = (int64_t)blockIdx.x * run;
  const int64_t end = min(begin + run, (int64_t)c.rows[b]);
  if (begin >= end) return;  // the whole wave
  char* pages = isv ? c.pool.V : c.pool.K;
  uint8_t* scales = isv ? c.pool.Vs : c.pool.Ks;
  const int64_t slice_row = (int64_t)slice * c.pool.T.d;
  const int32_t* keep = c.keep + ((int64_t)(c.b0 + b) * c.map.slices + slice) * c.C;
  const int32_t* table = c.new_table + (int64_t)(c.b0 + b) * c.new_cols;
  const int32_t n = c.n[b];
  // rows of a step: they lie in one block
  const int step = block && c.map.R.d % ROWS != 0 ? 16 : ROWS;
  // what is stored of a row, eight elements of either half, and the row's scales
  struct Stored {
    uint32_t w[2][PIECE / 4];
    uint64_t scales;
  };
  uint32_t errors = 0;
  Bounds<F, D> got;
  for (int64_t j0 = begin; j0 < end; j0 += kWave) {
    const int held = (int)min(end - j0, (int64_t)min((int64_t)kWave, run));
    int32_t at;          // the lane's row's old position
    int64_t from, to;    // where it was, where it goes (-1: nowhere)
    int32_t new_page;
    {
      const uint32_t j = (uint32_t)(j0 + min(lane, held - 1));
      at = keep[j];
      new_page = table[fast_div(j, c.pool.T)];
      const bool out = (uint32_t)at >= (uint32_t)n;
      if (out) at = 0;
      const uint32_t p = (uint32_t)at;
      bool x, y;
      from = pool_row(c.pool, n > 0 ? pool_page(c.pool, c.b0 + b, p) : 0, p, &x) + slice_row;
      to = pool_row(c.pool, new_page, j, &y) + slice_row;
      if (out) errors |= kDevBadKeep;
      if ((x & !out) | y) errors |= kDevBadPage;
      if (out | x | y) to = -1;
    }
    const auto fetch = [&](int64_t row, Stored& x) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const char* at = pages + row * RB + s * (RB / 2) + thread * PIECE;
        if constexpr (PIECE >= 16) {
#pragma unroll
          for (int i = 0; i < PIECE / 16; ++i) load_piece<16>(at + 16 * i, x.w[s] + 4 * i);
        } else {
          load_piece<PIECE>(at, x.w[s]);
        }
      }
      if constexpr (fmt_scaled(F)) x.scales = load_scales<D>(scales, row);
    };
    const auto store = [&](int64_t row, const Stored& x) __attribute__((always_inline)) {  // past the caches, as it is not read soon
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        char* at = pages + row * RB + s * (RB / 2) + thread * PIECE;
        if constexpr (PIECE >= 16) {
#pragma unroll
          for (int i = 0; i < PIECE / 16; ++i)
            __builtin_nontemporal_store(U32x4{x.w[s][4 * i], x.w[s][4 * i + 1], x.w[s][4 * i + 2], x.w[s][4 * i + 3]},
                                        reinterpret_cast<U32x4*>(at + 16 * i));
        } else if constexpr (PIECE == 8) {
          *reinterpret_cast<U32x2*>(at) = U32x2{x.w[s][0], x.w[s][1]};
        } else {
          *reinterpret_cast<uint32_t*>(at) = x.w[s][0];
        }
      }
      if constexpr (fmt_scaled(F)) {
        if (thread == 0) {
          uint8_t* at = scales + row * (D / kScaleBlock);
          if (D == 32) *at = (uint8_t)x.scales;
          else if (D == 64) *reinterpret_cast<uint16_t*>(at) = (uint16_t)x.scales;
          else if (D == 128) *reinterpret_cast<uint32_t*>(at) = (uint32_t)x.scales;
          else reinterpret_cast<uint32_t*>(at)[0] = (uint32_t)x.scales, reinterpret_cast<uint32_t*>(at)[1] = (uint32_t)(x.scales >> 32);
        }
      }
    };
    if (isv || !(TURN || BOUNDS)) {  // copied: four steps at a time
      constexpr int STEPS = 4;
      for (int r0 = 0; r0 < held; r0 += STEPS * ROWS) {
        Stored x[STEPS];
#pragma unroll
        for (int u = 0; u < STEPS; ++u) fetch(shfl64(from, min(r0 + u * ROWS + lane / RT, held - 1)), x[u]);
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
          const int r = r0 + u * ROWS + lane / RT;
          const int64_t row = shfl64(to, min(r, held - 1));
          if (r < held && row >= 0) store(row, x[u]);
        }
      }
      continue;
    }
    if constexpr (TURN || BOUNDS) for (int r0 = 0; r0 < held; r0 += step) {
      const int r = r0 + lane / RT, own = min(r, held - 1);
      Stored x;
      fetch(shfl64(from, own), x);
      const int64_t row = shfl64(to, own);
      const uint32_t j = (uint32_t)(j0 + r), p = (uint32_t)__shfl(at, own, kWave);
      Angles<D> old, now;
      if constexpr (TURN) {
        old.load(c.rotary, [&](int y) __attribute__((always_inline)) { return __shfl(at, min(r0 + y, held - 1), kWave); });
        now.load(c.rotary, [&](int y) __attribute__((always_inline)) { return j0 + min(r0 + y, held - 1); });
      }
      // as bf16 or fp32
      uint32_t a[W], z[W];
      if constexpr (!fmt_scaled(F)) {
#pragma unroll
        for (int i = 0; i < W; ++i) a[i] = x.w[0][i], z[i] = x.w[1][i];
      } else {
        const float fl = scale_at(x.scales, d / kScaleBlock), fh = scale_at(x.scales, (D / 2 + d) / kScaleBlock);
        const Raw16 u = F == kFmtFp8 ? fp8_to_bf16(x.w[0][0], x.w[0][PIECE / 4 - 1], fl) : fp4_to_bf16(x.w[0][0], fl);
        const Raw16 v = F == kFmtFp8 ? fp8_to_bf16(x.w[1][0], x.w[1][PIECE / 4 - 1], fh) : fp4_to_bf16(x.w[1][0], fh);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = u.w[i], z[i] = v.w[i];
      }
      float lo[8], hi[8];
      if constexpr (TURN) {
        if constexpr (F == kFmtF32) {
#pragma unroll
          for (int i = 0; i < 8; ++i) lo[i] = __uint_as_float(a[i]), hi[i] = __uint_as_float(z[i]);
        } else {
          Lane<uint16_t>::decode(Raw16{a[0], a[1], a[2], a[3]}, lo);
          Lane<uint16_t>::decode(Raw16{z[0], z[1], z[2], z[3]}, hi);
        }
        float cs[8], sn[8];
        old.spread(lds_angles[threadIdx.x / kWave], cs, sn);
        turn(lo, hi, cs, sn, true);
        now.spread(lds_angles[threadIdx.x / kWave], cs, sn);
        turn(lo, hi, cs, sn, false);
      }
      if ((lane / RT < step) & (r < held) & (row >= 0)) {  // (whole rows' threads together)
        if (TURN && p != j) {
          uint32_t el, eh, xl[2], xh[2];
          put_row<F, D, true, true>(pages, scales, row, d, lo, hi, c.err, xl, xh, el, eh);
          if constexpr (BOUNDS) got.add_put(lo, hi, xl, xh, el, eh);
        } else {
          store(row, x);
          if constexpr (BOUNDS) got.add(a, z);
        }
      }
      if constexpr (!BOUNDS) continue;
      // the block's last step: its bounds
      const uint32_t done = (uint32_t)(j0 + min(r0 + step, held)), before = (uint32_t)(j0 + r0);
      if (done < (uint32_t)end && done - fast_div(done, c.map.R) * c.map.R.d != 0) continue;
      const int32_t page = __shfl(new_page, r0, kWave);
      if ((uint32_t)page < (uint32_t)c.pool.pages)  // (else reported above)
        got.store_wave(c.bounds + c.map.block(page, slice, fast_div(before, c.map.R) * c.map.R.d, c.pool.T) * bound_bytes(F, D));
      got = Bounds<F, D>();
    }
  }
  if (errors != 0) atomicOr(c.err, errors);
}

// ------------------------------------------------------------ pages onto pages
struct CopyPart {
  char* base;
  int64_t page_units, slice_units;  // of a page, and from one of its slices to the next
  FastDiv units;                    // to copy of a slice
  int64_t all;                      // to copy of a page
};
struct CopyCall {
  CopyPart part[3];
  const int32_t* from;
  const int32_t* to;
  uint32_t* err;
  int32_t pages;
};
constexpr int kCopyUnits = 4;  // units that a thread has in hand

// blockIdx.x: units of a page; .y: K, V or the bounds (or either's scales); .z: page. UNIT: the widest
// access that the parts' sizes allow. Bound by the bytes, past the caches: 49 pages of 28 layers of 4 heads of 64 rows of 128 in
// 66.7 us (5.4 TB/s of reading and writing; 70.3 through them), one such page's first 37 rows in 3.0.
template <class UNIT>
__global__ __launch_bounds__(kPageThreads) void k_page_copy(CopyCall c, int32_t z0) {
  const CopyPart p = c.part[blockIdx.y];
  if ((int64_t)blockIdx.x * (kPageThreads * kCopyUnits) >= p.all) return;
  const int64_t i0 = (int64_t)blockIdx.x * (kPageThreads * kCopyUnits) + threadIdx.x;
  const int32_t from = c.from[z0 + blockIdx.z], to = c.to[z0 + blockIdx.z];
  if ((uint32_t)from >= (uint32_t)c.pages || (uint32_t)to >= (uint32_t)c.pages) {
    if (i0 == 0 && blockIdx.y == 0) atomicOr(c.err, kDevBadPage);
    return;
  }
  if (from == to) return;
  const UNIT* src = reinterpret_cast<const UNIT*>(p.base) + from * p.page_units;
  UNIT* dst = reinterpret_cast<UNIT*>(p.base) + to * p.page_units;
  UNIT v[kCopyUnits];
  int64_t at[kCopyUnits];
#pragma unroll
  for (int u = 0; u < kCopyUnits; ++u) {
    const int64_t i = min(i0 + u * kPageThreads, p.all - 1);
    // (slices that are copied whole follow each other: p.units.d is 1 then, and the slices are units)
    const uint32_t s = fast_div((uint32_t)i, p.units);
    at[u] = s * p.slice_units + ((uint32_t)i - s * p.units.d);
    v[u] = __builtin_nontemporal_load(src + at[u]);
  }
#pragma unroll
  for (int u = 0; u < kCopyUnits; ++u)
    if (i0 + u * kPageThreads < p.all) __builtin_nontemporal_store(v[u], dst + at[u]);
}

}  // namespace ipv
