// Pages of cache rows: how a row is found, its 8- and 4-bit elements, and the
// kernels that write rows into pages and read them back.
#pragma once

#include <type_traits>

#include "ipv_device.hpp"

namespace ipv {

typedef __bf16 Bf16x8 __attribute__((ext_vector_type(8)));
typedef float F32x4 __attribute__((ext_vector_type(4)));
typedef float F32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t U32x2 __attribute__((ext_vector_type(2)));

// Element formats of a pool (ipv_page_format).
constexpr int kFmtBf16 = 0, kFmtF32 = 1, kFmtFp8 = 2, kFmtFp4 = 3;
constexpr int kScaleBlock = 32;  // elements that share a scale
constexpr uint32_t kDevNan = 16u, kDevBadPage = 64u;

constexpr int fmt_bits(int f) { return f == kFmtBf16 ? 16 : f == kFmtF32 ? 32 : f == kFmtFp8 ? 8 : 4; }
constexpr bool fmt_scaled(int f) { return f == kFmtFp8 || f == kFmtFp4; }
constexpr int fmt_row_bytes(int f, int D) { return fmt_bits(f) * D / 8; }

// A pool and the table of its pages. Rows are counted over the whole pool
// (page, layer, head, slot), in 64 bits: bytes are rows times the row's bytes.
struct Pool {
  char* K;
  char* V;
  uint8_t* Ks;
  uint8_t* Vs;
  const int32_t* table;  // null: stream b's only page is page b
  int32_t cols, pages;
  int64_t page_rows_all;  // rows of a page over all its layers and heads
  int64_t layer_rows;     // rows of a page's layer: H * T
  FastDiv T;              // rows of a page's (layer, head)
};

// The page of position j of stream b, as the table has it. Where a loop looks rows up
// ahead, this load is apart from what is made of it, so that nothing waits for it meanwhile.
__device__ __forceinline__ int32_t pool_page(const Pool& p, int b, uint32_t j) {
  return p.table ? p.table[(int64_t)b * p.cols + fast_div(j, p.T)] : b;
}

// The same where j is the same in all lanes: a scalar load (the table is not written meanwhile).
__device__ __forceinline__ int32_t pool_page_uniform(const Pool& p, int b, uint32_t j) {
  if (!p.table) return b;
  typedef const int32_t __attribute__((address_space(4))) * Constant;
  return *(Constant)(uintptr_t)(p.table + ((int64_t)b * p.cols + fast_div(j, p.T)));
}

// Row of position j, which lies in that page, counted from the pool's first within
// the first (layer, head); add (layer * H + head) * T. *bad: there is no such page
// (page 0 is taken in its place).
__device__ __forceinline__ int64_t pool_row(const Pool& p, int32_t page, uint32_t j, bool* bad) {
  *bad = (uint32_t)page >= (uint32_t)p.pages;
  return (int64_t)(*bad ? 0 : page) * p.page_rows_all + (j - fast_div(j, p.T) * p.T.d);
}

// Where the bounds of blocks are: [page][slice][block of the page's slice].
struct BlockMap {
  FastDiv R;       // rows of a block, which divide a page's
  int64_t slices;  // of a page: layers times heads
  uint32_t per;    // blocks of a page's slice
  // Number of the block that starts at that position, which lies in that page.
  __device__ __forceinline__ int64_t block(int64_t page, uint32_t slice, uint32_t position, const FastDiv& T) const {
    return (page * slices + slice) * per + fast_div(position - fast_div(position, T) * T.d, R);
  }
};

// A scale byte as the power of two that the conversions take (255: NaN).
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 B2 __attribute__((ext_vector_type(2)));
  const B2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// Eight stored elements (8 bytes of e4m3, 4 of e2m1) as bf16: exact, since a
// bf16 has more mantissa bits and the scale is a power of two.
__device__ __forceinline__ Raw16 fp8_to_bf16(uint32_t lo, uint32_t hi, float scale) {
  Raw16 r;
  r.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  r.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  r.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  r.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  return r;
}
__device__ __forceinline__ Raw16 fp4_to_bf16(uint32_t x, float scale) {
  Raw16 r;
  r.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0));
  r.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1));
  r.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2));
  r.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3));
  return r;
}

// Scale bytes of a row as a 64-bit word.
template <int D>
__device__ __forceinline__ uint64_t load_scales(const uint8_t* scales, int64_t row) {
  const uint8_t* p = scales + row * (D / kScaleBlock);
  if (D == 32) return *p;
  if (D == 64) return *reinterpret_cast<const uint16_t*>(p);
  if (D == 128) return *reinterpret_cast<const uint32_t*>(p);
  const uint32_t lo = reinterpret_cast<const uint32_t*>(p)[0], hi = reinterpret_cast<const uint32_t*>(p)[1];
  return ((uint64_t)hi << 32) | lo;
}
__device__ __forceinline__ float scale_at(uint64_t w, int block) { return scale_of((uint32_t)(w >> (8 * block)) & 255u); }

__device__ __forceinline__ int64_t shfl64(int64_t v, int lane) {
  const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)v, lane, kWave);
  const uint32_t hi = (uint32_t)__shfl((int)(uint32_t)((uint64_t)v >> 32), lane, kWave);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

template <int BYTES>
__device__ __forceinline__ void load_piece(const char* p, uint32_t* w) {
  if (BYTES == 16) {
    const Raw16 r = load16(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = r.w[i];
  } else if (BYTES == 8) {
    const U32x2 r = *reinterpret_cast<const U32x2*>(p);
    w[0] = r.x, w[1] = r.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// Sum over aligned groups of G lanes (2, 4, 8 or 16), the same in all of them.
template <int G>
__device__ __forceinline__ double group_sum64(double v) {
  const auto other = [](double x, auto ctrl) __attribute__((always_inline)) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = dpp_u32<decltype(ctrl)::value>((uint32_t)u), hi = dpp_u32<decltype(ctrl)::value>((uint32_t)(u >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  v += other(v, std::integral_constant<int, kDppXor1>());
  if (G >= 4) v += other(v, std::integral_constant<int, kDppXor2>());
  if (G >= 8) v += other(v, std::integral_constant<int, kDppHalfMirror>());
  if (G >= 16) v += other(v, std::integral_constant<int, kDppRowMirror>());
  return v;
}

// ------------------------------------------------------------ rows in and out
constexpr int kPageStreams = 128;  // streams of one launch (their counts travel in its arguments)
constexpr int kPageThreads = 256;
constexpr int kPageSlices = 4;     // (layer, head) slices a thread takes, at one position

struct PageCall {
  Pool pool;
  char* K;  // the caller's rows
  char* V;
  int64_t sb, sl, sh, sr;  // strides of stream, layer, head, row (elements)
  const float* rotary;
  uint32_t* err;
  int32_t b0;              // first stream of the launch
  int32_t H, LH;           // KV heads, slices of the call (its layers times heads)
  int64_t first_slice;     // rows of a page before the call's first layer
  FastDiv H_div;
  int32_t first[kPageStreams], rows[kPageStreams];
};

// k' of the pairs (lo[i], hi[i]), or back; products and sums rounded one by
// one, so that a pair turns the same wherever it is computed.
__device__ __forceinline__ void turn(float (&lo)[8], float (&hi)[8], const float (&c)[8], const float (&s)[8], bool back) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float sn = back ? -s[i] : s[i];
    const float a = lo[i] * c[i], b = hi[i] * sn, d = hi[i] * c[i], e = lo[i] * sn;
    lo[i] = a - b;
    hi[i] = d + e;
  }
}

__device__ __forceinline__ void load_angles(const float* table, int64_t pos, int half, int d, float (&c)[8], float (&s)[8]) {
  const F32x4* t = reinterpret_cast<const F32x4*>(table + (pos * half + d) * 2);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const F32x4 v = t[i];
    c[2 * i] = v.x, s[2 * i] = v.y, c[2 * i + 1] = v.z, s[2 * i + 1] = v.w;
  }
}

// Eight elements of a caller's row.
template <int SRC>
__device__ __forceinline__ void load_row8(const char* base, int64_t elem, float (&f)[8]) {
  if (SRC == kFmtBf16) {
    Lane<uint16_t>::decode(load16(base + elem * 2), f);
  } else {
    float a[4], b[4];
    Lane<float>::decode(load16(base + elem * 4), a);
    Lane<float>::decode(load16(base + elem * 4 + 16), b);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = a[i], f[4 + i] = b[i];
  }
}
// STREAM: past the caches. Rows that come back are written once and read by a later
// kernel over all of them; as dirty lines they held up the kernels around (28 layers of
// 3136 rows: read 53 -> 45 us, the write before it 64 -> 51 us).
template <int DST, bool STREAM>
__device__ __forceinline__ void store_row8(char* base, int64_t elem, const float (&f)[8]) {
  if (DST == kFmtBf16) {
    Raw16 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
    if (STREAM) store16(base + elem * 2, r);
    else *reinterpret_cast<Raw16*>(base + elem * 2) = r;
  } else {
    F32x4* p = reinterpret_cast<F32x4*>(base + elem * 4);
    const F32x4 a = {f[0], f[1], f[2], f[3]}, b = {f[4], f[5], f[6], f[7]};
    if (STREAM) __builtin_nontemporal_store(a, p), __builtin_nontemporal_store(b, p + 1);
    else p[0] = a, p[1] = b;
  }
}

__device__ __forceinline__ uint32_t max_abs_bits(const float (&f)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
  return m;
}

// The scale byte of a block whose largest magnitude has these bits: the
// smallest e >= -126 with amax <= TOP * 2^e, plus 127; TOP is 1.75 * 2^8
// (e4m3) or 1.5 * 2^2 (e2m1). 255 for infinities and NaN. AGAIN: of stored values turned
// anew, whose largest is often TOP * 2^e itself: up to (1 + 2^-16) times that, so that one that
// a turn of next to nothing, or its rounding, made larger does not cost the block a bit.
template <int F, bool AGAIN = false>
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
  constexpr int shift = F == kFmtFp8 ? 8 : 2;
  constexpr uint32_t top = (F == kFmtFp8 ? 0x600000u : 0x400000u) + (!AGAIN ? 0u : F == kFmtFp8 ? 224u : 192u);  // mantissa bits of 1.75, 1.5
  const int e = (int)(bits >> 23) - shift + ((bits & 0x7fffffu) > top ? 1 : 0);
  return bits >= 0x7f800000u ? 255u : (uint32_t)max(e, 1);
}

// Eight elements to their stored bits (one dword of e2m1, two of e4m3).
template <int F>
__device__ __forceinline__ void encode8(const float (&f)[8], uint32_t byte, uint32_t (&w)[2]) {
  const float inv = __uint_as_float((254u - (byte == 255u ? 127u : byte)) << 23);  // 2^-e
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = f[i] * inv;
  if (F == kFmtFp8) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], v, true);
    }
    if (byte == 255u) w[0] = w[1] = 0x7f7f7f7fu;
  } else {
    uint32_t v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], 1.0f, 0);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[2], y[3], 1.0f, 1);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[4], y[5], 1.0f, 2);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, y[6], y[7], 1.0f, 3);
    w[0] = byte == 255u ? 0u : v;
    w[1] = 0;
  }
}

// One row of a slice is written by D / 16 threads, each with eight elements of
// the row's first half and the eight it is paired with for the rotation; four
// neighbours (two for D = 32, with both their halves) hold a scale's block.
template <int D>
struct RowSplit {
  static constexpr int kThreads = D / 16;                      // threads a row
  static constexpr int kRows = kPageThreads / kThreads;        // rows a workgroup has in hand
};

// The scale bytes of a row, from the threads that have them (el, eh: of the block
// that a thread's elements of the first and of the second half lie in), stored
// by the row's first thread at once.
template <int D>
__device__ __forceinline__ void store_scales(uint8_t* at, int thread, uint32_t el, uint32_t eh) {
  if (D == 32) {
    if (thread == 0) *at = (uint8_t)el;
  } else if (D == 64) {
    if (thread == 0) *reinterpret_cast<uint16_t*>(at) = (uint16_t)(el | eh << 8);
  } else {
    // row_shl 4, 8, 12: the values of the threads 4, 8 and 12 further on
    uint32_t lo = el | dpp_u32<0x104>(el) << 8, hi = eh | dpp_u32<0x104>(eh) << 8;
    if (D == 128) {
      if (thread == 0) *reinterpret_cast<uint32_t*>(at) = lo | hi << 16;
    } else {
      lo |= dpp_u32<0x108>(lo) << 16, hi |= dpp_u32<0x108>(hi) << 16;
      if (thread == 0) *reinterpret_cast<uint32_t*>(at) = lo, *reinterpret_cast<uint32_t*>(at + 4) = hi;
    }
  }
}

// A row into the pool, from the threads that hold it (lo and hi: eight elements of either half).
// wl, wh: what is stored, as dwords of e4m3 (two) or e2m1 (one); el, eh: the scales' bytes.
template <int F, int D, bool AGAIN = false, bool STREAM = false>
__device__ __forceinline__ void put_row(char* pages, uint8_t* scales, int64_t row, int d, const float (&lo)[8], const float (&hi)[8],
                                        uint32_t* err, uint32_t (&wl)[2], uint32_t (&wh)[2], uint32_t& el, uint32_t& eh) {
  if (!fmt_scaled(F)) {
    store_row8<F, STREAM>(pages, row * D + d, lo);
    store_row8<F, STREAM>(pages, row * D + D / 2 + d, hi);
  } else {
    uint32_t ml = max_abs_bits(lo), mh = max_abs_bits(hi);
    if (D == 32) ml = mh = max(ml, mh);
    ml = max(ml, dpp_u32<kDppXor1>(ml));
    mh = max(mh, dpp_u32<kDppXor1>(mh));
    if (D > 32) {
      ml = max(ml, dpp_u32<kDppXor2>(ml));
      mh = max(mh, dpp_u32<kDppXor2>(mh));
    }
    el = scale_byte<F, AGAIN>(ml), eh = scale_byte<F, AGAIN>(mh);
    encode8<F>(lo, el, wl);
    encode8<F>(hi, eh, wh);
    char* at = pages + row * fmt_row_bytes(F, D);
    if (F == kFmtFp8) {
      *reinterpret_cast<U32x2*>(at + d) = U32x2{wl[0], wl[1]};
      *reinterpret_cast<U32x2*>(at + D / 2 + d) = U32x2{wh[0], wh[1]};
    } else {
      *reinterpret_cast<uint32_t*>(at + d / 2) = wl[0];
      *reinterpret_cast<uint32_t*>(at + D / 4 + d / 2) = wh[0];
    }
    store_scales<D>(scales + row * (D / kScaleBlock), d / 8, el, eh);
    if (el == 255u || eh == 255u) atomicOr(err, kDevNan);
  }
}

// blockIdx.x: kRows positions of a stream; .y: kPageSlices slices, of K or of V;
// .z: stream. A workgroup's rows follow each other in the caller's slices and,
// page by page, in the pool. Bound by the bytes: 28 layers of 4 heads of 3136 rows of 128, bf16 to
// fp8 with the rotation, 272 MB in 52 us (5.3 TB/s); one row of 16 streams 4.9 us.
template <int F, int SRC, int D>
__global__ __launch_bounds__(kPageThreads) void k_page_write(PageCall c) {
  using S = RowSplit<D>;
  const int b = blockIdx.z;
  const int i = (int)(blockIdx.x * S::kRows + threadIdx.x / S::kThreads);
  if (i >= c.rows[b]) return;  // whole rows' threads leave together
  const uint32_t g = blockIdx.y >> 1;
  const bool isv = blockIdx.y & 1;
  const int d = (int)(threadIdx.x % S::kThreads) * 8;
  const int64_t pos = (int64_t)c.first[b] + i;
  bool bad;
  const int64_t row0 = pool_row(c.pool, pool_page(c.pool, c.b0 + b, (uint32_t)pos), (uint32_t)pos, &bad) + c.first_slice;
  if (bad) {
    if (d == 0) atomicOr(c.err, kDevBadPage);
    return;
  }
  const char* src = isv ? c.V : c.K;
  char* dst = isv ? c.pool.V : c.pool.K;
  uint8_t* sc = isv ? c.pool.Vs : c.pool.Ks;
  const bool rot = !isv && c.rotary != nullptr;
  float cs[8], sn[8];
  if (rot) load_angles(c.rotary, pos, D / 2, d, cs, sn);
  const int64_t src0 = (int64_t)(c.b0 + b) * c.sb + (int64_t)i * c.sr + d;
  float lo[kPageSlices][8], hi[kPageSlices][8];
#pragma unroll
  for (int u = 0; u < kPageSlices; ++u) {
    const uint32_t lh = min(g * kPageSlices + u, (uint32_t)c.LH - 1u);
    const uint32_t l = fast_div(lh, c.H_div);
    const int64_t at = src0 + (int64_t)l * c.sl + (int64_t)(lh - l * c.H) * c.sh;
    load_row8<SRC>(src, at, lo[u]);
    load_row8<SRC>(src, at + D / 2, hi[u]);
  }
#pragma unroll
  for (int u = 0; u < kPageSlices; ++u) {
    const uint32_t lh = g * kPageSlices + u;
    if (lh >= (uint32_t)c.LH) break;
    if (rot) turn(lo[u], hi[u], cs, sn, false);
    uint32_t wl[2], wh[2], el, eh;
    put_row<F, D>(dst, sc, row0 + (int64_t)lh * c.pool.T.d, d, lo[u], hi[u], c.err, wl, wh, el, eh);
  }
}

template <int F, int D>
__device__ __forceinline__ void decode_row8(const char* pages, const uint8_t* scales, int64_t row, int d, float (&f)[8]) {
  if (!fmt_scaled(F)) {
    load_row8<F>(pages, row * D + d, f);
    return;
  }
  const float scale = scale_of(scales[row * (D / kScaleBlock) + d / kScaleBlock]);
  Raw16 r;
  if (F == kFmtFp8) {
    const U32x2 w = *reinterpret_cast<const U32x2*>(pages + row * D + d);
    r = fp8_to_bf16(w.x, w.y, scale);
  } else {
    r = fp4_to_bf16(*reinterpret_cast<const uint32_t*>(pages + row * (D / 2) + d / 2), scale);
  }
  Lane<uint16_t>::decode(r, f);
}

// The way back, split alike: the same rows 43 us after their writing, 49 us from memory (5.6 TB/s).
template <int F, int DST, int D>
__global__ __launch_bounds__(kPageThreads) void k_page_read(PageCall c) {
  using S = RowSplit<D>;
  const int b = blockIdx.z;
  const int i = (int)(blockIdx.x * S::kRows + threadIdx.x / S::kThreads);
  if (i >= c.rows[b]) return;  // whole rows' threads leave together
  const uint32_t g = blockIdx.y >> 1;
  const bool isv = blockIdx.y & 1;
  const int d = (int)(threadIdx.x % S::kThreads) * 8;
  const int64_t pos = (int64_t)c.first[b] + i;
  bool bad;
  const int64_t row0 = pool_row(c.pool, pool_page(c.pool, c.b0 + b, (uint32_t)pos), (uint32_t)pos, &bad) + c.first_slice;
  if (bad && d == 0) atomicOr(c.err, kDevBadPage);
  const char* src = isv ? c.pool.V : c.pool.K;
  char* dst = isv ? c.V : c.K;
  const uint8_t* sc = isv ? c.pool.Vs : c.pool.Ks;
  const bool rot = !isv && c.rotary != nullptr;
  float cs[8], sn[8];
  if (rot) load_angles(c.rotary, pos, D / 2, d, cs, sn);
  const int64_t dst0 = (int64_t)(c.b0 + b) * c.sb + (int64_t)i * c.sr + d;
  float lo[kPageSlices][8], hi[kPageSlices][8];
#pragma unroll
  for (int u = 0; u < kPageSlices; ++u) {
    const int64_t row = row0 + (int64_t)min(g * kPageSlices + u, (uint32_t)c.LH - 1u) * c.pool.T.d;
    decode_row8<F, D>(src, sc, row, d, lo[u]);
    decode_row8<F, D>(src, sc, row, D / 2 + d, hi[u]);
  }
#pragma unroll
  for (int u = 0; u < kPageSlices; ++u) {
    const uint32_t lh = g * kPageSlices + u;
    if (lh >= (uint32_t)c.LH) break;
    if (rot) turn(lo[u], hi[u], cs, sn, true);
    const uint32_t l = fast_div(lh, c.H_div);
    const int64_t at = dst0 + (int64_t)l * c.sl + (int64_t)(lh - l * c.H) * c.sh;
    // past the caches where a store covers whole 128-byte lines; parts of lines are put together there
    // (to fp32 from e4m3, 151 MB of heads of 64: 47 us past the caches and 28 through them; bf16 heads
    // of 32, 120 MB: 24.6 and 21.5)
    constexpr bool STREAM = DST == kFmtBf16 && D >= 128;
    store_row8<DST, STREAM>(dst, at, lo[u]);
    store_row8<DST, STREAM>(dst, at + D / 2, hi[u]);
  }
}

}  // namespace ipv
