// A paged cache of keys and values in 8 or 16 bits: rows written and read back, and the attention of new tokens, a tree of
// drafted ones among them, over it (rnnt_cache_write, rnnt_cache_read, rnnt_cache_attend).
//
// A row, the `dim` values of one token and head, is kept as y 2^s with one exponent s for the row: y in OCP e4m3 or in float16, s the smallest
// for which the largest |x| is at most 448 2^s, or below 2^15 2^s.  A power of two as scale makes everything but the rounding of y exact: a
// row that is read back and written again stands for the same values, and the products of the attention take y as it is, the exponents
// enter the exponents of the soft-max.
#pragma once
#include "token_types.h"

namespace rb {

struct CacheView {
  char *k, *v;             // [n_pages][heads][page_size][dim]
  uint8_t *k_exp, *v_exp;  // [n_pages][heads][page_size]: s + 127, 255 = a row of NaN
  int n_pages, page_size, page_shift, heads, dim;  // page_shift: log2(page_size)
  const int *table;        // [B][width]: page of positions width by width
  int64_t table_stride;
  int width;
};
constexpr int kExpNaN = 255, kExpZero = 127;

// Row index of a position, or -1 where the table gives none: positions outside it and pages outside the cache are not there.
__device__ __forceinline__ int64_t cache_row(const CacheView &c, int b, int64_t pos, int head) {
  if (pos < 0 || pos >= (int64_t)c.width << c.page_shift) return -1;
  const int page = c.table[b * c.table_stride + (pos >> c.page_shift)];
  if ((unsigned)page >= (unsigned)c.n_pages) return -1;
  return (((int64_t)page * c.heads + head) << c.page_shift) + (pos & (c.page_size - 1));
}

// ---- rows in and out of the cache
// x / d for x below 2^31: the upper half of a product
struct Divisor {
  uint32_t mul;
  int shift;  // -1: d = 1
};
__device__ __forceinline__ int divide(int x, Divisor d) { return d.shift < 0 ? x : (int)(__umulhi((uint32_t)x, d.mul) >> d.shift); }

struct RowsArgs {
  CacheView c;
  const void *in[2];  // [B][n][heads][dim], strides in elements, dim contiguous
  void *out[2];
  int64_t stride_b[2], stride_n[2], stride_h[2];
  const int *start, *count;  // [B]; count may be NULL
  int B, n, blocks;          // blocks of a sequence
  Divisor by_heads;
};

__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const floatx2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));  // to the nearest, subnormals kept
}
// largest of aligned groups of LANES lanes, a power of two up to 32
template <int LANES>
__device__ __forceinline__ uint32_t row_max_u(uint32_t v) {
  if constexpr (LANES >= 2) v = max(v, (uint32_t)dpp_i<kDppXor1>((int)v));
  if constexpr (LANES >= 4) v = max(v, (uint32_t)dpp_i<kDppXor2>((int)v));
  if constexpr (LANES >= 8) v = max(v, (uint32_t)dpp_i<kDppHalfMirror>((int)v));
  if constexpr (LANES >= 16) v = max(v, (uint32_t)dpp_i<kDppMirror>((int)v));
  if constexpr (LANES >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16));
  return v;
}

// 8 values of a row for each lane, LANES lanes (the power of two from dim / 8 on) for a row, four rows for each of their groups: a row's largest |x|
// stays in registers, every byte is read and written once.  Bound by memory: a block's loads all leave at once.  With one row for a group
// 16 x 1501 tokens of 8 x 128 were read in 29 us, now 24.5 (6 TB/s); 8 x 2048 are written in 22 us (4.5 TB/s); small calls take 4 to 5 us either way.
// The rows of a sequence are counted through its tokens' heads; `which`: keys or values.
struct RowAt {
  int i, h;
  bool mine;  // a row of the call, and dims of it
};
constexpr int kRowsOfGroup = 4;
template <int LANES>
__device__ __forceinline__ RowAt row_at(const RowsArgs &a, int r) {
  RowAt o;
  o.i = divide(r, a.by_heads);
  o.h = r - o.i * a.c.heads;
  o.mine = r < a.n * a.c.heads && (int)(threadIdx.x % LANES) * 8 < a.c.dim;
  return o;
}

template <typename TT, int FMT, int LANES>
__global__ __launch_bounds__(256) void k_cache_write(RowsArgs a) {
  typedef typename TT::T T;
  constexpr int ROWS = 256 / LANES, U = kRowsOfGroup;
  const int which = blockIdx.y, l = threadIdx.x % LANES, b = blockIdx.x / a.blocks, dim = a.c.dim;
  const int r0 = (blockIdx.x - b * a.blocks) * ROWS * U + threadIdx.x / LANES;
  const int start = a.start[b], count = a.count ? a.count[b] : a.n;
  const T *in = static_cast<const T *>(a.in[which]) + b * a.stride_b[which] + l * 8;
  T raw[U][8];
  int64_t row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const RowAt at = row_at<LANES>(a, r0 + u * ROWS);
    __builtin_memcpy(raw[u], at.mine ? in + at.i * a.stride_n[which] + at.h * a.stride_h[which] : static_cast<const T *>(a.in[which]), sizeof(raw[u]));
    row[u] = at.mine && at.i < count ? cache_row(a.c, b, (int64_t)start + at.i, at.h) : -1;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float x[8];
    uint32_t most = 0;
    const bool mine = row_at<LANES>(a, r0 + u * ROWS).mine;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = to_float(raw[u][j]);
      most = max(most, __float_as_uint(x[j]) & 0x7fffffffu);  // (of infinities and NaN the largest)
    }
    most = row_max_u<LANES>(mine ? most : 0);
    if (row[u] < 0) continue;
    const int e = (int)(most >> 23);
    // 448 = 1.75 2^8: a mantissa beyond 1.75 takes the next exponent
    int s = FMT == 8 ? e - 8 + ((most & 0x7fffffu) > 0x600000u) : e - 14;
    s = most == 0 ? kExpZero : max(s, 1);
    const bool nan = e == 255;
    if (nan) s = kExpNaN;
    const float inv = nan ? 0.f : __uint_as_float((uint32_t)(254 - s) << 23);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = nan ? 0.f : x[j] * inv;
    char *base = which ? a.c.v : a.c.k;
    if constexpr (FMT == 8) {
      const uintx2_t w = {pack_e4m3(x[0], x[1], x[2], x[3]), pack_e4m3(x[4], x[5], x[6], x[7])};
      *reinterpret_cast<uintx2_t *>(base + row[u] * dim + l * 8) = w;
    } else {
      const uintx4_t w = {pack_f16(x[0], x[1]), pack_f16(x[2], x[3]), pack_f16(x[4], x[5]), pack_f16(x[6], x[7])};
      *reinterpret_cast<uintx4_t *>(base + (row[u] * dim + l * 8) * 2) = w;
    }
    if (l == 0) (which ? a.c.v_exp : a.c.k_exp)[row[u]] = (uint8_t)s;
  }
}

__device__ __forceinline__ float row_scale(int e) { return e == kExpNaN ? NAN : e == 0 ? 0x1p-127f : __uint_as_float((uint32_t)e << 23); }

__device__ __forceinline__ void put8(float *p, const float (&x)[8]) { __builtin_memcpy(p, x, 32); }
__device__ __forceinline__ void put8(_Float16 *p, const float (&x)[8]) {
  const uint32_t w[4] = {pack_f16(x[0], x[1]), pack_f16(x[2], x[3]), pack_f16(x[4], x[5]), pack_f16(x[6], x[7])};
  __builtin_memcpy(p, w, 16);
}
__device__ __forceinline__ void put8(uint16_t *p, const float (&x)[8]) {
  const uint32_t w[4] = {pack_bf16_rne(x[0], x[1]), pack_bf16_rne(x[2], x[3]), pack_bf16_rne(x[4], x[5]), pack_bf16_rne(x[6], x[7])};
  __builtin_memcpy(p, w, 16);
}

template <typename TT, int FMT, int LANES>
__global__ __launch_bounds__(256) void k_cache_read(RowsArgs a) {
  typedef typename TT::T T;
  constexpr int ROWS = 256 / LANES, U = kRowsOfGroup;
  const int which = blockIdx.y, l = threadIdx.x % LANES, b = blockIdx.x / a.blocks, dim = a.c.dim;
  const int r0 = (blockIdx.x - b * a.blocks) * ROWS * U + threadIdx.x / LANES;
  const int start = a.start[b], count = a.count ? a.count[b] : a.n;
  const char *base = which ? a.c.v : a.c.k;
  const uint8_t *exps = which ? a.c.v_exp : a.c.k_exp;
  int64_t row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const RowAt at = row_at<LANES>(a, r0 + u * ROWS);
    row[u] = at.mine && at.i < count ? cache_row(a.c, b, (int64_t)start + at.i, at.h) : -1;
  }
  uint32_t w[U][FMT / 4];
  int e[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {  // (row 0 for rows that are not there)
    const int64_t from = row[u] < 0 ? 0 : row[u] * dim + l * 8;
    __builtin_memcpy(w[u], __builtin_assume_aligned(base + from * (FMT / 8), FMT), FMT);
    e[u] = exps[row[u] < 0 ? 0 : row[u]];
  }
  T *out = static_cast<T *>(a.out[which]) + b * a.stride_b[which] + l * 8;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const RowAt at = row_at<LANES>(a, r0 + u * ROWS);
    if (!at.mine) continue;
    const float scale = row_scale(e[u]);
    float x[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t pair;
      if constexpr (FMT == 8)
        pair = __builtin_bit_cast(uint32_t, j % 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w[u][j / 2], 1.f, true)
                                                  : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w[u][j / 2], 1.f, false));
      else
        pair = w[u][j];
      const f16x2_t y = __builtin_bit_cast(f16x2_t, pair);
      x[2 * j] = row[u] < 0 ? 0.f : (float)y[0] * scale;
      x[2 * j + 1] = row[u] < 0 ? 0.f : (float)y[1] * scale;
    }
    put8(out + at.i * a.stride_n[which] + at.h * a.stride_h[which], x);
  }
}

}  // namespace rb
