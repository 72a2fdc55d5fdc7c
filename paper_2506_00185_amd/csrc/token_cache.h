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
struct RowsArgs {
  CacheView c;
  const void *in[2];  // [B][n][heads][dim], strides in elements, dim contiguous
  void *out[2];
  int64_t stride_b[2], stride_n[2], stride_h[2];
  const int *start, *count;  // [B]; count may be NULL
  int B, n;
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

// 8 values of a row for each lane, LANES lanes (the power of two from dim / 8 on) for a row: its largest |x| stays in
// registers, every byte is read and written once.  Bound by memory.
template <typename TT, int FMT, int LANES>
__global__ __launch_bounds__(256) void k_cache_write(RowsArgs a) {
  typedef typename TT::T T;
  constexpr int ROWS = 256 / LANES;
  const int which = blockIdx.y, l = threadIdx.x % LANES;
  const int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  const int heads = a.c.heads, dim = a.c.dim;
  const int h = (int)(r % heads);
  const int64_t bn = r / heads;
  const int n = (int)(bn % a.n), b = (int)(bn / a.n);
  int64_t row = -1;
  if (b < a.B && !(a.count && n >= a.count[b])) row = cache_row(a.c, b, (int64_t)a.start[b] + n, h);
  float x[8] = {};
  uint32_t most = 0;
  const bool mine = row >= 0 && l * 8 < dim;
  if (mine) {
    const T *p = static_cast<const T *>(a.in[which]) + b * a.stride_b[which] + n * a.stride_n[which] + h * a.stride_h[which] + l * 8;
    T raw[8];
    __builtin_memcpy(raw, p, sizeof(raw));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = to_float(raw[j]);
      most = max(most, __float_as_uint(x[j]) & 0x7fffffffu);  // (of infinities and NaN the largest)
    }
  }
  most = row_max_u<LANES>(most);
  if (!mine) return;
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
    *reinterpret_cast<uintx2_t *>(base + row * dim + l * 8) = w;
  } else {
    const uintx4_t w = {pack_f16(x[0], x[1]), pack_f16(x[2], x[3]), pack_f16(x[4], x[5]), pack_f16(x[6], x[7])};
    *reinterpret_cast<uintx4_t *>(base + (row * dim + l * 8) * 2) = w;
  }
  if (l == 0) (which ? a.c.v_exp : a.c.k_exp)[row] = (uint8_t)s;
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
  constexpr int ROWS = 256 / LANES;
  const int which = blockIdx.y, l = threadIdx.x % LANES;
  const int64_t r = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
  const int heads = a.c.heads, dim = a.c.dim;
  const int h = (int)(r % heads);
  const int64_t bn = r / heads;
  const int n = (int)(bn % a.n), b = (int)(bn / a.n);
  if (b >= a.B || l * 8 >= dim) return;
  int64_t row = -1;
  if (!(a.count && n >= a.count[b])) row = cache_row(a.c, b, (int64_t)a.start[b] + n, h);
  float x[8] = {};
  if (row >= 0) {
    const float scale = row_scale((which ? a.c.v_exp : a.c.k_exp)[row]);
    const char *base = which ? a.c.v : a.c.k;
    uint32_t w[4];
    if constexpr (FMT == 8) {
      const uintx2_t q = *reinterpret_cast<const uintx2_t *>(base + row * dim + l * 8);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        w[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)q[j], 1.f, false));
        w[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)q[j], 1.f, true));
      }
    } else {
      const uintx4_t q = *reinterpret_cast<const uintx4_t *>(base + (row * dim + l * 8) * 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = q[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)__builtin_bit_cast(f16x2_t, w[j / 2])[j % 2] * scale;
  }
  T *p = static_cast<T *>(a.out[which]) + b * a.stride_b[which] + n * a.stride_n[which] + h * a.stride_h[which] + l * 8;
  put8(p, x);
}

}  // namespace rb
