// Attention of new tokens over the paged cache (rnnt_cache_attend).
#pragma once
#include "token_cache.h"

namespace rb {

// A block takes MT * 16 rows, a row being one query head of one node: the nodes of a sequence and the query heads that share a key head
// side by side, so that a tree's nodes and the heads of a group fill a tile and the cache is read once for all of them.  Its four waves
// take tiles of 32 tokens in turn; nothing goes through LDS but the tiles' exponents and row indices:
//   S^T = K Q^T   a lane loads a quarter of a key row as it lies in memory, the matrix instruction's 8-k slices being cut
//                 from those quarters (Q is held in the same order); it gets the logits of 4 + 4 tokens for one row,
//   O^T = V^T P^T exactly which it hands back as the operand, again in an order of its own: k-slice j of lane group g is token 4 g + j
//                 of the first 16 and of the second.  V^T's operand are the same tokens' values of dim / 16 neighbouring dims, which a
//                 lane loads as they lie in memory and transposes in registers.
// Exponents: x = log2(e) scale q.k 2^(s_k) is the logit in base 2.  A value row's exponent is added to it: P' = 2^(x + s_v - M) is rounded to
// float16 and multiplied by y_v as stored, and the soft-max's denominator sums P' 2^(-s_v).  P' is at most 2^15 and the largest of a row at
// least 2^7: float16 keeps 11 bits of those down to 2^-21 of the largest.  Precision: Q is scaled by a power of two for each row and
// rounded to float16 (bfloat16 values down to 2^-28 of the row's largest are exact), float32 Q as a sum of two float16; P' is one float16 where
// the output is bfloat16, whose rounding is eight times as coarse, else a sum of two; sums are float32.
// M follows the running maximum only when a logit passes it by 2^8 (the range that float16 leaves above), so that the accumulators are
// multiplied by a correction a few times in a row of thousands of tokens.
struct AttendArgs {
  CacheView c;
  const void *q;
  void *out;  // [B][n][q_heads][dim]
  int64_t stride_b, stride_n, stride_h;  // of q, in elements
  const int *lens, *parents;             // parents [B][tree] or NULL: node i's is i - 1
  int B, n, tree, group;                 // queries are the last n of `tree` nodes
  int rows, row_tiles, splits, split_len;  // split_len: tokens, a multiple of 128
  float scale;
  float *part;   // [splits][B * heads][rows][dim]
  float2 *stat;  // [splits][B * heads][rows]: (M, sum); a negative sum: the row's node is not there
};

constexpr int kTreeMax = 1024;  // nodes of a tree with parents
constexpr float kMStart = -1e30f;
constexpr float kTop = 7.f;   // P' of the running maximum is 2^kTop
constexpr float kSlack = 8.f;

__device__ __forceinline__ uint32_t perm_b32(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }
__device__ __forceinline__ uint32_t e4m3_lo(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, false)); }
__device__ __forceinline__ uint32_t e4m3_hi(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, true)); }

// Value exponents are taken relative to one of the sequence's first rows, so that the sums of a block stay far from float32's ends: the first that
// tells anything (zero rows have kExpZero).  One call per wave; the same for all blocks of a sequence's head.
__device__ __forceinline__ int reference_exp(const CacheView &c, int b, int h, int total) {
  const int lane = threadIdx.x & 63;
  const int64_t row = lane < total ? cache_row(c, b, lane, h) : -1;
  const int e = row >= 0 ? c.v_exp[row] : kExpNaN;
  const uint64_t good = __ballot(e != kExpZero && e != kExpNaN);
  return good ? __builtin_amdgcn_readlane(e, __ffsll((unsigned long long)good) - 1) : kExpZero;
}

// what two values rounded to float16 leave, rounded to float16
__device__ __forceinline__ uint32_t pack_f16_rest(float a, float b, uint32_t hi) {
  const f16x2_t h = __builtin_bit_cast(f16x2_t, hi);
  return pack_f16(a - (float)h[0], b - (float)h[1]);
}

// a pair of float16 with zeros in place of NaN and infinities
__device__ __forceinline__ uint32_t finite_f16(uint32_t w) {
  w = (w & 0x7c00u) == 0x7c00u ? w & 0xffff0000u : w;
  return (w & 0x7c000000u) == 0x7c000000u ? w & 0xffffu : w;
}

// the N bytes at p (N = 4, 8, 16, 32, 64), or zeros
template <int N>
struct Bytes {
  uint32_t w[N / 4];
};
template <int N>
__device__ __forceinline__ void load_bytes(Bytes<N> &d, const char *p) {
  if constexpr (N >= 16) {
#pragma unroll
    for (int i = 0; i < N / 16; ++i) {
      const uintx4_t t = reinterpret_cast<const uintx4_t *>(p)[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) d.w[4 * i + j] = t[j];
    }
  } else if constexpr (N == 8) {
    const uintx2_t t = *reinterpret_cast<const uintx2_t *>(p);
    d.w[0] = t[0];
    d.w[1] = t[1];
  } else {
    d.w[0] = *reinterpret_cast<const uint32_t *>(p);
  }
}

template <typename TT, int FMT, int DP, int MT>
struct Attend {
  typedef typename TT::T T;
  static constexpr int FB = FMT / 8;                       // bytes of a kept value
  static constexpr bool Q2 = std::is_same<T, float>::value;        // Q as two float16
  static constexpr bool P2 = !std::is_same<T, uint16_t>::value;    // P' as two float16
  static constexpr int KS = DP / 32;                       // k-steps of Q.K
  static constexpr int KQ = DP / 4;                        // values of a key row that a lane holds
  static constexpr int VN = DP / 16;                       // values of a value row that a lane holds
  static constexpr int QN = Q2 ? 2 : 1;

  struct Shared {
    uint32_t mask[MT * 16][kTreeMax / 32];
    float m[4][MT * 16], l[4][MT * 16];
    float o[4][MT * 16][DP + 4];
    uint8_t gone[MT * 16];
  };
  struct Meta {  // of a wave's tile of 32 tokens
    uint32_t row[32];
    float k_scale[32], v_exp[32], v_inv[32];
  };
  struct Tile {
    Bytes<KQ * FB> k[2];
    Bytes<VN * FB> v[8];
  };
};

template <typename TT, int FMT, int DP, int MT>
__global__ __launch_bounds__(256) void k_attend(AttendArgs a) {
  using A = Attend<TT, FMT, DP, MT>;
  typedef typename A::T T;
  constexpr int KS = A::KS, KQ = A::KQ, VN = A::VN, FB = A::FB, QN = A::QN;
  __shared__ typename A::Shared sh;
  __shared__ typename A::Meta meta[4];
  const CacheView &c = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g4 = lane >> 4;

  // blocks of the same tokens on one XCD, one after the other: block i runs on XCD i % 8
  const int groups = a.B * c.heads * a.splits;
  const int per = 8 * a.row_tiles, slab = blockIdx.x / per, in = blockIdx.x - slab * per;
  const int item = slab * 8 + (in & 7), tile_r = in >> 3;
  if (item >= groups) return;
  const int split = item % a.splits, bh = item / a.splits, b = bh / c.heads, h = bh - b * c.heads;
  const int row0 = tile_r * MT * 16;

  const int64_t room = (int64_t)c.width << c.page_shift;
  const int len = max(a.lens[b], 0);
  const int total = (int)min((int64_t)len + a.tree, room);
  const int t_begin = (int)min((int64_t)split * a.split_len, (int64_t)total);
  const int t_end = split + 1 < a.splits ? (int)min((int64_t)t_begin + a.split_len, (int64_t)total) : total;
  if (split && t_begin >= t_end) return;
  const int D = c.dim;

  // ---- which nodes a row sees, where the block's tokens reach into the tree
  const int first_q = a.tree - a.n;  // node of query 0
  const bool treed = a.parents && t_end > t_begin && (t_end > len || t_end == total);
  if (treed) {
    for (int i = threadIdx.x; i < MT * 16 * (kTreeMax / 32); i += 256) (&sh.mask[0][0])[i] = 0;
    __syncthreads();
    if (threadIdx.x < MT * 16) {
      const int r = row0 + threadIdx.x;
      bool gone = false;
      if (r < a.rows) {
        const int *parents = a.parents + (int64_t)b * a.tree;
        int j = first_q + r / a.group;
        while (true) {
          sh.mask[threadIdx.x][j >> 5] |= 1u << (j & 31);
          const int p = parents[j];
          if (p < -1 || p >= j) {
            gone = true;
            break;
          }
          if (p < 0) break;
          j = p;
        }
      }
      sh.gone[threadIdx.x] = gone;
    }
    __syncthreads();
  }

  // ---- Q, in the order of the key rows: lane (l16, g4) holds values g4 KQ .. of row l16 of each tile
  uintx4_t q[MT][QN][KS];
  float q_scale[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int r = row0 + m * 16 + l16, node = r / a.group, head = h * a.group + r % a.group;
    float x[KQ];
    float most = 0.f;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < KQ; i += 8) {
      const bool there = r < a.rows && g4 * KQ + i < D;
      T raw[8] = {};
      if (there) __builtin_memcpy(raw, static_cast<const T *>(a.q) + b * a.stride_b + node * a.stride_n + head * a.stride_h + g4 * KQ + i, sizeof(raw));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[i + j] = to_float(raw[j]);
        most = fmaxf(most, fabsf(x[i + j]));
        bad |= !(fabsf(x[i + j]) < INFINITY);
      }
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    bad = bad || most == INFINITY;
    bad = __shfl_xor((int)bad, 16) | (int)bad;
    bad = __shfl_xor((int)bad, 32) | (int)bad;
    // the row's largest to [2^14, 2^15)
    const int e = min(max((int)(__float_as_uint(most) >> 23), 15), 254);
    const float to = __uint_as_float((uint32_t)(min(254 + 14 - e, 254)) << 23);
    const int back = 127 - (min(254 + 14 - e, 254) - 127);
    q_scale[m] = bad ? NAN : __uint_as_float((uint32_t)max(back, 1) << 23) * a.scale * (float)kLog2E;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float u = x[s * 8 + 2 * w] * to, v = x[s * 8 + 2 * w + 1] * to;
        if (bad) u = v = 0.f;
        const uint32_t hi = pack_f16(u, v);
        q[m][0][s][w] = hi;
        if constexpr (A::Q2) q[m][1][s][w] = pack_f16_rest(u, v, hi);
      }
  }

  floatx4 acc[MT][VN];
  float M[MT], sum[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    M[m] = kMStart;
    sum[m] = 0.f;
#pragma unroll
    for (int i = 0; i < VN; ++i) acc[m][i] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  const int e0 = reference_exp(c, b, h, total);

  typename A::Tile tile;
  typename A::Meta &mt = meta[wave];
  // page of the lane's token of a tile: lanes 0..31 and 32..63 the same tokens
  auto page_of = [&](int t0) {
    const int t = t0 + (lane & 31);
    return t < t_end ? c.table[b * c.table_stride + (t >> c.page_shift)] : -1;
  };
  // lanes 0..31: row of its token, and the exponent of K's row; 32..63: of V's
  struct Head {
    uint32_t row;
    int e;
    bool there;
  };
  auto head_of = [&](int t0, int page) {
    Head o;
    const int t = t0 + (lane & 31);
    o.there = (unsigned)page < (unsigned)c.n_pages;
    o.row = o.there ? (((uint32_t)page * c.heads + h) << c.page_shift) + (t & (c.page_size - 1)) : 0xffffffffu;
    o.e = o.there ? (lane < 32 ? c.k_exp : c.v_exp)[o.row] : 0;
    return o;
  };
  auto put_rows = [&](const Head &o) {
    wave_lds_order();
    if (lane < 32) mt.row[lane] = o.row;
    wave_lds_order();
  };
  auto load_tile = [&]() {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t row = mt.row[16 * i + l16];
      const char *p = c.k + ((uint64_t)row * D + g4 * KQ) * FB;
#pragma unroll
      for (int j = 0; j < KQ * FB / 16; ++j) {
        Bytes<16> part = {};
        if (row != 0xffffffffu && g4 * KQ + j * 16 / FB < D) load_bytes(part, p + 16 * j);
#pragma unroll
        for (int w = 0; w < 4; ++w) tile.k[i].w[4 * j + w] = part.w[w];
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t row = mt.row[(j >> 2) * 16 + 4 * g4 + (j & 3)];
      const char *p = c.v + ((uint64_t)row * D + l16 * VN) * FB;
      tile.v[j] = {};
      if (row != 0xffffffffu && l16 * VN < D) load_bytes(tile.v[j], p);
    }
  };

  int t0 = t_begin + wave * 32;
  Head head = {};
  int page_next = -1;
  if (t0 < t_end) {
    head = head_of(t0, page_of(t0));
    put_rows(head);
    load_tile();
    page_next = page_of(t0 + 128);
  }
  for (; t0 < t_end; t0 += 128) {
    // exponents of this tile
    {
      const bool nan = head.e == kExpNaN;
      wave_lds_order();
      if (lane < 32) {
        mt.k_scale[lane] = !head.there ? 0.f : nan ? NAN : ldexpf(1.f, head.e - 127);
      } else {
        const int e = min(max(head.e - e0, -100), 100);
        mt.v_exp[lane - 32] = !head.there ? -INFINITY : nan ? NAN : (float)e;
        mt.v_inv[lane - 32] = !head.there ? 1.f : ldexpf(1.f, -e);
      }
      wave_lds_order();
    }
    if (__any(lane >= 32 && head.there && head.e == kExpZero)) {
      // maybe a row of zeros, whose exponent says nothing about the others' and must not become the largest: 16 lanes hold its words
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t any = 0;
#pragma unroll
        for (int w = 0; w < VN * FB / 4; ++w) any |= tile.v[j].w[w] & (FMT == 8 ? 0x7f7f7f7fu : 0x7fff7fffu);
        const uint64_t held = __ballot(any != 0);
        const int t = (j >> 2) * 16 + 4 * g4 + (j & 3);
        if (l16 == 0 && !(held >> (16 * g4) & 0xffff) && fabsf(mt.v_exp[t]) < INFINITY) {
          mt.v_exp[t] = 0.f;
          mt.v_inv[t] = 1.f;
        }
      }
      wave_lds_order();
    }
    float ks[8], ve[8], vi[8];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        ks[4 * i + r] = mt.k_scale[16 * i + 4 * g4 + r];
        ve[4 * i + r] = mt.v_exp[16 * i + 4 * g4 + r];
        vi[4 * i + r] = mt.v_inv[16 * i + 4 * g4 + r];
      }
    // operands
    uintx4_t ka[2][KS];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        if constexpr (FMT == 8) {
          const uint32_t w0 = tile.k[i].w[2 * s], w1 = tile.k[i].w[2 * s + 1];
          ka[i][s] = uintx4_t{e4m3_lo(w0), e4m3_hi(w0), e4m3_lo(w1), e4m3_hi(w1)};
        } else {
          ka[i][s] = uintx4_t{tile.k[i].w[4 * s], tile.k[i].w[4 * s + 1], tile.k[i].w[4 * s + 2], tile.k[i].w[4 * s + 3]};
        }
      }
    uintx4_t va[VN];
#pragma unroll
    for (int jp = 0; jp < 4; ++jp) {
#pragma unroll
      for (int w = 0; w < VN * FB / 4; ++w) {
        const uint32_t lo = tile.v[2 * jp].w[w], hi = tile.v[2 * jp + 1].w[w];
        if constexpr (FMT == 8) {
          const uint32_t p0 = perm_b32(hi, lo, 0x05010400u), p1 = perm_b32(hi, lo, 0x07030602u);
          va[4 * w][jp] = e4m3_lo(p0);
          va[4 * w + 1][jp] = e4m3_hi(p0);
          va[4 * w + 2][jp] = e4m3_lo(p1);
          va[4 * w + 3][jp] = e4m3_hi(p1);
        } else {
          va[2 * w][jp] = perm_b32(hi, lo, 0x05040100u);
          va[2 * w + 1][jp] = perm_b32(hi, lo, 0x07060302u);
        }
      }
    }
    const bool masked = t0 + 32 > len;
    if (masked) {  // rows of padding, or of nodes that no query sees, hold anything: a p of zero must not meet a NaN or an infinity
#pragma unroll
      for (int i = 0; i < VN; ++i)
#pragma unroll
        for (int jp = 0; jp < 4; ++jp) va[i][jp] = finite_f16(va[i][jp]);
    }
    // the next tile's loads leave before this one's products
    Head head_next = {};
    const int t_next = t0 + 128;
    if (t_next < t_end) {
      head_next = head_of(t_next, page_next);
      put_rows(head_next);
      load_tile();
      page_next = page_of(t_next + 128);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      floatx4 s[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s[i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < QN; ++n)
#pragma unroll
          for (int k = 0; k < KS; ++k) s[i] = mfma16_f16(ka[i][k], q[m][n][k], s[i]);
      }
      float x[8];
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = fmaf(s[j >> 2][j & 3], ks[j] * q_scale[m], ve[j]);
      if (masked) {
        const int r = m * 16 + l16, node = first_q + (row0 + r) / a.group;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int at = t0 + (j >> 2) * 16 + 4 * g4 + (j & 3) - len;
          bool sees = at < 0;
          if (at >= 0 && at < a.tree) sees = a.parents ? (sh.mask[r][at >> 5] >> (at & 31)) & 1 : at <= node;
          x[j] = sees ? x[j] : -INFINITY;
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, x[j]);
      if (__any(top > M[m] + kSlack)) {
        float t = fmaxf(top, __shfl_xor(top, 16));
        t = fmaxf(t, __shfl_xor(t, 32));
        const float m_new = fmaxf(M[m], fminf(t, 3e38f)), alpha = __builtin_amdgcn_exp2f(M[m] - m_new);
        M[m] = m_new;
        sum[m] *= alpha;
#pragma unroll
        for (int i = 0; i < VN; ++i) acc[m][i] *= alpha;
      }
      float p[8];
      const float off = M[m] - kTop;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        p[j] = __builtin_amdgcn_exp2f(x[j] - off);
        sum[m] = fmaf(p[j], vi[j], sum[m]);
      }
      uintx4_t pb, pl;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t hi = pack_f16(p[2 * w], p[2 * w + 1]);
        pb[w] = hi;
        if constexpr (A::P2) pl[w] = pack_f16_rest(p[2 * w], p[2 * w + 1], hi);
      }
#pragma unroll
      for (int i = 0; i < VN; ++i) {
        acc[m][i] = mfma16_f16(va[i], pb, acc[m][i]);
        if constexpr (A::P2) acc[m][i] = mfma16_f16(va[i], pl, acc[m][i]);
      }
    }
    head = head_next;
  }

  // ---- the four waves' shares
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    float l = sum[m];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g4 == 0) {
      sh.m[wave][m * 16 + l16] = M[m];
      sh.l[wave][m * 16 + l16] = l;
    }
#pragma unroll
    for (int i = 0; i < VN; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) sh.o[wave][m * 16 + l16][(4 * g4 + r) * VN + i] = acc[m][i][r];
  }
  __syncthreads();
  const int64_t part_row = ((int64_t)split * a.B * c.heads + bh) * a.rows;
  for (int e = threadIdx.x; e < MT * 16 * (DP / 4); e += 256) {
    const int r = e / (DP / 4), d = e % (DP / 4) * 4, row = row0 + r;
    if (row >= a.rows) continue;
    float m_all = kMStart, l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) m_all = fmaxf(m_all, sh.m[w][r]);
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(sh.m[w][r] - m_all);
      l = fmaf(f, sh.l[w][r], l);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = fmaf(f, sh.o[w][r][d + j], o[j]);
    }
    const bool gone = treed && sh.gone[r];
    if (a.splits > 1) {
      if (d == 0) a.stat[part_row + row] = make_float2(m_all, gone ? -1.f : l);
      if (d < D) *reinterpret_cast<floatx4 *>(a.part + (part_row + row) * D + d) = o;
    } else if (d < D) {
      const int node = row / a.group, head_i = h * a.group + row % a.group;
      T *out = static_cast<T *>(a.out) + (((int64_t)b * a.n + node) * (c.heads * a.group) + head_i) * D + d;
      const float inv = gone || l == 0.f ? 0.f : 1.f / l;
      const float back = gone || l == 0.f ? 0.f : ldexpf(1.f, e0 - 127);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float y = back == 0.f ? 0.f : o[j] * inv * back;
        if constexpr (std::is_same<T, uint16_t>::value) out[j] = (uint16_t)pack_bf16_rne(y, y);
        else out[j] = (T)y;
      }
    }
  }
}

// ---- shares of the splits of a row: a block per 4 rows, a wave for each
template <typename TT>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a) {
  typedef typename TT::T T;
  const CacheView &c = a.c;
  const int lane = threadIdx.x & 63, D = c.dim;
  const int64_t all = (int64_t)a.B * c.heads * a.rows, at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= all) return;
  const int bh = (int)(at / a.rows), row = (int)(at - (int64_t)bh * a.rows), b = bh / c.heads, h = bh - b * c.heads;
  const int64_t room = (int64_t)c.width << c.page_shift;
  const int total = (int)min((int64_t)max(a.lens[b], 0) + a.tree, room);
  const int e0 = reference_exp(c, b, h, total);
  const int used = min(a.splits, (total + a.split_len - 1) / a.split_len);
  float m_all = kMStart, l = 0.f;
  bool gone = false;
  for (int s = lane; s < used; s += 64) {
    const float2 st = a.stat[s * all + at];
    m_all = fmaxf(m_all, st.x);
    gone |= st.y < 0.f;
  }
  m_all = wave_max(m_all);
  gone = __any(gone);
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  const int d = lane * 4;
  if (!gone)
    for (int s = 0; s < used; ++s) {
      const float2 st = a.stat[s * all + at];
      const float f = __builtin_amdgcn_exp2f(st.x - m_all);
      l = fmaf(f, st.y, l);
      if (d < D) o += f * *reinterpret_cast<const floatx4 *>(a.part + (s * all + at) * D + d);
    }
  if (d >= D) return;
  const int node = row / a.group, head_i = h * a.group + row % a.group;
  T *out = static_cast<T *>(a.out) + (((int64_t)b * a.n + node) * (c.heads * a.group) + head_i) * D + d;
  const bool none = gone || l == 0.f;
  const float inv = 1.f / l, back = ldexpf(1.f, e0 - 127);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float y = none ? 0.f : o[j] * inv * back;
    if constexpr (std::is_same<T, uint16_t>::value) out[j] = (uint16_t)pack_bf16_rne(y, y);
    else out[j] = (T)y;
  }
}

}  // namespace rb
