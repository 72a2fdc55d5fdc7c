// Attention of new tokens over the paged cache (rnnt_cache_attend).
#pragma once
#include "token_cache.h"

namespace rb {

// A block takes MT * 16 rows, a row being one query head of one node: the nodes of a sequence and the query heads that share a key head
// side by side, so that a tree's nodes and the heads of a group fill a tile and the cache is read once for all of them.  Its four waves
// take tiles of 32 tokens in turn; nothing goes through LDS but the tiles' exponents and row indices:
//   S^T = K Q^T   a lane loads every fourth 16 bytes of a key row as they lie in memory, the matrix instruction's 8-k slices being cut
//                 from those (Q is held in the same order); it gets the logits of 4 + 4 tokens for one row,
//   O^T = V^T P^T exactly which it hands back as the operand, again in an order of its own: k-slice j of lane group g is token 4 g + j
//                 of the first 16 and of the second.  V^T's operand are the same tokens' values of dim / 16 neighbouring dims, which a
//                 lane loads as they lie in memory and transposes in registers.
// Exponents: x = log2(e) scale q.k 2^(s_k) is the logit in base 2.  A value row's exponent is added to it: P' = 2^(x + s_v - M) is rounded to
// float16 and multiplied by y_v as stored, and the soft-max's denominator sums P' 2^(-s_v).  P' is at most 2^15 and the largest of a row at
// least 2^7: float16 keeps 11 bits of those down to 2^-21 of the largest.  Precision: Q is scaled by a power of two for each row and
// rounded to float16 (bfloat16 values down to 2^-28 of the row's largest are exact), float32 Q as a sum of two float16, and so is P', for all
// types: with one, whose 11 bits are less than float32 keeps, outputs in bfloat16 were rounded to a neighbour now and then; sums are float32.
// M follows the running maximum only when a logit passes it by 2^8 (the range that float16 leaves above), so that the accumulators are
// multiplied by a correction a few times in a row of thousands of tokens.
// Measured: one token for each of 32 sequences of 1000 to 8000, 32 heads on 8 of 128 in e4m3: 62 us and 4 for the join, 4.5 TB/s of a large copy's
// 5.3; bound by memory, a block's beginning (three dependent loads, 5 us) and the lengths' spread are the rest.  61 nodes for each of 16 sequences of 400 to 1900 tokens,
// 16 heads on 4 of 128, float32 on a cache of 16 bits: 51 us, 180 TFLOP/s of products: for a tile of 32 tokens and 32 rows a wave issues 64 products and
// some 350 vector instructions, half of the 5 000 cycles that a tile takes with two waves on a SIMD; the other half are waits, and a block's beginning
// and end, 17 000 and 6 000 cycles.  One sequence of 187 tokens: 7 us, a chain of loads.
struct AttendArgs {
  CacheView c;
  const void *q;
  void *out;  // [B][n][q_heads][dim]
  int64_t stride_b, stride_n, stride_h;  // of q, in elements
  const int *lens, *parents;             // parents [B][tree] or NULL: node i's is i - 1
  int B, n, tree, group;                 // queries are the last n of `tree` nodes
  int rows, row_tiles, splits, split_len;  // split_len: tokens, a multiple of 128
  float scale;
  float *part;      // [splits][B * heads][rows][dim]: outputs of a split's tokens
  float2 *stat;     // [splits][B * heads][rows]: (M, sum); a negative sum: the row's node is not there
  int join_shares;  // threads of the join for 4 values of a row
};

constexpr int kTreeMax = 1024;  // nodes of a tree with parents
constexpr float kMStart = -1e30f;
constexpr float kTop = 7.f;   // P' of the running maximum is 2^kTop
constexpr float kSlack = 8.f;
// Value exponents are relative to the head's first row's (reference_exp), and those of rows of zeros, which could be any, the lowest for which the range of
// float32 holds: with rows up to 2^45 on either side, of two that weigh alike the smaller's P' is 2^-90 of the larger's, which leaves 36 bits above 2^-126
// for what weighs less.
constexpr int kZeroRow = -45;

__device__ __forceinline__ uint32_t perm_b32(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }
__device__ __forceinline__ uint32_t e4m3_lo(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, false)); }
__device__ __forceinline__ uint32_t e4m3_hi(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.f, true)); }

// Value exponents are taken relative to one of the sequence's first rows, so that the sums of a block stay far from float32's ends: the first that
// tells anything (zero rows have kExpZero; padding nodes, and those below them, hold anything).  One call per wave; the same for all blocks of a
// sequence's head.
__device__ __forceinline__ int reference_page(const CacheView &c, int b) {  // of the lane's token, the lane-th
  return c.table[b * c.table_stride + min((int)(threadIdx.x & 63) >> c.page_shift, c.width - 1)];
}
__device__ __forceinline__ int reference_exp(const AttendArgs &a, int b, int h, int page, int len, int total) {
  const CacheView &c = a.c;
  const int lane = threadIdx.x & 63;
  bool there = lane < total && (unsigned)page < (unsigned)c.n_pages;
  const uint32_t row = there ? (((uint32_t)page * c.heads + h) << c.page_shift) + (lane & (c.page_size - 1)) : 0u;
  const int e = c.v_exp[row];
  if (a.parents && len < 64) {
    const int node = lane - len, p = node >= 0 && node < a.tree ? a.parents[(int64_t)b * a.tree + node] : -1;
    int padding = p < -1 || p >= max(node, 0), up = padding || p < 0 ? lane : len + p;
    for (int i = 0; i < 6; ++i) {  // (64 nodes: twice as far up each time)
      padding |= __shfl(padding, up);
      up = __shfl(up, up);
    }
    there = there && !padding;
  }
  const uint64_t good = __ballot(there && e != kExpZero && e != kExpNaN);
  return good ? __builtin_amdgcn_readlane(e, __ffsll((unsigned long long)good) - 1) : kExpZero;
}

// what two values rounded to float16 leave, rounded to float16
__device__ __forceinline__ uint32_t pack_f16_rest(float a, float b, uint32_t hi) {
  const f16x2_t h = __builtin_bit_cast(f16x2_t, hi);
  return pack_f16(fmaf((float)h[0], -1.f, a), fmaf((float)h[1], -1.f, b));  // (one mixed multiply-add each; exact)
}

// a pair of float16 with zeros in place of NaN and infinities
__device__ __forceinline__ uint32_t finite_f16(uint32_t w) {
  w = (w & 0x7c00u) == 0x7c00u ? w & 0xffff0000u : w;
  return (w & 0x7c000000u) == 0x7c000000u ? w & 0xffffu : w;
}

// whether one of a word's four e4m3 values, or of its two float16, is NaN or infinite: not zero
template <int FMT>
__device__ __forceinline__ uint32_t odd_codes(uint32_t w) {
  return FMT == 8 ? ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u : ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u;
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

__device__ __forceinline__ int64_t out_row(const AttendArgs &a, int b, int h, int row) {
  return (((int64_t)b * a.n + row / a.group) * (a.c.heads * a.group) + h * a.group + row % a.group) * a.c.dim;
}
// (from any address of their type: the hardware takes such stores whole)
__device__ __forceinline__ void put_output(float *p, floatx4 o) { __builtin_memcpy(p, &o, 16); }
__device__ __forceinline__ void put_output(_Float16 *p, floatx4 o) {
  const uint32_t w[2] = {pack_f16(o[0], o[1]), pack_f16(o[2], o[3])};
  __builtin_memcpy(p, w, 8);
}
__device__ __forceinline__ void put_output(uint16_t *p, floatx4 o) {
  const uint32_t w[2] = {pack_bf16_rne(o[0], o[1]), pack_bf16_rne(o[2], o[3])};
  __builtin_memcpy(p, w, 8);
}

// blocks of four waves that a compute unit holds, one wave of each on a SIMD: what the registers allow
constexpr int attend_blocks(int fmt, int dp, int mt) { return mt > 1 ? 2 : dp == 64 ? 4 : dp == 128 && fmt == 8 ? 3 : 2; }

template <typename TT, int FMT, int DP, int MT>
struct Attend {
  typedef typename TT::T T;
  static constexpr int FB = FMT / 8;                       // bytes of a kept value
  static constexpr bool Q2 = std::is_same<T, float>::value;        // Q as two float16
  static constexpr int KS = DP / 32;                       // k-steps of Q.K
  static constexpr int KQ = DP / 4;                        // values of a key row that a lane holds
  static constexpr int VN = DP / 16;                       // values of a value row that a lane holds
  static constexpr int QN = Q2 ? 2 : 1;

  struct Shared {
    union {
      struct {
        uint4 q[MT][QN][KS][64];  // operands of Q K, by lane
        uint32_t mask[MT * 16][kTreeMax / 32];
        int parents[kTreeMax];
      };
      float o[4][MT * 16][DP + 4];  // the waves' sums, when all have multiplied their last tile
    };
    float m[4][MT * 16], l[4][MT * 16];
    float q_scale[MT * 16];
    uint8_t gone[MT * 16];
  };
  struct Meta {  // of a wave's tile of 32 tokens
    uint32_t at[32];  // of the tokens' rows, in 16 bytes
    float k_scale[32], v_exp[32], v_inv[32];
  };
  // a lane's part of a tile: key rows l16 and 16 + l16, and its dims of eight value rows
  typedef Bytes<KQ * FB> Keys[2];
  typedef Bytes<VN * FB> Values[8];
  static constexpr int WAVES = attend_blocks(FMT, DP, MT);
};

template <typename TT, int FMT, int DP, int MT>
__global__ __launch_bounds__(256, (Attend<TT, FMT, DP, MT>::WAVES)) void k_attend(AttendArgs a) {
  using A = Attend<TT, FMT, DP, MT>;
  typedef typename A::T T;
  constexpr int KS = A::KS, KQ = A::KQ, VN = A::VN, FB = A::FB, QN = A::QN;
  __shared__ typename A::Shared sh;
  __shared__ typename A::Meta meta[4];
  const CacheView &c = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g4 = lane >> 4;

  // Blocks of the same tokens on one XCD, one after the other (block i runs on XCD i % 8); first splits first: which of the later ones have work
  // hangs on the lengths, and with the splits of a sequence side by side some XCDs had those that do not (32 sequences of 1000 to 8000 tokens: 78 us, now 66)
  const int groups = a.B * c.heads * a.splits;
  const int per = 8 * a.row_tiles, slab = blockIdx.x / per, in = blockIdx.x - slab * per;
  const int item = slab * 8 + (in & 7), tile_r = a.row_tiles - 1 - (in >> 3);  // the longest first
  if (item >= groups) return;
  const int pairs = a.B * c.heads, split = item / pairs, bh = item - split * pairs, b = bh / c.heads, h = bh - b * c.heads;
  const int row0 = tile_r * MT * 16;

  // ---- Q (a wave one tile's), parents and the first tokens' pages hang on nothing and leave first: a block begins with a chain of dependent
  // loads, lengths -> pages -> rows, of one to two microseconds each, and is otherwise a few times that long
  const int D = c.dim, q_tile = wave % MT;
  // lane (l16, g4) takes of row l16 of a tile what a key row has in its bytes 64 j + 16 g4 .. + 16
  const auto dim_of = [&](int s) { return FMT == 8 ? (s >> 1) * 64 + g4 * 16 + (s & 1) * 8 : s * 32 + g4 * 8; };
  T raw[KS][8];
  {
    const int r = row0 + q_tile * 16 + l16, node = r / a.group, head = h * a.group + r % a.group;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const bool there = r < a.rows && dim_of(s) < D;
      const T *p = static_cast<const T *>(a.q) + (there ? b * a.stride_b + node * a.stride_n + head * a.stride_h + dim_of(s) : 0);
      __builtin_memcpy(raw[s], p, sizeof(raw[s]));  // (the first row of all where there is none)
    }
  }
  int parent[kTreeMax / 256] = {};
  if (a.parents)
#pragma unroll
    for (int i = 0; i < kTreeMax / 256; ++i) parent[i] = a.parents[(int64_t)b * a.tree + min(i * 256 + (int)threadIdx.x, a.tree - 1)];
  const int ref_page = reference_page(c, b);

  const int64_t room = (int64_t)c.width << c.page_shift;
  const int len = max(a.lens[b], 0);
  const int total = (int)min((int64_t)len + a.tree, room);
  const int t_begin = (int)min((int64_t)split * a.split_len, (int64_t)total);
  const int t_split = split + 1 < a.splits ? (int)min((int64_t)t_begin + a.split_len, (int64_t)total) : total;
  if (split && t_begin >= t_split) return;

  const int first_q = a.tree - a.n;  // node of query 0
  const bool treed = a.parents && t_split > t_begin && (t_split > len || t_split == total);
  // no row of the block sees a node behind its last one's
  const int last_node = first_q + min((row0 + MT * 16 - 1) / a.group, a.n - 1);
  const int t_end = (int)min((int64_t)len + last_node + 1, (int64_t)t_split);

  floatx4 acc[MT][VN];
  float M[MT], sum[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    M[m] = kMStart;
    sum[m] = 0.f;
#pragma unroll
    for (int i = 0; i < VN; ++i) acc[m][i] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  typename A::Meta &mt = meta[wave];
  // Where a lane's part of a row lies: a lane whose dims a row does not have reads the first ones, against zeros of Q or for nothing.
  const char *k_from[KQ * FB / 16];
#pragma unroll
  for (int j = 0; j < KQ * FB / 16; ++j) k_from[j] = c.k + (64 * j + 16 * g4 < D * FB ? 64 * j + 16 * g4 : 0);
  const char *const v_from = c.v + (l16 * VN < D ? l16 * VN * FB : 0);
  const int row_bytes = D * FB;
  // Loads are never left out: those of tokens that are not there read row 0 of the cache.  A load behind a branch would make every wait one for all
  // loads under way, the next tile's among them.
  struct Head {  // lanes 0..31 and 32..63: the 32 tokens of a tile; row, exponent of K's row (lanes 32..63: of V's)
    uint32_t row;
    int e;
    bool there;
  };
  auto page_of = [&](int t0) { return c.table[b * c.table_stride + (min(t0 + (lane & 31), t_end - 1) >> c.page_shift)]; };
  const uint8_t *exps = lane < 32 ? c.k_exp : c.v_exp;
  // row indices of a tile, for load_keys and load_values behind it
  auto head_of = [&](int t0, int page) {
    Head o;
    const int t = t0 + (lane & 31);
    o.there = t < t_end && (unsigned)page < (unsigned)c.n_pages;
    o.row = o.there ? (((uint32_t)page * c.heads + h) << c.page_shift) + (t & (c.page_size - 1)) : 0u;
    wave_lds_order();
    if (lane < 32) mt.at[lane] = o.row * (uint32_t)(row_bytes >> 4);
    wave_lds_order();
    o.e = exps[o.row];
    return o;
  };
  auto load_keys = [&](typename A::Keys &keys) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint64_t at = (uint64_t)mt.at[16 * i + l16] << 4;
#pragma unroll
      for (int j = 0; j < KQ * FB / 16; ++j) {
        Bytes<16> part;
        load_bytes(part, k_from[j] + at);
#pragma unroll
        for (int w = 0; w < 4; ++w) keys[i].w[4 * j + w] = part.w[w];
      }
    }
  };
  auto load_values = [&](typename A::Values &values) {
#pragma unroll
    for (int j = 0; j < 8; ++j) load_bytes(values[j], v_from + ((uint64_t)mt.at[(j >> 2) * 16 + 4 * g4 + (j & 3)] << 4));
  };

  // ---- the first tile's loads leave ahead of everything that does not need them
  int t0 = t_begin + wave * 32;
  const bool busy = t0 < t_end;
  typename A::Keys keys;
  typename A::Values values;
  Head head[2] = {};
  int page_next = 0;
  if (busy) {
    const int page = page_of(t0);
    page_next = page_of(t0 + 128);
    head[0] = head_of(t0, page);
    load_keys(keys);
    load_values(values);
  }
  const int e0 = reference_exp(a, b, h, ref_page, len, total);

  {
    const int r = row0 + q_tile * 16 + l16;
    float most = 0.f;
    bool bad = false;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const bool there = r < a.rows && dim_of(s) < D;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!there) raw[s][j] = 0;
        most = fmaxf(most, fabsf(to_float(raw[s][j])));
        bad |= !(fabsf(to_float(raw[s][j])) < INFINITY);
      }
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    bad = __shfl_xor((int)bad, 16) | (int)bad;
    bad = __shfl_xor((int)bad, 32) | (int)bad;
    // the row's largest to [2^14, 2^15)
    const int e = min(max((int)(__float_as_uint(most) >> 23), 15), 254);
    const float to = __uint_as_float((uint32_t)(268 - e) << 23);
    if (g4 == 0 && wave < MT) sh.q_scale[q_tile * 16 + l16] = bad ? NAN : __uint_as_float((uint32_t)(e - 14) << 23) * a.scale * (float)kLog2E;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      if (s % (4 / MT) != wave / MT) continue;  // the waves of a tile share its steps
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float u = bad ? 0.f : to_float(raw[s][2 * w]) * to, v = bad ? 0.f : to_float(raw[s][2 * w + 1]) * to;
        hi[w] = pack_f16(u, v);
        if constexpr (A::Q2) lo[w] = pack_f16_rest(u, v, hi[w]);
      }
      sh.q[q_tile][0][s][lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      if constexpr (A::Q2) sh.q[q_tile][1][s][lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
  }

  // ---- which nodes a row sees, where the block's tokens reach into the tree
  if (treed) {
    // (the walk is a chain of dependent reads: through LDS)
    const int words = (a.tree + 31) >> 5;
    for (int i = threadIdx.x; i < MT * 16 * words; i += 256) sh.mask[i / words][i % words] = 0;
#pragma unroll
    for (int i = 0; i < kTreeMax / 256; ++i) sh.parents[i * 256 + threadIdx.x] = parent[i];
    __syncthreads();
    if (threadIdx.x < MT * 16) {
      const int r = row0 + threadIdx.x;
      bool gone = false;
      if (r < a.rows) {
        int j = first_q + r / a.group;
        while (true) {
          sh.mask[threadIdx.x][j >> 5] |= 1u << (j & 31);
          const int p = sh.parents[j];
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
  }
  __syncthreads();
  float q_scale[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) q_scale[m] = sh.q_scale[m * 16 + l16];

  // one tile; `next_keys` and `next_values` are called when its registers may be written again
  auto take_tile = [&](int t0, const Head &head, const typename A::Keys &keys, const typename A::Values &values, auto next_keys, auto next_values) {
    // tiles that reach beyond the tokens kept before, or hold tokens that are not there
    const bool careful = t0 + 32 > len || __any(!head.there);
    {
      const bool nan = head.e == kExpNaN;
      const int e = min(max(head.e - e0, -100), 100);
      wave_lds_order();
      if (lane < 32) {
        mt.k_scale[lane] = nan ? NAN : ldexpf(1.f, head.e - 127);
      } else {
        mt.v_exp[lane - 32] = !head.there ? -INFINITY : nan ? NAN : (float)e;
        mt.v_inv[lane - 32] = ldexpf(1.f, -e);
      }
      wave_lds_order();
      if (__any(lane >= 32 && head.there && head.e == kExpZero)) {
        // maybe a row of zeros, whose P' must not push those of smaller rows beyond float16's range, since it adds nothing: 16 lanes hold its words
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint32_t any = 0;
#pragma unroll
          for (int w = 0; w < VN * FB / 4; ++w) any |= values[j].w[w] & (FMT == 8 ? 0x7f7f7f7fu : 0x7fff7fffu);
          const uint64_t held = __ballot(any != 0);
          const int t = (j >> 2) * 16 + 4 * g4 + (j & 3);
          if (l16 == 0 && !(held >> (16 * g4) & 0xffff) && fabsf(mt.v_exp[t]) < INFINITY) {
            mt.v_exp[t] = (float)kZeroRow;
            mt.v_inv[t] = __uint_as_float((uint32_t)(127 - kZeroRow) << 23);
          }
        }
        wave_lds_order();
      }
    }
    // Values that are not finite, in arrays that the caller filled, make their row one of NaN.  Where all rows are seen they reach the sums by
    // themselves; elsewhere they must not meet the p of zero of a query that does not see them, nor may what rows that are not there hold.
    bool odd = false;
    if (careful) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t any = 0;
#pragma unroll
        for (int w = 0; w < VN * FB / 4; ++w) any |= odd_codes<FMT>(values[j].w[w]);
        const uint64_t held = __ballot(any != 0);
        if (!held) continue;
        odd = true;
        const int t = (j >> 2) * 16 + 4 * g4 + (j & 3);
        if (l16 == 0 && (held >> (16 * g4) & 0xffff) && fabsf(mt.v_exp[t]) < INFINITY) mt.v_exp[t] = NAN;
      }
      if (odd) wave_lds_order();
    }
    floatx4 ks[2], ve[2], vi[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ks[i] = *reinterpret_cast<const floatx4 *>(&mt.k_scale[16 * i + 4 * g4]);
      ve[i] = *reinterpret_cast<const floatx4 *>(&mt.v_exp[16 * i + 4 * g4]);
      vi[i] = *reinterpret_cast<const floatx4 *>(&mt.v_inv[16 * i + 4 * g4]);
    }
    floatx4 s[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m) s[m][0] = s[m][1] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uintx4_t ka;
        if constexpr (FMT == 8) {
          const uint32_t w0 = keys[i].w[2 * k], w1 = keys[i].w[2 * k + 1];
          ka = uintx4_t{e4m3_lo(w0), e4m3_hi(w0), e4m3_lo(w1), e4m3_hi(w1)};
        } else {
          ka = uintx4_t{keys[i].w[4 * k], keys[i].w[4 * k + 1], keys[i].w[4 * k + 2], keys[i].w[4 * k + 3]};
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int n = 0; n < QN; ++n) s[m][i] = mfma16_f16(ka, __builtin_bit_cast(uintx4_t, sh.q[m][n][k][lane]), s[m][i]);
      }
    next_keys();
    uintx4_t pb[MT], pl[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float x[8];
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = fmaf(s[m][j >> 2][j & 3], ks[j >> 2][j & 3] * q_scale[m], ve[j >> 2][j & 3]);
      if (careful) {
        const int r = m * 16 + l16, node = first_q + (row0 + r) / a.group;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int at = t0 + (j >> 2) * 16 + 4 * g4 + (j & 3) - len;
          bool sees = at < 0;
          if (at >= 0 && at < a.tree) sees = a.parents ? (sh.mask[r][at >> 5] >> (at & 31)) & 1 : at <= node;
          x[j] = sees && ve[j >> 2][j & 3] != -INFINITY ? x[j] : -INFINITY;
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
        sum[m] = fmaf(p[j], vi[j >> 2][j & 3], sum[m]);
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t hi = pack_f16(p[2 * w], p[2 * w + 1]);
        pb[m][w] = hi;
        pl[m][w] = pack_f16_rest(p[2 * w], p[2 * w + 1], hi);
      }
    }
    // four (two) dims at a time: the words of eight tokens that hold them, transposed
#pragma unroll
    for (int w = 0; w < VN * FB / 4; ++w) {
      constexpr int PER = 4 / FB;
      uintx4_t va[PER];
#pragma unroll
      for (int jp = 0; jp < 4; ++jp) {
        const uint32_t lo = values[2 * jp].w[w], hi = values[2 * jp + 1].w[w];
        if constexpr (FMT == 8) {
          const uint32_t p0 = perm_b32(hi, lo, 0x05010400u), p1 = perm_b32(hi, lo, 0x07030602u);
          va[0][jp] = e4m3_lo(p0);
          va[1][jp] = e4m3_hi(p0);
          va[2][jp] = e4m3_lo(p1);
          va[3][jp] = e4m3_hi(p1);
        } else {
          va[0][jp] = perm_b32(hi, lo, 0x05040100u);
          va[1][jp] = perm_b32(hi, lo, 0x07060302u);
        }
      }
      if (odd) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
          for (int jp = 0; jp < 4; ++jp) va[i][jp] = finite_f16(va[i][jp]);
      }
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          acc[m][PER * w + i] = mfma16_f16(va[i], pb[m], acc[m][PER * w + i]);
          acc[m][PER * w + i] = mfma16_f16(va[i], pl[m], acc[m][PER * w + i]);
        }
    }
    next_values();
  };

  if (busy) {
    // one tile in registers, whose keys are followed by the next ones when they have been multiplied, and its values likewise
    do {
      head[1] = head_of(t0 + 128, page_next);
      page_next = page_of(t0 + 256);
      take_tile(t0, head[0], keys, values, [&] { load_keys(keys); }, [&] { load_values(values); });
      head[0] = head[1];
      t0 += 128;
    } while (t0 < t_end);
  }

  // ---- the four waves' shares
  __syncthreads();
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
    // (a row's DP / 4 lanes: all of its values are NaN if one of the rows it sees has one that is not finite)
    const bool finite = fabsf(o[0]) < INFINITY && fabsf(o[1]) < INFINITY && fabsf(o[2]) < INFINITY && fabsf(o[3]) < INFINITY;
    const uint64_t others = ~0ull >> (64 - DP / 4) << (lane & ~(DP / 4 - 1));
    const bool gone = treed && sh.gone[r], none = gone || l == 0.f;
    const float inv = __ballot(!finite) & others ? NAN : 1.f / l, back = ldexpf(1.f, e0 - 127);
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = none ? 0.f : o[j] * inv * back;
    if (a.splits > 1 && d == 0) a.stat[part_row + row] = make_float2(m_all, gone ? -1.f : l);
    if (d >= D) continue;
    if (a.splits == 1) put_output(static_cast<T *>(a.out) + out_row(a, b, h, row) + d, o);
    else *reinterpret_cast<floatx4 *>(a.part + (part_row + row) * D + d) = o;
  }
}

// ---- the splits of a row: `join_shares` threads for 4 values of it, each a split at a time.  4 to 5 us, a launch and two loads
template <typename TT>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a) {
  typedef typename TT::T T;
  __shared__ floatx4 sh_o[256];
  __shared__ float2 sh_s[256];
  const CacheView &c = a.c;
  const int D = c.dim, lanes = D / 4, per_row = lanes * a.join_shares, rows = 256 / per_row;
  const int64_t all = (int64_t)a.B * c.heads * a.rows;
  const int r = threadIdx.x / per_row, mine = threadIdx.x % per_row / lanes, d = threadIdx.x % lanes * 4;
  const int64_t at = (int64_t)blockIdx.x * rows + r;
  const bool there = r < rows && at < all;
  const int bh = there ? (int)(at / a.rows) : 0, b = bh / c.heads;
  float m = kMStart, l = 0.f;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  bool gone = false;
  if (there) {
    const int64_t total = min((int64_t)max(a.lens[b], 0) + a.tree, (int64_t)c.width << c.page_shift);
    const int used = (int)min((int64_t)a.splits, (total + a.split_len - 1) / a.split_len);
#pragma unroll 4
    for (int s = mine; s < used; s += a.join_shares) {
      const int64_t from = s * all + at;
      const float2 st = a.stat[from];
      const floatx4 part = *reinterpret_cast<const floatx4 *>(a.part + from * D + d);
      gone |= st.y < 0.f;
      const float m_new = fmaxf(m, st.x), keep = __builtin_amdgcn_exp2f(m - m_new), add = st.y * __builtin_amdgcn_exp2f(st.x - m_new);
      l = fmaf(l, keep, add);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = fmaf(o[j], keep, add * part[j]);
      m = m_new;
    }
  }
  if (a.join_shares > 1) {
    sh_o[threadIdx.x] = o;
    sh_s[threadIdx.x] = make_float2(m, gone ? -1.f : l);
    __syncthreads();
    if (mine) return;
    for (int i = 1; there && i < a.join_shares; ++i) {
      const float2 st = sh_s[threadIdx.x + i * lanes];
      gone |= st.y < 0.f;
      const float m_new = fmaxf(m, st.x), keep = __builtin_amdgcn_exp2f(m - m_new), add = __builtin_amdgcn_exp2f(st.x - m_new);
      l = fmaf(l, keep, add * st.y);
      o = o * keep + sh_o[threadIdx.x + i * lanes] * add;
      m = m_new;
    }
  }
  if (!there) return;
  const bool none = gone || l == 0.f;
  const float inv = 1.f / l;
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = none ? 0.f : o[j] * inv;
  put_output(static_cast<T *>(a.out) + out_row(a, b, bh - b * c.heads, (int)(at - (int64_t)bh * a.rows)) + d, o);
}

}  // namespace rb
