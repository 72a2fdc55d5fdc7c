// Selection of a beam's best tokens from logits that the caller computed, and the reordering of states by the parents it
// names (rnnt_select_tokens, rnnt_reorder_states).
#pragma once
#include "token_types.h"

namespace rb {

// ---- soft-max statistics in float64
// The keys of an utterance's hypotheses are compared with each other, and the sums of rows decide between candidates whose logits differ by
// little: float32 exponentials leave 1e-8 to 1e-7 of a row's log sum open.  float64 multiply-adds run at the rate of float32 ones here, so
// the exponential is a polynomial in float64: e^d = 2^n e^f with n = d / ln 2 rounded, and for e^f the polynomial of degree 10 through the
// Chebyshev points of [-ln 2 / 2, ln 2 / 2], off by at most 3.3e-16 of its value, three half steps of float64 (degree 7 would leave 5.5e-11, and keys
// off by 1e-12 to 2e-11; 128 x 10 x 8192 logits take 20.3 us for 19.4).  Of float64 only sums and multiply-adds run at that rate: n is
// read from the last bits of d / ln 2 + 1.5 2^52 and added to the exponent of e^f, in place of instructions that round, convert and scale.
__device__ __forceinline__ double exp_d(double d) {  // d up to 700
  constexpr double kRound = 6755399441055744.;
  d = fmax(d, -690.);  // (of -inf too: e^-690 is nothing beside the 1 of the largest)
  const double s = fma(d, kLog2E, kRound), f = fma(s - kRound, -0.6931471805599453, d);
  double p = 2.7626357241447223e-07;
  p = fma(p, f, 2.764018079620985e-06);
  p = fma(p, f, 2.4801504346997686e-05);
  p = fma(p, f, 0.00019841170270440067);
  p = fma(p, f, 0.0013888888932488599);
  p = fma(p, f, 0.008333333385667782);
  p = fma(p, f, 0.04166666666657314);
  p = fma(p, f, 0.16666666666554406);
  p = fma(p, f, 0.5000000000000006);
  p = fma(p, f, 1.0000000000000067);
  p = fma(p, f, 1.0);
  return __hiloint2double(__double2hiint(p) + (__double2loint(s) << 20), __double2loint(p));
}

constexpr int kSelBuf = 64;    // candidates that a wave ranks at a time: one per lane
constexpr int kSelLists = 64;  // lists that a wave joins: one per lane

// a logit and its index as one number (zeros of both signs are equal)
__device__ __forceinline__ uint64_t make_cand(float v, int i) { return pack_cand(v + 0.f, i); }

// What a wave knows of its part of a row: the `beam` best logits, in lanes 0 .. beam - 1 in order (no_cand() behind the last), and
// sum exp(x - ref), each lane's share of it.
struct RowPart {
  uint64_t best = no_cand();
  double sum = 0.;
  float ref = -INFINITY;
  bool bad = false;  // a NaN or +inf among them (of this lane)
};

// The maxima of 32 groups of logits as whole numbers, made different by their group's number in the last bits: a little smaller, which
// a bound may be.
struct alignas(16) GroupKeys {
  uint32_t k[32];
};
__device__ __forceinline__ uint32_t group_key(float v, int group) { return (orderable(v) & ~31u) | group; }
// what the `nth` (1 ..) largest of them reaches, as orderable() has it
__device__ __forceinline__ uint32_t nth_group(const GroupKeys &g, int nth) {
  const int lane = threadIdx.x & 63;
  const uint32_t key = g.k[lane & 31];
  int rank = 0;  // half a wave compares with half of the groups
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint4 o = reinterpret_cast<const uint4 *>(g.k)[(lane >> 5) * 4 + j];
    rank += (int)(o.x > key) + (int)(o.y > key) + (int)(o.z > key) + (int)(o.w > key);
  }
  rank += __shfl_xor(rank, 32);
  return __builtin_amdgcn_readlane((int)key, __ffsll((unsigned long long)__ballot(rank == nth - 1)) - 1) & ~31u;
}

struct alignas(16) CandBuf {
  uint64_t c[kSelBuf];
  GroupKeys group;
};

// The first n places of the buffer hold candidates: the best `beam` of them go to its first places in order, no_cand() behind the last.
__device__ __forceinline__ uint64_t rank_candidates(int n, int beam, CandBuf &buf) {
  const int lane = threadIdx.x & 63;
  wave_lds_order();
  if (lane >= n) buf.c[lane] = 0;
  wave_lds_order();
  const uint64_t own = buf.c[lane];
  int rank = 0;
  for (int j = 0; j < n; j += 8)
#pragma unroll
    for (int u = 0; u < 8; ++u) rank += buf.c[j + u] > own;
  wave_lds_order();
  if (lane < beam) buf.c[lane] = no_cand();  // (equal ones, places without a candidate, have one rank)
  wave_lds_order();
  if (lane < n && rank < beam) buf.c[rank] = own;
  wave_lds_order();
  const uint64_t out = lane < beam ? buf.c[lane] : no_cand();
  wave_lds_order();
  return out;
}

// One tile of 64 * E logits of a row from index `base` on, lane l's in x: adds them to the sum and the list.
// The list: a bound that the `beam` best reach is the beam-th largest of the maxima of 32 pairs of lanes, or what the list holds already; those logits that
// reach it, few more than `beam` as a rule, are collected and ranked.  Where more than a wave ranks at a time reach it (many equal
// logits), the best are taken out one after the other instead.
template <int E, int VE>
__device__ __forceinline__ void take_tile(const float (&x)[E], int base, int beam, RowPart &part, CandBuf &buf) {
  const int lane = threadIdx.x & 63;
  auto index = [&](int e) { return base + (e / VE) * 64 * VE + lane * VE + e % VE; };
  float top = x[0];
  bool bad = false;
#pragma unroll
  for (int e = 1; e < E; ++e) top = fmaxf(top, x[e]);
#pragma unroll
  for (int e = 0; e + 1 < E; e += 2) bad |= __builtin_isunordered(x[e], x[e + 1]);
  if constexpr (E % 2) bad |= __builtin_isunordered(x[E - 1], x[E - 1]);
  part.bad |= bad || top == INFINITY;
  const float most = wave_max(top);
  if (!(most > -INFINITY)) return;
  if (!(most < part.ref + 500.f)) {  // (the first tile too; float64 holds exp(500) times exp(200) more)
    const float ref = most < INFINITY ? most : 0.f;
    part.sum *= part.ref == -INFINITY ? 0. : exp((double)part.ref - ref);
    part.ref = ref;
  }
  const double ref = part.ref;
#pragma unroll
  for (int e = 0; e < E; ++e) part.sum += exp_d((double)x[e] - ref);

  const float last = readlane_f(cand_key(part.best), beam - 1);
  if (!(most > last)) return;  // equal ones come after those of the list, whose indices are smaller
  const float pair = fmaxf(top, dpp_f<kDppXor1>(top));
  wave_lds_order();
  if (!(lane & 1)) buf.group.k[lane >> 1] = group_key(pair, lane >> 1);
  wave_lds_order();
  const uint32_t nth = nth_group(buf.group, beam), after = orderable(last) + 1;
  const float bound = from_orderable(nth > after ? nth : after);
  int n = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const uint64_t at = __ballot(x[e] >= bound);
    if (at) {
      const int pos = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(at >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)at, 0));
      if (x[e] >= bound && pos < kSelBuf) buf.c[pos] = make_cand(x[e], index(e));
      n += __popcll(at);
    }
  }
  const int held = __popcll(__ballot(lane < beam && part.best > no_cand()));
  if (n + held > kSelBuf) {
    uint32_t taken = 0;
    n = 0;
    while (n < beam) {
      float v = -INFINITY;
      int i = 0x7fffffff, at = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const bool better = !(taken >> e & 1) && x[e] > v;
        v = better ? x[e] : v;
        i = better ? index(e) : i;
        at = better ? e : at;
      }
      const int own = i;
      wave_best(v, i);
      if (!(v > last)) break;
      if (own == i) taken |= 1u << at;
      wave_lds_order();
      if (lane == 0) buf.c[n] = make_cand(v, i);
      ++n;
    }
  }
  wave_lds_order();
  if (lane < held) buf.c[n + lane] = part.best;
  part.best = rank_candidates(n + held, beam, buf);
}

// A wave's part [begin, end) of a row.
template <typename T, int E>
__device__ __forceinline__ void scan_row(const T *row, int begin, int end, int beam, RowPart &part, CandBuf &buf) {
  constexpr int VE = 16 / sizeof(T), NV = E / VE;
  const int lane = threadIdx.x & 63;
  for (int base = begin; base < end; base += 64 * E) {
    float x[E];
    if (base + 64 * E <= end) {
      T raw[NV][VE];
#pragma unroll
      for (int i = 0; i < NV; ++i) load16(row + base + i * 64 * VE + lane * VE, raw[i]);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VE; ++j) x[i * VE + j] = to_float(raw[i][j]);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = base + i * 64 * VE + lane * VE;
        if (at + VE <= end) {
          T raw[VE];
          load16(row + at, raw);
#pragma unroll
          for (int j = 0; j < VE; ++j) x[i * VE + j] = to_float(raw[j]);
        } else {
#pragma unroll
          for (int j = 0; j < VE; ++j) x[i * VE + j] = at + j < end ? to_float(row[at + j]) : -INFINITY;
        }
      }
    }
    take_tile<E, VE>(x, base, beam, part, buf);
  }
}

__device__ __forceinline__ double wave_sum_d(double v) {
  v += dpp_d<kDppXor1>(v);
  v += dpp_d<kDppXor2>(v);
  v += dpp_d<kDppHalfMirror>(v);
  v += dpp_d<kDppMirror>(v);
  return (readlane_d(v, 0) + readlane_d(v, 16)) + (readlane_d(v, 32) + readlane_d(v, 48));
}

// A list as it is handed on: the best of a part of a row and the sum of its exponentials.
struct SelList {
  uint64_t c[kMaxBeam];
};
struct SelStat {
  double sum;  // NaN: a NaN or +inf among the logits
  float ref;   // -inf: all logits were
  int pad;
};

struct SelectArgs {
  const void *logits;
  int64_t stride_b, stride_k;
  const double *scores;
  const uint8_t *done;
  double *out_scores;
  int *out_parent, *out_token;
  uint8_t *out_done;
  SelList *lists;  // [B][beam][parts]
  SelStat *stats;
  int B, beam, V, eos, parts, part_len;
};

struct alignas(16) SelJoin {
  float low[64];  // the first few of every list, rounded down
  double key[kSelLists * kMaxBeam];  // of the candidates
  int token[kSelLists * kMaxBeam];
  float x[kSelLists * kMaxBeam];
  uint8_t k[kSelLists * kMaxBeam];
  double sum[kSelLists];
  float ref[kSelLists];
};

// One wave: the `beam` best of an utterance from the lists of its rows, lane l's being list l = k * parts + p.  A bound that they reach is the
// beam-th largest of the first few of every list; each lane hands on those of its list that reach it, and they are
// ranked by (key descending, hypothesis, logit descending, token): lists hold the largest logits, whose keys may round to one float64.
__device__ __forceinline__ void join_lists(const SelectArgs &a, int b, const SelList *lists, const SelStat *stats, SelJoin &sh) {
  const int lane = threadIdx.x & 63, beam = a.beam, parts = a.parts, n_lists = beam * parts;
  const int l = min(lane, n_lists - 1), k = l / parts;
  // everything that is read leaves at once (what a finished hypothesis' lists hold is not looked at)
  const SelStat st = stats[l];
  uint64_t c[kMaxBeam];
  __builtin_memcpy(c, lists[l].c, sizeof(c));
  const double score = a.scores[(int64_t)b * beam + k];
  const bool finished = a.done && a.done[(int64_t)b * beam + k];
  // log sum exp of the row
  float ref = st.ref;
  double sum = st.sum;
  if (parts > 1) {
    sh.ref[lane] = ref;
    wave_lds_order();
    for (int p = 0; p < parts; ++p) ref = fmaxf(ref, sh.ref[k * parts + p]);
    // (a part that held nothing but -inf, or NaN: its sum is 0, or NaN, whatever it is multiplied by)
    sh.sum[lane] = st.ref > -INFINITY ? sum * exp((double)st.ref - ref) : sum;
    wave_lds_order();
    sum = 0.;
    for (int p = 0; p < parts; ++p) sum += sh.sum[k * parts + p];
  }
  const double lse = (double)ref + log(sum);
  if (finished) c[0] = lane == k * parts ? make_cand(0.f, a.eos) : no_cand();  // its one candidate: eos, with the score that it has
  // (a list's keys descend; NaN is none)
  const auto key_of = [&](int j) {
    const double key = finished ? score : score + ((double)cand_key(c[j]) - lse);
    return c[j] > no_cand() && key > -INFINITY && (j == 0 || !finished) && lane < n_lists ? key : -INFINITY;
  };
  // the bound, in float32 rounded down (a list has `beam` places, what lies behind them nobody wrote)
  const int firsts = min(max(min(64, 4 * beam) / n_lists, 1), beam);
  sh.low[lane] = -INFINITY;
  wave_lds_order();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float one = (float)key_of(j);
    if (j < firsts && lane < n_lists && one > -INFINITY) sh.low[lane * firsts + j] = from_orderable(orderable(one) - 1);  // (-inf for what float32 has no number for)
  }
  wave_lds_order();
  const float low = sh.low[lane];
  int before = 0;
  for (int j = 0; j < n_lists * firsts; j += 8)
#pragma unroll
    for (int u = 0; u < 8; ++u) before += sh.low[j + u] > low;
  const double bound = -wave_max(before < beam ? -low : -INFINITY);
  int n = 0;
#pragma unroll
  for (int j = 0; j < kMaxBeam; ++j) {
    const double key = j < beam ? key_of(j) : -INFINITY;
    const bool in = key > -INFINITY && key >= bound;
    const uint64_t at = __ballot(in);
    if (!at) break;
    if (in) {
      const int pos = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(at >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)at, 0));
      sh.key[pos] = key;
      sh.token[pos] = cand_idx(c[j]);
      sh.x[pos] = cand_key(c[j]);
      sh.k[pos] = (uint8_t)k;
    }
    n += __popcll(at);
  }
  wave_lds_order();
  const int64_t out = (int64_t)b * beam;
  for (int p = lane; p < n; p += 64) {
    const double key = sh.key[p];
    const float x = sh.x[p];
    const int token = sh.token[p], parent = sh.k[p];
    int r = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
      const double other = sh.key[j];
      r += other > key;
      if (other == key && j != p) r += sh.k[j] != parent ? sh.k[j] < parent : sh.x[j] != x ? sh.x[j] > x : sh.token[j] < token;
    }
    if (r >= beam) continue;
    a.out_scores[out + r] = key;
    a.out_parent[out + r] = parent;
    a.out_token[out + r] = token;
    if (a.out_done) a.out_done[out + r] = token == a.eos;
  }
  for (int r = n + lane; r < beam; r += 64) {  // empty slots
    a.out_scores[out + r] = -INFINITY;
    a.out_parent[out + r] = -1;
    a.out_token[out + r] = -3;
    if (a.out_done) a.out_done[out + r] = 0;
  }
}

__device__ __forceinline__ void put_list(const RowPart &part, double sum, bool bad, int beam, SelList &list, SelStat &stat) {
  const int lane = threadIdx.x & 63;
  if (lane < beam) list.c[lane] = part.best;
  if (lane == 0) stat = SelStat{bad ? (double)NAN : sum, part.ref, 0};
}

// ---- everything of an utterance in one block of 16 waves, parts = 16 / beam of them for a row: no workspace, one launch.  Bound by the chain
// of its steps (load, sums, bound, ranking, the same again for the join), each of a few hundred to 1500 cycles: 6 us for 4 x 1024.
template <typename TT, int NV>
__global__ __launch_bounds__(1024) void k_select_one(SelectArgs a) {
  typedef typename TT::T T;
  __shared__ SelJoin sh;
  __shared__ SelList list[16];
  __shared__ SelStat stat[16];
  __shared__ CandBuf buf[16];
  const int b = blockIdx.x, wave = threadIdx.x >> 6, k = wave / a.parts, p = wave - k * a.parts;
  if (k < a.beam) {
    RowPart part;
    if (!(a.done && a.done[(int64_t)b * a.beam + k])) {
      const T *row = static_cast<const T *>(a.logits) + b * a.stride_b + k * a.stride_k;
      const int begin = min(p * a.part_len, a.V);
      scan_row<T, NV * 16 / sizeof(T)>(row, begin, min(begin + a.part_len, a.V), a.beam, part, buf[wave]);
    }
    const double sum = wave_sum_d(part.sum);
    put_list(part, sum, __any(part.bad), a.beam, list[wave], stat[wave]);
  }
  __syncthreads();
  if (wave == 0) join_lists(a, b, list, stat, sh);
}

// ---- many blocks for a row: each leaves the best of its part, a second launch joins them.  A block's four waves take tiles of 256 E logits
// together: a bound that the `beam` best of a tile reach is the beam-th largest of the maxima of 32 groups of 8 lanes; of the logits
// that reach it and what earlier tiles left, rarely more than twice `beam`, one wave takes the best.
// Measured: 128 x 10 x 8192 logits of 16 bits in 15 us (read at 5.3 TB/s they would take 4), 32 x 12 x 32003 of 32, a fifth of the rows finished, in 19 (7.4).  Of the 15 some 5 go
// into the float64 exponentials (19 instructions for a logit), 3 each into the first loads, which all blocks wait for at once, and into finding
// and ranking the candidates.  Five blocks share a unit: what keeps the registers to 96, with 80 some are spilt, which costs 1.7.
struct SelScan {
  float group[32];
  GroupKeys group_key;
  CandBuf buf;  // the list, in its first `beam` places, and what a tile adds
  int n;
  CandBuf wave_buf[4];
  SelList list[4];
  SelStat stat[4];
};

template <typename TT, int E>
__global__ __launch_bounds__(256, 5) void k_select_scan(SelectArgs a) {
  typedef typename TT::T T;
  constexpr int VE = 16 / sizeof(T), NV = E / VE;
  __shared__ SelScan sh;
  const int p = blockIdx.x % a.parts, row_i = blockIdx.x / a.parts, b = row_i / a.beam, k = row_i - b * a.beam, beam = a.beam;
  if (a.done && a.done[row_i]) return;  // (the join takes nothing from its lists)
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const T *row = static_cast<const T *>(a.logits) + b * a.stride_b + k * a.stride_k;
  const int begin = min(p * a.part_len, a.V), end = min(begin + a.part_len, a.V);
  const int64_t at = (int64_t)row_i * a.parts + p;
  double sum = 0.;
  float ref = -INFINITY, last = -INFINITY;  // of the block's list: its beam-th
  bool bad = false, many = false;
  int held = 0;  // places of the list that are filled
  if (threadIdx.x < kMaxBeam) sh.buf.c[threadIdx.x] = no_cand();
  const int ranker = blockIdx.x / 256 & 3;  // of the blocks that share a unit each another wave, so another SIMD
  for (int base = begin; base < end; base += 256 * E) {
    float x[E];
    const int mine = base + wave * 64 * E + lane * VE;  // of vector i: 64 VE i further on
    if (base + (wave + 1) * 64 * E <= end) {
      T raw[NV][VE];
#pragma unroll
      for (int i = 0; i < NV; ++i) load16(row + mine + i * 64 * VE, raw[i]);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VE; ++j) x[i * VE + j] = to_float(raw[i][j]);
    } else {
      // vectors that end behind the row read its last 16 bytes (a row here is longer), shifted
      T raw[NV][VE];
#pragma unroll
      for (int i = 0; i < NV; ++i) load16(row + min(mine + i * 64 * VE, a.V - VE), raw[i]);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int first = mine + i * 64 * VE, off = first - min(first, a.V - VE);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          float v = -INFINITY;
#pragma unroll
          for (int u = j; u < VE; ++u) v = j + off == u ? to_float(raw[i][u]) : v;
          x[i * VE + j] = first + j < end ? v : -INFINITY;
        }
      }
    }
    float top = x[0];  // NaN if one of them is
#pragma unroll
    for (int e = 1; e < E; ++e) top = __builtin_elementwise_maximum(top, x[e]);
    bad |= !(top < INFINITY);
    const float eight = group_max<8>(top);
    if ((lane & 7) == 0) {
      const int i = wave * 8 + (lane >> 3);
      sh.group[i] = eight;
      sh.group_key.k[i] = group_key(eight, i);
    }
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    const float most = wave_max(sh.group[lane & 31]);
    // (equal logits come after those of the list, whose indices are smaller)
    if (!many && most > last) {
      const uint32_t nth = nth_group(sh.group_key, beam), after = orderable(last) + 1;
      const float bound = from_orderable(nth > after ? nth : after);
      // (a wave asks for all its places at once; most of its elements have no lane that reaches the bound)
      int count = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) count += __popcll(__ballot(x[e] >= bound));
      if (count) {
        int pos = 0;
        if (lane == 0) pos = atomicAdd(&sh.n, count);
        pos = held + __builtin_amdgcn_readfirstlane(pos);
        float again = bound;
        asm volatile("" : "+v"(again));  // (compared again: kept, the masks would not fit the scalar registers)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const uint64_t at = __ballot(x[e] >= again);
          if (!at) continue;
          const int to = pos + __builtin_amdgcn_mbcnt_hi((uint32_t)(at >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)at, 0));
          if (x[e] >= again && to < kSelBuf) sh.buf.c[to] = make_cand(x[e], mine + (e / VE) * 64 * VE + e % VE);
          pos += __popcll(at);
        }
      }
    }
    __syncthreads();
    const int n = sh.n;
    many = many || held + n > kSelBuf;
    // one wave ranks while the others add up
    if (n && !many && wave == ranker) rank_candidates(held + n, beam, sh.buf);
    if (most > -INFINITY) {
      if (!(most < ref + 500.f)) {  // (the first tile too; float64 holds exp(500) times exp(200) more)
        const float to = most < INFINITY ? most : 0.f;
        sum *= ref == -INFINITY ? 0. : exp((double)ref - to);
        ref = to;
      }
      const double r = ref;
#pragma unroll
      for (int e = 0; e < E; ++e) sum += exp_d((double)x[e] - r);
    }
    if (base + 256 * E >= end) break;
    __syncthreads();
    if (n) held = beam;
    last = cand_key(sh.buf.c[beam - 1]);
  }
  sum = wave_sum_d(sum);
  if (lane == 0) sh.stat[wave].sum = __any(bad) ? (double)NAN : sum;
  if (many) {
    // more candidates than a wave ranks at a time (many equal logits): each wave its own quarter's best, one after the other
    RowPart part;
    const int len = ((end - begin + 3) / 4 + VE - 1) / VE * VE, first = min(begin + wave * len, end);
    scan_row<T, 8>(row, first, min(first + len, end), beam, part, sh.wave_buf[wave]);
    put_list(part, 0., false, beam, sh.list[wave], sh.stat[wave]);
    if (lane == 0) sh.stat[wave].sum = __any(bad) ? (double)NAN : sum;
    __syncthreads();
    if (wave == 0) {
      const int w = lane / beam, e = lane - w * beam;
      if (lane < 4 * beam) sh.buf.c[lane] = sh.list[w].c[e];
      rank_candidates(4 * beam, beam, sh.buf);
    }
  }
  __syncthreads();
  if (wave) return;
  if (lane < beam) a.lists[at].c[lane] = sh.buf.c[lane];
  if (lane == 0) a.stats[at] = SelStat{(sh.stat[0].sum + sh.stat[1].sum) + (sh.stat[2].sum + sh.stat[3].sum), ref, 0};
}

// 5 to 6 us, a chain of dependent steps in one wave: lists in, exp and log of the sums, keys, bound, ranking
static __global__ __launch_bounds__(64) void k_select_join(SelectArgs a) {
  __shared__ SelJoin sh;
  const int64_t first = (int64_t)blockIdx.x * a.beam * a.parts;
  join_lists(a, blockIdx.x, a.lists + first, a.stats + first, sh);
}

// ---- states of hypotheses to the slots of their successors, in place: state[b, k] = state[b, parent[b, k]]
// A thread reads its column of all slots' sources and then writes those that move, so that no copy of the tensor is needed.  Slots that stay where they are
// are read (from themselves) but not written: with 16 x 8 slots of 4 x 8 runs of 25 KB, two tensors, none moving, 28 us.  Bound by memory: parents drawn at
// random move them in 66 us, 4.7 TB/s, a large copy's rate.
struct StateView {  // strides in bytes
  char *data;
  int64_t lead_stride, b_stride, slot_stride, inner_stride, row_bytes;
  int lead, inner;
  int chunks;       // blocks for one row
  int first_block;  // of this tensor
};
constexpr int kMaxStates = 16;
struct ReorderArgs {
  const int *parent;
  int B, beam, n;
  StateView s[kMaxStates];
};

typedef uintx4_t uintx4_any __attribute__((aligned(1)));  // at any address

template <typename V, int BEAM>
__device__ __forceinline__ void move_column(char *p, int64_t slot_stride, const int (&parent)[BEAM], int beam) {
  V v[BEAM];  // (of a slot that stays, itself, of places behind the beam, slot 0: without branches all loads leave at once)
#pragma unroll
  for (int k = 0; k < BEAM; ++k) v[k] = *reinterpret_cast<const V *>(p + (k < beam ? parent[k] : 0) * slot_stride);
#pragma unroll
  for (int k = 0; k < BEAM; ++k)
    if (parent[k] != k) *reinterpret_cast<V *>(p + k * slot_stride) = v[k];
}

// A column is 16 bytes from any address; what a row has behind its last 16 is columns of one byte
template <int BEAM>
__global__ __launch_bounds__(256) void k_reorder(ReorderArgs a) {
  int t = 0;
  while (t + 1 < a.n && (int)blockIdx.x >= a.s[t + 1].first_block) ++t;
  const StateView &s = a.s[t];
  const int block = blockIdx.x - s.first_block, chunk = block % s.chunks;
  int row = block / s.chunks;
  const int inner = row % s.inner;
  row /= s.inner;
  const int b = row % a.B, lead = row / a.B;
  int parent[BEAM];  // the same for all lanes: branches, not masks
#pragma unroll
  for (int k = 0; k < BEAM; ++k) {
    const int p = k < a.beam ? __builtin_amdgcn_readfirstlane(a.parent[(int64_t)b * a.beam + k]) : k;
    parent[k] = p >= 0 && p < a.beam ? p : k;  // an empty slot keeps what it holds
  }
  const int64_t column = (int64_t)chunk * 256 + threadIdx.x, wide = s.row_bytes >> 4;
  char *const p = s.data + lead * s.lead_stride + b * s.b_stride + inner * s.inner_stride;
  if (column < wide) move_column<uintx4_any, BEAM>(p + column * 16, s.slot_stride, parent, a.beam);
  else if (column - wide < (s.row_bytes & 15)) move_column<uint8_t, BEAM>(p + wide * 16 + (column - wide), s.slot_stride, parent, a.beam);
}

}  // namespace rb
