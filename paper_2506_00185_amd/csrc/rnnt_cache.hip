// Host side of the paged cache: rows in and out, and the attention over it.  See include/rnnt_beam.h for the contract.
#include "token_host.h"

#include <new>
#include <type_traits>

#include "token_attend.h"

using namespace rb;

namespace {

constexpr int kUnits = 256;  // compute units of an MI355X

int cache_view(const rnnt_cache_t *c, CacheView &v) {
  if (!c || c->struct_size != sizeof(rnnt_cache_t)) return refuse("NULL argument or struct_size mismatch");
  if (c->format != RNNT_CACHE_E4M3 && c->format != RNNT_CACHE_F16) return refuse("unknown cache format");
  if (!c->k || !c->v || !c->k_exp || !c->v_exp || !c->table) return refuse("NULL array");
  if (((uintptr_t)c->k | (uintptr_t)c->v) % 16) return refuse("k and v must be 16-byte aligned");
  if (c->n_pages < 1 || c->heads < 1 || c->width < 1) return refuse("n_pages, heads and width must be at least 1");
  if (c->dim < 16 || c->dim > 256 || c->dim % 16) return refuse("dim must be a multiple of 16 from 16 to 256");
  if (c->page_size < 1 || c->page_size > 4096 || (c->page_size & (c->page_size - 1))) return refuse("page_size must be a power of two up to 4096");
  if ((int64_t)c->n_pages * c->heads > 0xfffffffell / c->page_size) return refuse("n_pages * heads * page_size must be below 2^32 - 1");
  if ((int64_t)c->n_pages * c->heads * c->page_size > 0xffffffffll / (c->dim * (c->format == RNNT_CACHE_F16 ? 2 : 1) / 16)) return refuse("k and v may have up to 64 GiB each");
  if ((int64_t)c->width * c->page_size > 1 << 30) return refuse("width * page_size must be at most 2^30");
  v.k = static_cast<char *>(c->k);
  v.v = static_cast<char *>(c->v);
  v.k_exp = c->k_exp;
  v.v_exp = c->v_exp;
  v.n_pages = c->n_pages;
  v.page_size = c->page_size;
  v.page_shift = __builtin_ctz((unsigned)c->page_size);
  v.heads = c->heads;
  v.dim = c->dim;
  v.table = c->table;
  v.table_stride = c->table_stride;
  v.width = c->width;
  return RNNT_OK;
}

template <typename TT, int FMT, bool WRITE, int LANES>
int rows_lanes(RowsArgs &a, hipStream_t stream) {
  constexpr int kRows = kRowsOfGroup * 256 / LANES;
  a.blocks = (a.n * a.c.heads + kRows - 1) / kRows;
  const int64_t blocks = (int64_t)a.B * a.blocks;
  if constexpr (WRITE) return launch(k_cache_write<TT, FMT, LANES>, blocks, 2, 256, a, stream);
  else return launch(k_cache_read<TT, FMT, LANES>, blocks, 2, 256, a, stream);
}
template <typename TT, int FMT, bool WRITE>
int rows_typed(RowsArgs &a, hipStream_t stream) {
  const int lanes = a.c.dim / 8;
  if (lanes <= 2) return rows_lanes<TT, FMT, WRITE, 2>(a, stream);
  if (lanes <= 4) return rows_lanes<TT, FMT, WRITE, 4>(a, stream);
  if (lanes <= 8) return rows_lanes<TT, FMT, WRITE, 8>(a, stream);
  if (lanes <= 16) return rows_lanes<TT, FMT, WRITE, 16>(a, stream);
  return rows_lanes<TT, FMT, WRITE, 32>(a, stream);
}

template <bool WRITE>
int rows_call(const rnnt_cache_t *cache, const rnnt_rows_t *k, const rnnt_rows_t *v, int32_t type, int32_t B, int32_t n, const int32_t *start,
              const int32_t *count, void *hip_stream) {
  RowsArgs a;
  if (const int rc = cache_view(cache, a.c)) return rc;
  if (!k || !v || !start) return refuse("NULL argument");
  if (B < 1 || n < 0) return refuse("B must be at least 1, n not negative");
  if (n == 0) return RNNT_OK;
  if (!k->data || !v->data) return refuse("NULL array");
  if ((int64_t)n * a.c.heads > 1 << 30) return refuse("more work than one launch takes");
  const rnnt_rows_t *r[2] = {k, v};
  for (int i = 0; i < 2; ++i) {
    a.in[i] = r[i]->data;
    a.out[i] = r[i]->data;
    a.stride_b[i] = r[i]->stride_b;
    a.stride_n[i] = r[i]->stride_n;
    a.stride_h[i] = r[i]->stride_h;
  }
  a.start = start;
  a.count = count;
  a.B = B;
  a.n = n;
  // x / heads = upper half of x mul, shifted: mul = 2^(31 + l) / heads + 1 for 2^(l - 1) < heads <= 2^l, exact for x below 2^31
  int l = 0;
  while ((1 << l) < a.c.heads && l < 30) ++l;
  a.by_heads.shift = l - 1;
  a.by_heads.mul = l ? (uint32_t)(((uint64_t)1 << (31 + l)) / (uint32_t)a.c.heads + 1) : 0;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const bool f8 = cache->format == RNNT_CACHE_E4M3;
  switch (type) {
    case RNNT_TYPE_F32: return f8 ? rows_typed<TypeF32, 8, WRITE>(a, stream) : rows_typed<TypeF32, 16, WRITE>(a, stream);
    case RNNT_TYPE_F16: return f8 ? rows_typed<TypeF16, 8, WRITE>(a, stream) : rows_typed<TypeF16, 16, WRITE>(a, stream);
    case RNNT_TYPE_BF16: return f8 ? rows_typed<TypeBf16, 8, WRITE>(a, stream) : rows_typed<TypeBf16, 16, WRITE>(a, stream);
  }
  return refuse("unknown type");
}

// How the work of a call is cut
struct AttendPlan {
  int dp, mt, rows, row_tiles, splits, split_len, join_shares;
  int64_t blocks, workspace;
};
int attend_plan(const CacheView &c, bool f8, const rnnt_attend_t *s, AttendPlan &p) {
  if (!s || s->struct_size != sizeof(rnnt_attend_t)) return refuse("NULL argument or struct_size mismatch");
  if (s->B < 1 || s->n < 1 || s->tree < s->n) return refuse("B and n must be at least 1, n at most tree");
  if (s->parents && s->tree > kTreeMax) return refuse("a tree with parents has at most 1024 nodes");
  if (s->q_heads < 1 || s->q_heads % c.heads) return refuse("q_heads must be a multiple of the cache's heads");
  if (s->max_len < 0) return refuse("max_len must not be negative");
  const int64_t rows = (int64_t)s->n * (s->q_heads / c.heads), pairs = (int64_t)s->B * c.heads;
  if (rows > 1 << 24 || pairs > 1 << 24 || rows * pairs > (int64_t)1 << 32) return refuse("more work than one launch takes");
  p.rows = (int)rows;
  p.dp = c.dim <= 64 ? 64 : c.dim <= 128 ? 128 : 256;
  // Two tiles of rows for a block: a token's key and value are loaded and unpacked once for both, but half as many waves fit.  That pays where
  // blocks of one tile would fill the chip, and where a row is more than 64 bytes (trees of 61 nodes over 500 to 2000 tokens, microseconds with
  // one tile and two: 16 sequences x 32 heads on 8 of 128, float32 on a cache of 16 bits 131 and 85, bfloat16 on e4m3 86 and 72; of 64 on 16
  // bits 77 and 55, on e4m3 50 and 48, but 25 and 26 with 8 sequences x 16 heads, and 58 and 72 for 2 chunks of 2000; 2 sequences x 8 heads of 128: 21 and 22).
  // With 256 dims the sums of two tiles do not fit the registers.
  const int64_t tiles = (rows + 15) / 16;
  p.mt = tiles > 1 && pairs * tiles > kUnits && (f8 ? p.dp == 128 : p.dp < 256) ? 2 : 1;
  p.row_tiles = (int)((rows + 16 * p.mt - 1) / (16 * p.mt));
  // Splits of equal length for all sequences, so that short ones leave no long ones behind: enough blocks for two on every unit, four where a
  // unit holds three or more (32 sequences of 1000 to 8000 tokens, 32 heads on 8 of 128: 76 us with two, 66 with four, 71 with six; where it holds two, four
  // cost: 16 trees of 61 nodes 64 us for 51), none shorter than 256 tokens, two tiles for each of its waves (one sequence of 8000 tokens:
  // 16.0 us from 128 tokens on, 13.1 from 256, 14.5 from 512).
  const int64_t room = (int64_t)c.width << c.page_shift, longest = s->max_len < room ? (s->max_len > 1 ? s->max_len : 1) : room;
  const int64_t others = pairs * p.row_tiles, want = ((attend_blocks(f8 ? 8 : 16, p.dp, p.mt) > 2 ? 4 : 2) * kUnits + others - 1) / others, most = (longest + 255) / 256;
  int64_t splits = want < most ? want : most;
  int64_t len = ((longest + splits - 1) / splits + 127) / 128 * 128;
  splits = (longest + len - 1) / len;
  p.splits = (int)splits;
  p.split_len = (int)len;
  p.blocks = (pairs * splits + 7) / 8 * 8 * p.row_tiles;
  p.join_shares = 1;  // four splits for each thread of the join (one sequence of 8000 tokens: 13.1 us, with all splits on one thread 16.3)
  while (p.join_shares < 8 && p.join_shares * 4 < splits && c.dim / 4 * p.join_shares * 2 <= 256) p.join_shares *= 2;
  p.workspace = splits > 1 ? splits * pairs * rows * (int64_t)(c.dim * sizeof(float) + sizeof(float2)) : 0;
  return RNNT_OK;
}

}  // namespace

extern "C" {

int rnnt_cache_write(const rnnt_cache_t *cache, const rnnt_rows_t *k, const rnnt_rows_t *v, int32_t type, int32_t B, int32_t n,
                     const int32_t *start, const int32_t *count, void *hip_stream) try {
  return rows_call<true>(cache, k, v, type, B, n, start, count, hip_stream);
} catch (const std::bad_alloc &) {
  return RNNT_E_NOMEM;
} catch (...) {
  return RNNT_E_HIP;
}

int rnnt_cache_read(const rnnt_cache_t *cache, const rnnt_rows_t *k, const rnnt_rows_t *v, int32_t type, int32_t B, int32_t n,
                    const int32_t *start, const int32_t *count, void *hip_stream) try {
  return rows_call<false>(cache, k, v, type, B, n, start, count, hip_stream);
} catch (const std::bad_alloc &) {
  return RNNT_E_NOMEM;
} catch (...) {
  return RNNT_E_HIP;
}

int64_t rnnt_cache_attend_workspace(const rnnt_cache_t *cache, const rnnt_attend_t *s) try {
  CacheView c;
  AttendPlan p;
  if (const int rc = cache_view(cache, c)) return rc;
  if (const int rc = attend_plan(c, cache->format == RNNT_CACHE_E4M3, s, p)) return rc;
  return p.workspace;
} catch (...) {
  return RNNT_E_NOMEM;
}

int rnnt_cache_attend(const rnnt_cache_t *cache, const rnnt_attend_t *s, void *hip_stream) try {
  AttendArgs a;
  AttendPlan p;
  if (const int rc = cache_view(cache, a.c)) return rc;
  if (const int rc = attend_plan(a.c, cache->format == RNNT_CACHE_E4M3, s, p)) return rc;
  if (!s->q.data || !s->out || !s->lens) return refuse("NULL array");
  if (p.workspace && (!s->workspace || (uintptr_t)s->workspace % 16 || s->workspace_bytes < p.workspace))
    return refuse("workspace is missing, too small or not aligned");
  a.q = s->q.data;
  a.out = s->out;
  a.stride_b = s->q.stride_b;
  a.stride_n = s->q.stride_n;
  a.stride_h = s->q.stride_h;
  a.lens = s->lens;
  a.parents = s->parents;
  a.B = s->B;
  a.n = s->n;
  a.tree = s->tree;
  a.group = s->q_heads / a.c.heads;
  a.rows = p.rows;
  a.row_tiles = p.row_tiles;
  a.splits = p.splits;
  a.split_len = p.split_len;
  a.join_shares = p.join_shares;
  a.scale = s->scale;
  a.part = static_cast<float *>(s->workspace);
  a.stat = reinterpret_cast<float2 *>(a.part + (int64_t)p.splits * s->B * a.c.heads * p.rows * a.c.dim);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const bool f8 = cache->format == RNNT_CACHE_E4M3;
  switch (s->type) {
    case RNNT_TYPE_F32:
      return f8 ? launch_attend<TypeF32, 8>(a, p.dp, p.mt, p.blocks, stream) : launch_attend<TypeF32, 16>(a, p.dp, p.mt, p.blocks, stream);
    case RNNT_TYPE_F16:
      return f8 ? launch_attend<TypeF16, 8>(a, p.dp, p.mt, p.blocks, stream) : launch_attend<TypeF16, 16>(a, p.dp, p.mt, p.blocks, stream);
    case RNNT_TYPE_BF16:
      return f8 ? launch_attend<TypeBf16, 8>(a, p.dp, p.mt, p.blocks, stream) : launch_attend<TypeBf16, 16>(a, p.dp, p.mt, p.blocks, stream);
  }
  return refuse("unknown type");
} catch (const std::bad_alloc &) {
  return RNNT_E_NOMEM;
} catch (...) {
  return RNNT_E_HIP;
}

}  // extern "C"
