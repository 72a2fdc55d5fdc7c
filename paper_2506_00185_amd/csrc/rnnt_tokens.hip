// Host side of the selection from a caller's logits and of the reordering of states.  See include/rnnt_beam.h for the contract.
#include <algorithm>
#include <new>
#include <unordered_map>

#include "token_host.h"
#include "token_select.h"

using namespace rb;

namespace {

// Logits of an utterance that k_select_one takes in one tile per wave.  Up to there one launch is faster than two: 4 x 1024 7.5 us and 8.7,
// 32 x 8 x 2048 12.2 and 12.3; twice as many would take its 16 waves two tiles each, one after the other.
constexpr int kSelOneMax = 16 * 64 * 16;

// Parts of a row.  In one launch 16 / beam waves share a row; in two, blocks of up to 8192 logits, a tile for their four waves, as many as the
// join takes (64 lists).
struct SelectPlan {
  bool one;
  int parts, part_len;
};
SelectPlan select_plan(int B, int beam, int V) {
  SelectPlan p;
  p.one = (int64_t)beam * V <= kSelOneMax;
  if (p.one) {
    p.parts = 16 / beam;
    p.part_len = (V + p.parts - 1) / p.parts;
    return p;
  }
  const int most = kSelLists / beam;
  // a chip's worth of blocks, of 1024 to 8192 logits each (10 x 8192: 10.8 us, with blocks of 8192 alone 11.5; for twice as many blocks
  // 128 x 10 x 8192 would take 23.5 us for 20.4)
  const int64_t rows = (int64_t)B * beam;
  int64_t parts = (V + 8191) / 8192;
  const int64_t fill = (1024 + rows - 1) / rows, fine = (V + 1023) / 1024;
  if (parts < fill) parts = fill < fine ? fill : fine;
  p.parts = (int)(parts < most ? parts : most);
  p.part_len = (V + p.parts - 1) / p.parts;
  return p;
}

template <typename TT>
int select_typed(const SelectArgs &a, bool one, hipStream_t stream) {
  // tiles no longer than the parts need: what a tile has beyond a part costs as much as what it has in it (10 x 8192 in parts of 1024: 10.8 us,
  // with tiles of 8192 16.5; long parts in tiles of 4096: 128 x 10 x 8192 23.0 us for 20.4)
  constexpr int kVec = 16 / (int)sizeof(typename TT::T);
  if (one) {
    const int vecs = (a.part_len + 64 * kVec - 1) / (64 * kVec);
    if (vecs <= 1) return launch(k_select_one<TT, 1>, a.B, 1, 1024, a, stream);
    if (vecs <= 2 || kVec == 8) return launch(k_select_one<TT, 2>, a.B, 1, 1024, a, stream);
    if constexpr (kVec == 4) return launch(k_select_one<TT, 4>, a.B, 1, 1024, a, stream);
  }
  const int64_t blocks = (int64_t)a.B * a.beam * a.parts;
  const int rc = launch(a.part_len <= 2048 ? k_select_scan<TT, 8> : a.part_len <= 4096 ? k_select_scan<TT, 16> : k_select_scan<TT, 32>, blocks, 1, 256, a, stream);
  return rc ? rc : launch(k_select_join, a.B, 1, 64, a, stream);
}

// Whether a row of the tensor reaches into the `bytes` from `first` on.  (Rows do not overlap: of those that begin before their end, the last would.)
bool holds(const rnnt_states_t &s, int B, int beam, const void *first, int64_t bytes) {
  int64_t size[4] = {s.lead, B, beam, s.inner}, stride[4] = {s.lead_stride, s.b_stride, s.slot_stride, s.inner_stride};
  int64_t behind = (int64_t)((uintptr_t)first - (uintptr_t)s.data) + bytes - 1;  // how far the last byte lies behind a row's beginning
  if (behind < 0) return false;
  bool done[4] = {};
  for (int i = 0; i < 4; ++i) {
    int top = -1;
    for (int j = 0; j < 4; ++j)
      if (!done[j] && size[j] > 1 && (top < 0 || stride[j] > stride[top])) top = j;
    if (top < 0) break;
    done[top] = true;
    behind -= stride[top] * std::min(behind / stride[top], size[top] - 1);
  }
  return behind - (bytes - 1) < s.row_bytes;
}

int64_t select_lists(int B, int beam, const SelectPlan &p) { return p.one ? 0 : (int64_t)B * beam * p.parts; }

}  // namespace

extern "C" {

int64_t rnnt_select_tokens_workspace(int32_t B, int32_t beam, int32_t V) {
  if (B < 1 || beam < 1 || beam > kMaxBeam || V < 1) return 0;
  return select_lists(B, beam, select_plan(B, beam, V)) * (int64_t)(sizeof(SelList) + sizeof(SelStat));
}

int rnnt_select_tokens(const rnnt_select_t *s, void *hip_stream) try {
  if (!s || s->struct_size != sizeof(rnnt_select_t)) return refuse("NULL argument or struct_size mismatch");
  if (!s->logits || !s->scores || !s->out_scores || !s->out_parent || !s->out_token) return refuse("NULL array");
  if (s->B < 1 || s->V < 1) return refuse("B and V must be at least 1");
  if (s->beam < 1 || s->beam > kMaxBeam) return refuse("beam must be 1 to 16");
  if ((int64_t)s->beam * s->V > 0x7fff0000) return refuse("beam * V must be at most 2^31 - 2^16");
  if (s->eos < -1 || s->eos >= s->V) return refuse("eos must be a token, or -1");
  if (s->eos < 0 && (s->done || s->out_done)) return refuse("done needs eos");
  if (s->eos >= 0 && !s->out_done) return refuse("out_done is missing");
  const SelectPlan p = select_plan(s->B, s->beam, s->V);
  const int64_t lists = select_lists(s->B, s->beam, p);
  if (lists && (!s->workspace || (uintptr_t)s->workspace % 16 || s->workspace_bytes < lists * (int64_t)(sizeof(SelList) + sizeof(SelStat))))
    return refuse("workspace is missing, too small or not aligned");
  SelectArgs a;
  a.logits = s->logits;
  a.stride_b = s->stride_b;
  a.stride_k = s->stride_k;
  a.scores = s->scores;
  a.done = s->done;
  a.out_scores = s->out_scores;
  a.out_parent = s->out_parent;
  a.out_token = s->out_token;
  a.out_done = s->out_done;
  a.lists = static_cast<SelList *>(s->workspace);
  a.stats = lists ? reinterpret_cast<SelStat *>(a.lists + lists) : nullptr;
  a.B = s->B;
  a.beam = s->beam;
  a.V = s->V;
  a.eos = s->eos;
  a.parts = p.parts;
  a.part_len = p.part_len;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  switch (s->type) {
    case RNNT_TYPE_F32: return select_typed<TypeF32>(a, p.one, stream);
    case RNNT_TYPE_F16: return select_typed<TypeF16>(a, p.one, stream);
    case RNNT_TYPE_BF16: return select_typed<TypeBf16>(a, p.one, stream);
  }
  return refuse("unknown type");
} catch (const std::bad_alloc &) {
  return RNNT_E_NOMEM;
} catch (...) {
  return RNNT_E_HIP;
}

int rnnt_reorder_states(const int32_t *parent, int32_t B, int32_t beam, const rnnt_states_t *states, int32_t n, void *hip_stream) try {
  if (!parent || (n > 0 && !states)) return refuse("NULL argument");
  if (B < 1) return refuse("B must be at least 1");
  if (beam < 1 || beam > kMaxBeam) return refuse("beam must be 1 to 16");
  if (n < 0 || n > kMaxStates) return refuse("at most 16 tensors");
  ReorderArgs a;
  a.parent = parent;
  a.B = B;
  a.beam = beam;
  a.n = 0;
  int64_t blocks = 0;
  for (int t = 0; t < n; ++t) {
    const rnnt_states_t &s = states[t];
    if (s.lead < 0 || s.inner < 0 || s.row_bytes < 0) return refuse("negative size");
    if (s.lead == 0 || s.inner == 0 || s.row_bytes == 0) continue;
    if (!s.data) return refuse("NULL tensor");
    // rows must not overlap: in order of their strides, each reaches behind all that the smaller ones span
    int64_t size[4] = {s.lead, B, beam, s.inner}, stride[4] = {s.lead_stride, s.b_stride, s.slot_stride, s.inner_stride}, span = s.row_bytes;
    for (int i = 0; i < 4; ++i)
      for (int j = i + 1; j < 4; ++j)
        if (stride[j] < stride[i]) {
          const int64_t x = stride[i], y = size[i];
          stride[i] = stride[j], stride[j] = x;
          size[i] = size[j], size[j] = y;
        }
    for (int i = 0; i < 4; ++i) {
      if (size[i] == 1) continue;
      if (stride[i] < span) return refuse("rows of a tensor overlap");
      span += stride[i] * (size[i] - 1);
    }
    for (int u = 0; u < t; ++u)
      if (states[u].data == s.data && states[u].lead && states[u].inner && states[u].row_bytes) return refuse("a tensor is named twice");
    StateView &v = a.s[a.n++];
    v.data = static_cast<char *>(s.data);
    v.lead_stride = s.lead_stride;
    v.b_stride = s.b_stride;
    v.slot_stride = s.slot_stride;
    v.inner_stride = s.inner_stride;
    v.row_bytes = s.row_bytes;
    v.lead = s.lead;
    v.inner = s.inner;
    const int64_t chunks = ((s.row_bytes >> 4) + (s.row_bytes & 15) + 255) / 256;
    // (each factor is below 2^31, and a product beyond what a launch takes is refused before the next one is formed)
    int64_t count = chunks;
    if (count > 0x7fffffff) return refuse("more work than one launch takes");
    for (int64_t f : {(int64_t)s.lead, (int64_t)B, (int64_t)s.inner}) {
      count *= f;
      if (count > 0x7fffffff) return refuse("more work than one launch takes");
    }
    v.chunks = (int)chunks;
    v.first_block = (int)blocks;
    blocks += count;  // (up to 16 such: the launch refuses what is too much)
  }
  if (!a.n || beam == 1) return RNNT_OK;
  for (int t = 0; t < n; ++t)  // all blocks read the parents
    if (states[t].lead && states[t].inner && states[t].row_bytes && holds(states[t], B, beam, parent, (int64_t)B * beam * (int64_t)sizeof(int32_t)))
      return refuse("parents lie in a tensor that is reordered");
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (beam <= 4) return launch(k_reorder<4>, blocks, 1, 256, a, stream);
  if (beam <= 8) return launch(k_reorder<8>, blocks, 1, 256, a, stream);
  return launch(k_reorder<16>, blocks, 1, 256, a, stream);
} catch (const std::bad_alloc &) {
  return RNNT_E_NOMEM;
} catch (...) {
  return RNNT_E_HIP;
}

int rnnt_nbest_tree(const int32_t *tokens, const int32_t *lens, int32_t B, int32_t beam, int32_t cap, int32_t max_nodes, int32_t *node_token,
                    int32_t *node_parent, int32_t *leaf, int32_t *n_nodes) try {
  if (!tokens || !lens || !node_token || !node_parent || !leaf || !n_nodes) return refuse("NULL array");
  if (B < 1 || beam < 1 || cap < 1 || max_nodes < 1) return refuse("sizes must be at least 1");
  int most = 0;
  std::unordered_map<uint64_t, int> child;  // (parent node + 1, token) -> node
  for (int64_t b = 0; b < B; ++b) {
    int32_t *tok = node_token + b * max_nodes, *par = node_parent + b * max_nodes;
    child.clear();
    int n = 0;
    for (int k = 0; k < beam; ++k) {
      const int32_t *t = tokens + (b * beam + k) * cap;
      const int len = lens[b * beam + k];
      if (len > cap) return refuse("a length is beyond cap");
      int node = -1;
      for (int i = 0; i < len; ++i) {
        const auto found = child.emplace((uint64_t)(uint32_t)(node + 1) << 32 | (uint32_t)t[i], n);
        if (found.second) {
          if (n == max_nodes) return refuse("an utterance's tree has more than max_nodes nodes");
          tok[n] = t[i];
          par[n++] = node;
        }
        node = found.first->second;
      }
      leaf[b * beam + k] = node;
    }
    n_nodes[b] = n;
    most = n > most ? n : most;
    for (int i = n; i < max_nodes; ++i) {
      tok[i] = 0;
      par[i] = -2;
    }
  }
  return most;
} catch (const std::bad_alloc &) {
  return RNNT_E_NOMEM;
} catch (...) {
  return RNNT_E_HIP;
}

}  // extern "C"
