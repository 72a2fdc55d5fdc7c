"""The operators with which an attention decoder or a neural language model takes part in the beam search, as cases.

A step of a beam search over a network that the caller runs itself needs, beside that network's products: the keys and
values of the new tokens written to a paged cache that keeps them in 8 or 16 bits (``write``) and, for a program that works on them, read
back (``read``); the attention of the new tokens, a tree of drafted tokens or of an n-best list's prefixes, one token or a
chunk of a transcript, over that cache (``attend``); the best tokens of all hypotheses of an utterance (``select``); and the
states of the hypotheses moved to the slots of their successors (``reorder``).

``own`` false: each operator in elementary torch operations.  ``own`` true: the framework's entry points.

Formulas.
  select: key(k, v) = score_k + x[k, v] - log sum_u exp x[k, u]; a finished hypothesis has the one candidate (k, eos) with key score_k; the K
    largest keys of an utterance in order, of equal ones the smallest k V + v first.  No candidate: a key of NaN or -inf.
  reorder: state[b, k] = state[b, parent[b, k]], in place.
  write: a row x (the dim values of one token and head) is kept as y 2^s, s the smallest exponent for which max |x| <= 448 2^s ("e4m3") or
    max |x| < 2^15 2^s ("f16"; 2^15 itself only by rounding), y = x 2^-s rounded to the nearest; stored exponent s + 127; rows that hold NaN or infinities: y 0,
    exponent 255, which reads as NaN.
  attend: out_i = sum_t softmax_t(scale q_i . k_t) v_t over the lens[b] tokens kept before and over node i and its ancestors.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
PAGE = 16  # tokens of a page wherever a case does not say otherwise


def _select(name, batch, beam, vocab, dtype, finish=0.0):
    """``finish``: share of the hypotheses that have finished."""
    c = dict(op="select", batch=batch, beam=beam, vocab=vocab, dtype=dtype, finish=finish)
    return dict(c, name=name) if name else c


def _reorder(name, batch, beam, lead, inner, run, stride, count, dtype):
    """``count`` tensors [lead, batch, beam, inner, stride], of which the first ``run`` values of the last axis move."""
    c = dict(op="reorder", batch=batch, beam=beam, lead=lead, inner=inner, run=run, stride=stride, count=count, dtype=dtype)
    return dict(c, name=name) if name else c


def _cache(name, op, batch, tokens, heads, dim, dtype, fmt, page=PAGE):
    """``tokens`` per sequence, written to or read from positions behind a prefix of some other length."""
    c = dict(op=op, batch=batch, tokens=tokens, heads=heads, dim=dim, dtype=dtype, fmt=fmt, page=page)
    return dict(c, name=name) if name else c


def _attend(name, batch, nodes, len_min, len_max, heads, kv_heads, dim, dtype, fmt, tree=False, page=PAGE):
    """``nodes`` queries per sequence (``tree``: with parents, a few of them padding; else each the successor of the one before it)
    over ``len_min`` to ``len_max`` tokens kept before."""
    c = dict(op="attend", batch=batch, nodes=nodes, len_min=len_min, len_max=len_max, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, fmt=fmt,
             tree=tree, page=page)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one utterance, beam and vocabulary of this repository's headline decoders: latency of the call
        _select("select_b1_beam4_v1024", 1, 4, 1024, "f32"),
        # batch, beam and vocabulary of the large stateless workload, logits as a bfloat16 product leaves them (many equal ones)
        _select("select_b128_beam10_v8192", 128, 10, 8192, "bf16"),
        # an attention decoder with a large odd vocabulary, wide beam, some hypotheses finished
        _select("select_b32_beam12_v32003", 32, 12, 32003, "f32", finish=0.2),
        # hidden and cell state of the LSTM prediction network of this repository's workloads
        _reorder("reorder_lstm_b32_beam4", 32, 4, 1, 1, 640, 640, 2, "f32"),
        # keys and values of four layers in contiguous caches with room for 256 tokens, 201 of them filled, beam 8
        _reorder("reorder_layers_b16_beam8", 16, 8, 4, 8, 201 * 64, 256 * 64, 2, "f16"),
        # one new token of each of 64 sequences, a small decoder
        _cache("write_step_b64", "write", 64, 1, 8, 64, "bf16", "e4m3"),
        # prompts or encoder outputs of eight sequences at once
        _cache("write_prompt_b8", "write", 8, 2048, 8, 128, "bf16", "e4m3"),
        # the tail of a few sequences read back in float32 from a cache of 16 bits
        _cache("read_tail_b4", "read", 4, 93, 4, 96, "f32", "f16"),
        # whole sequences read back
        _cache("read_all_b16", "read", 16, 1501, 8, 128, "bf16", "e4m3"),
        # one token of one short sequence: latency of the call
        _attend("attend_b1_len187", 1, 1, 187, 187, 8, 8, 64, "bf16", "e4m3"),
        # a step of 32 ragged sequences with shared heads
        _attend("attend_b32_len8000", 32, 1, 1000, 8000, 32, 8, 128, "bf16", "e4m3"),
        # prefix trees of n-best lists rescored in float32 after prompts, 16-bit cache, odd number of nodes
        _attend("attend_tree_b16_n61", 16, 61, 400, 1900, 16, 4, 128, "f32", "f16", tree=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """Cases of the listed ones' ranges: beams 1 to 16 with vocabularies of 17 to 60 000; states of a few hundred bytes to a hundred MB; rows of
    32 to 256 values; 1 to 80 nodes over up to 8000 tokens, 1 to 8 heads to a key head; each type and format."""
    op = rng.choice(["select", "select", "reorder", "write", "read", "attend", "attend", "attend"])
    if op == "select":
        beam = rng.randint(1, 16)
        vocab = _log_int(rng, 17, 60000)
        batch = min(_log_int(rng, 1, 128), max(1, 10_000_000 // (beam * vocab)))
        return _select("", batch, beam, vocab, rng.choice(["f32", "f16", "bf16"]), rng.choice([0.0, 0.0, 0.3]))
    if op == "reorder":
        beam, lead, inner = rng.randint(2, 16), rng.randint(1, 4), rng.randint(1, 8)
        run = _log_int(rng, 33, 16000)
        count = rng.randint(1, 3)
        batch = min(_log_int(rng, 1, 64), max(1, 25_000_000 // (beam * lead * inner * run * count)))
        return _reorder("", batch, beam, lead, inner, run, run + rng.choice([0, 0, 8, 128, 1027]), count, rng.choice(["f32", "f16", "bf16"]))
    heads, dim = rng.choice([1, 2, 4, 5, 8]), rng.choice([32, 64, 64, 80, 96, 128, 128, 192, 256])
    dtype, fmt, page = rng.choice(["f32", "f16", "bf16", "bf16"]), rng.choice(["e4m3", "e4m3", "f16"]), rng.choice([1, 8, 16, 16, 64])
    if op != "attend":
        tokens = _log_int(rng, 1, 2000)
        return _cache("", op, min(_log_int(rng, 1, 64), max(1, 8_000_000 // (tokens * heads * dim))), tokens, heads, dim, dtype, fmt, page)
    nodes, group = rng.choice([1, 1, 1, rng.randint(2, 80)]), rng.choice([1, 2, 4, 7, 8])
    longest = _log_int(rng, 1, 8000)
    batch = _log_int(rng, 1, 64)
    share, tree = rng.uniform(0.1, 1.0), nodes > 1 and rng.random() < 0.7

    def made():
        return _attend("", batch, nodes, int(longest * share), longest, heads * group, heads, dim, dtype, fmt, tree, page)

    while work(made())["bytes"] > 2.9e8 or work(made())["flops"] > 9e9:
        if batch > 1:
            batch -= 1
        else:
            longest = max(1, longest // 2)
    return made()


# ---------------------------------------------------------------- inputs
def _lens(c):
    n = c["batch"]
    return [c["len_max"] - (c["len_max"] - c["len_min"]) * i // max(1, n - 1) for i in range(n)]


def _pages(c, tokens, g):
    """A table that gives each sequence pages of its own for ``tokens`` positions, in any order, and the number of pages."""
    width = -(-tokens // c["page"])
    n = c["batch"] * width
    return torch.randperm(n, generator=g, device=DEVICE).to(torch.int32).reshape(c["batch"], width), n


def _quantise(x, fmt):
    """(y, s + 127) of rows along the last axis, see above."""
    x = x.float()
    amax = x.abs().amax(-1)
    mant, e = torch.frexp(amax)
    s = e - 15 if fmt == "f16" else torch.where(mant > 0.875, e - 8, e - 9)
    s = torch.where(amax == 0, 0, s.clamp(min=-126))
    good = torch.isfinite(amax)  # NaN where a value is NaN
    s = torch.where(good, s, 0)
    y = torch.where(good[..., None], torch.ldexp(x, -s[..., None]), 0.0)
    y = y.to(torch.float16 if fmt == "f16" else torch.float8_e4m3fn)
    return y, torch.where(good, s + 127, 255).to(torch.uint8)


def _stands_for(y, e):
    """The float32 values of rows kept as (y, e)."""
    scale = torch.where(e == 255, math.nan, torch.ldexp(torch.ones((), device=e.device), e.int() - 127))
    return y.float() * scale[..., None]


def _bits(y):
    return y.view(torch.int16 if y.dtype == torch.float16 else torch.uint8)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEVICE)  # noqa: E731
    if c["op"] == "select":
        n, k, v = c["batch"], c["beam"], c["vocab"]
        # logits of a network that is fairly sure: a few tokens of each row stand out
        logits = (randn(n, k, v) * 2.5).to(DTYPES[c["dtype"]])
        scores = -20.0 - 3.0 * torch.rand(n, k, generator=g, device=DEVICE, dtype=torch.float64)
        done = torch.rand(n, k, generator=g, device=DEVICE) < c["finish"]
        return dict(case=c, logits=logits, scores=scores, done=done, eos=min(2, v - 1))
    if c["op"] == "reorder":
        n, k = c["batch"], c["beam"]
        parents = torch.randint(0, k, (n, k), generator=g, device=DEVICE, dtype=torch.int32)
        full = [randn(c["lead"], n, k, c["inner"], c["stride"]).to(DTYPES[c["dtype"]]) for _ in range(c["count"])]
        return dict(case=c, parents=parents, states=[t[..., :c["run"]] for t in full])
    heads = c["kv_heads"] if c["op"] == "attend" else c["heads"]
    if c["op"] == "attend":
        before, new = _lens(c), c["nodes"]
        order = torch.randperm(len(before), generator=g, device=DEVICE)
        start = torch.tensor(before, dtype=torch.int32, device=DEVICE)[order]
        most = max(before) + new
    else:
        new = c["tokens"]
        start = torch.randint(0, 40, (c["batch"],), generator=g, device=DEVICE, dtype=torch.int32)
        most = 40 + new
    table, n_pages = _pages(c, most, g)
    shape = (n_pages, heads, c["page"], c["dim"])
    if c["op"] == "write":
        kept = torch.float16 if c["fmt"] == "f16" else torch.float8_e4m3fn
        store = [torch.zeros(shape, dtype=torch.float32, device=DEVICE).to(kept) for _ in range(2)]
        exps = [torch.full(shape[:3], 127, dtype=torch.uint8, device=DEVICE) for _ in range(2)]
    else:
        (ky, ke), (vy, ve) = (_quantise(randn(*shape) * torch.exp(0.5 * randn(*shape[:3], 1)), c["fmt"]) for _ in range(2))
        store, exps = [ky, vy], [ke, ve]
    s = dict(case=c, store=store, exps=exps, table=table, start=start, most=most)
    if c["op"] == "write":
        s["k"], s["v"] = (randn(c["batch"], new, heads, c["dim"]).to(DTYPES[c["dtype"]]) for _ in range(2))
    if c["op"] == "attend":
        s["q"] = randn(c["batch"], new, c["heads"], c["dim"]).to(DTYPES[c["dtype"]])
        s["parents"] = None
        if c["tree"]:
            i = torch.arange(new, device=DEVICE)
            back = (torch.rand(c["batch"], new, generator=g, device=DEVICE).square() * 6).long()
            parents = (i - 1 - back).clamp(min=-1)
            # behind the last node of a sequence there is padding
            nodes = new - (torch.rand(c["batch"], 1, generator=g, device=DEVICE) * new / 4).long()
            s["parents"] = torch.where(i < nodes, parents, -2).to(torch.int32)
    if own:
        from paper_2506_00185_amd import KVCache
        s["cache"] = KVCache.from_tensors(store[0], store[1], exps[0], exps[1])
    return s


# ---------------------------------------------------------------- the operators
def _plain_select(s):
    x, scores, done, eos = s["logits"].double(), s["scores"], s["done"], s["eos"]
    n, k, v = x.shape
    top = x.amax(-1, keepdim=True)
    key = scores[..., None] + (x - top - torch.log(torch.exp(x - top).sum(-1, keepdim=True)))
    only = torch.full_like(key, -math.inf)
    only[..., eos] = scores
    key = torch.where(done[..., None], only, key)
    key = torch.where(torch.isnan(key), -math.inf, key).reshape(n, k * v)
    best, at = torch.sort(key, dim=-1, descending=True, stable=True)
    best, at = best[:, :k], at[:, :k]
    there = best > -math.inf
    parents = torch.where(there, at // v, -1).to(torch.int32)
    tokens = torch.where(there, at % v, -3).to(torch.int32)
    return best, parents, tokens, tokens == eos


def _plain_reorder(s):
    at = s["parents"].long()
    rows = torch.arange(at.shape[0], device=at.device)[:, None]
    for t in s["states"]:
        t.copy_(t[:, rows, at])
    return s["states"]


def _slots(s, tokens):
    """(page, place in it) of positions start[b] .. start[b] + tokens."""
    pos = s["start"][:, None].long() + torch.arange(tokens, device=DEVICE)
    page = s["case"]["page"]
    return torch.gather(s["table"].long(), 1, pos // page), pos % page


def _plain_write(s):
    page, place = _slots(s, s["case"]["tokens"])
    for x, store, exps in zip((s["k"], s["v"]), s["store"], s["exps"]):
        y, e = _quantise(x, s["case"]["fmt"])
        _bits(store)[page, :, place] = _bits(y)
        exps[page, :, place] = e
    return s["store"], s["exps"]


def _plain_read(s):
    page, place = _slots(s, s["case"]["tokens"])
    out = []
    for store, exps in zip(s["store"], s["exps"]):
        y = _bits(store)[page, :, place].view(store.dtype)
        out.append(_stands_for(y, exps[page, :, place]).to(DTYPES[s["case"]["dtype"]]))
    return out


def _plain_attend(s):
    c, q = s["case"], s["q"].float()
    n, new, heads, dim = q.shape
    kv, most = c["kv_heads"], s["most"]
    pos = torch.arange(most, device=DEVICE)
    page, place = s["table"].long()[:, pos // c["page"]], (pos % c["page"]).expand(n, most)
    k, v = (_stands_for(_bits(store)[page, :, place].view(store.dtype), exps[page, :, place]).transpose(1, 2).contiguous()
            for store, exps in zip(s["store"], s["exps"]))  # [n, kv, most, dim]
    i = torch.arange(new, device=DEVICE)
    if s["parents"] is None:
        reach = (i[:, None] >= i).expand(n, new, new)
        gone = torch.zeros(n, new, dtype=torch.bool, device=DEVICE)
    else:
        parents = s["parents"].long()
        gone = ((parents < -1) | (parents >= i)).float()
        step = torch.eye(new, device=DEVICE) + (parents[..., None] == i).float() * (1 - gone)[..., None]
        for _ in range(max(1, (new - 1).bit_length())):  # paths of twice the length each time
            step = (torch.matmul(step, step) > 0).float()
        reach, gone = step > 0, torch.matmul(step, gone[..., None])[..., 0] > 0
    sees = torch.zeros(n, new, most, dtype=torch.bool, device=DEVICE)
    start = s["start"].long()[:, None, None]
    sees |= pos < start
    node = pos - start  # [n, 1, most]: the node that stands at a position
    inside = (node >= 0) & (node < new)
    sees |= inside & torch.gather(reach, 2, node.clamp(0, new - 1).expand(n, new, most))
    sees &= ~gone[..., None]
    rows = q.reshape(n, new, kv, heads // kv, dim).permute(0, 2, 3, 1, 4).reshape(n, kv, -1, dim).contiguous()
    x = torch.matmul(rows * (1 / math.sqrt(dim)), k.transpose(2, 3).contiguous())
    sees = sees[:, None, None].expand(n, kv, heads // kv, new, most).reshape(n, kv, -1, most)
    x = torch.where(sees, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    out = torch.matmul(p, torch.nan_to_num(v)) / p.sum(-1, keepdim=True)
    out = torch.where(sees.any(-1, keepdim=True), out, 0.0)
    return out.reshape(n, kv, heads // kv, new, dim).permute(0, 3, 1, 2, 4).reshape(n, new, heads, dim).to(s["q"].dtype)


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"select": _plain_select, "reorder": _plain_reorder, "write": _plain_write, "read": _plain_read, "attend": _plain_attend}[c["op"]](s)
    import paper_2506_00185_amd as A
    if c["op"] == "select":
        return A.select_tokens(s["logits"], s["scores"], done=s["done"], eos=s["eos"])
    if c["op"] == "reorder":
        A.reorder_states(s["parents"], s["states"], lead=1)
        return s["states"]
    if c["op"] == "write":
        s["cache"].write(s["k"], s["v"], s["table"], s["start"])
        return s["store"], s["exps"]
    if c["op"] == "read":
        return list(s["cache"].read(s["table"], s["start"], c["tokens"], dtype=DTYPES[c["dtype"]]))
    return s["cache"].attend(s["q"], s["table"], s["start"], parents=s["parents"], max_len=s["most"])


def work(case):
    c = case
    if c["op"] == "select":
        rows = c["batch"] * c["beam"]
        read = rows * (1 - c["finish"]) * c["vocab"]  # a finished hypothesis needs none of its logits
        return {"bytes": read * BYTES[c["dtype"]] + rows * (8 + 1 + 8 + 4 + 4 + 1), "flops": 4 * read}
    if c["op"] == "reorder":
        k = c["beam"]  # parents are drawn from all slots alike: of k slots k - 1 move, from so many different ones
        moved, sources = k - 1, k * (1 - (1 - 1 / k) ** (k - 1))
        return {"bytes": c["count"] * c["lead"] * c["batch"] * c["inner"] * c["run"] * BYTES[c["dtype"]] * (moved + sources), "flops": 0}
    if c["op"] in ("write", "read"):
        rows = 2 * c["batch"] * c["tokens"] * c["heads"]
        return {"bytes": rows * (c["dim"] * (BYTES[c["dtype"]] + BYTES[c["fmt"]]) + 1), "flops": 2 * rows * c["dim"]}
    kept, new = sum(_lens(c)), c["batch"] * c["nodes"]
    io = 2 * new * c["heads"] * c["dim"] * BYTES[c["dtype"]]
    return {"bytes": 2 * (kept + new) * c["kv_heads"] * (c["dim"] * BYTES[c["fmt"]] + 1) + io, "flops": 4 * c["dim"] * c["heads"] * c["nodes"] * kept}


# ---------------------------------------------------------------- in 64 bits, from the definitions
def _exact_value(bits, e, fmt):
    """Values of stored bits and exponents, in 64 bits, from the formats' fields."""
    bits = bits.long()
    if fmt == "f16":
        sign, ex, man, m, bias = bits >> 15 & 1, bits >> 10 & 31, bits & 1023, 10, 15
    else:
        sign, ex, man, m, bias = bits >> 7 & 1, bits >> 3 & 15, bits & 7, 3, 7
    y = torch.where(ex > 0, torch.ldexp(1.0 + man.double() / 2**m, ex - bias), man.double() * 2.0 ** (1 - bias - m))
    return torch.where(sign == 1, -y, y) * torch.exp2(e.double() - 127)[..., None]


def _exact_rows(x, fmt):
    """(y, s + 127) of rows of finite values in 64 bits."""
    x = x.double()
    most = x.abs().amax(-1)
    s = torch.floor(torch.log2(torch.where(most > 0, most, 1.0)))  # next to a power of two it may be one off
    s = torch.where(torch.exp2(s) > most, s - 1, s)
    s = torch.where(torch.exp2(s + 1) <= most, s + 1, s)  # 2^s <= most < 2^(s + 1)
    s = s - 14 if fmt == "f16" else torch.where(most > 448 * torch.exp2(s - 8), s - 7, s - 8)
    s = torch.where(most > 0, s, 0.0)
    y = x / torch.exp2(s)[..., None]
    m, least = (10, -14) if fmt == "f16" else (3, -6)
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0**least))) - m)
    return torch.round(y / unit) * unit, s + 127  # torch.round: halves to even


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "select":
        scores, lse = s["scores"], torch.logsumexp(s["logits"].double(), -1)
        out = []
        for b in range(c["batch"]):
            keys = torch.where(s["done"][b], -math.inf, scores[b] - lse[b])[:, None] + s["logits"][b].double()
            keys = torch.cat([keys.reshape(-1), scores[b][s["done"][b]]])
            out.append(torch.topk(keys, c["beam"]).values)
        return torch.stack(out), None, None, None
    if c["op"] == "reorder":
        parents = s["parents"].tolist()
        out = []
        for t in s["states"]:
            r = torch.empty_like(t, dtype=torch.float64)
            for b, row in enumerate(parents):
                for k, p in enumerate(row):
                    r[:, b, k] = t[:, b, p].double()
            out.append(r)
        return out
    at = torch.arange(c["tokens"] if c["op"] != "attend" else s["most"], device=DEVICE)
    if c["op"] == "write":
        stores = [_bits(t).clone().double() for t in s["store"]]  # all zero before
        for x, store in zip((s["k"], s["v"]), stores):
            y, _ = _exact_rows(x, c["fmt"])
            for b in range(c["batch"]):
                pos = at + s["start"][b]
                store[s["table"][b].long()[pos // c["page"]], :, pos % c["page"]] = y[b]
        return stores, [None, None]
    if c["op"] == "read":
        out = []
        for store, exps in zip(s["store"], s["exps"]):
            rows = []
            for b in range(c["batch"]):
                pos = at + s["start"][b]
                page = s["table"][b].long()[pos // c["page"]]
                rows.append(_exact_value(_bits(store)[page, :, pos % c["page"]], exps[page, :, pos % c["page"]], c["fmt"]))
            out.append(torch.stack(rows))
        return out
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    group, starts = c["heads"] // c["kv_heads"], s["start"].tolist()
    parents = s["parents"].tolist() if s["parents"] is not None else [list(range(-1, c["nodes"] - 1))] * c["batch"]
    for b in range(c["batch"]):
        page = s["table"][b].long()[at // c["page"]]
        k, v = (_exact_value(_bits(store)[page, :, at % c["page"]], exps[page, :, at % c["page"]], c["fmt"]) for store, exps in zip(s["store"], s["exps"]))
        paths = []
        for i in range(c["nodes"]):
            path, j = [], i
            while j >= 0 and -1 <= parents[b][j] < j:
                path.append(j)
                j = parents[b][j]
            paths.append(path if j == -1 else None)
        sees = torch.zeros(c["nodes"], len(at), dtype=torch.bool)
        for i, path in enumerate(paths):
            if path is not None:
                sees[i, :starts[b]] = True
                sees[i, [starts[b] + j for j in path]] = True
        live = [i for i, path in enumerate(paths) if path is not None]
        if not live:
            continue
        sees = sees[live].to(DEVICE)
        for h in range(c["heads"]):
            x = s["q"][b, live, h].double() @ k[:, h // group].T.contiguous() / math.sqrt(c["dim"])
            out[b, live, h] = torch.softmax(x.masked_fill(~sees, -math.inf), -1) @ v[:, h // group].contiguous()
    return out
