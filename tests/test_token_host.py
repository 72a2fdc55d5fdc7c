"""Operators for networks that the caller runs itself, without a GPU: the prefix tree of n-best lists, what the host refuses (before any
launch; the pointers below are never read), the plain implementations the GPU tests compare with."""
import ctypes as C
import math

import numpy as np
import pytest

import token_ref as R

E_ARG = -1
FAKE = 1 << 20  # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    from paper_2506_00185_amd import binding, build
    import os
    if not os.path.exists(binding.library_path()):
        build.build()
    return binding.load_library()


def message(lib):
    return lib.rnnt_beam_last_error(None).decode()


# ---------------------------------------------------------------- prefix trees
def brute_tree(tokens, lens):
    nodes, leaf = {}, []
    for t, n in zip(tokens, lens):
        for i in range(1, n + 1):
            nodes.setdefault(tuple(t[:i]), len(nodes))
        leaf.append(nodes[tuple(t[:n])] if n > 0 else -1)
    return [p[-1] for p in nodes], [nodes.get(p[:-1], -1) for p in nodes], leaf


@pytest.mark.parametrize("B,beam,cap,V,seed", [(1, 1, 1, 2, 0), (3, 4, 9, 2, 1), (5, 12, 30, 3, 2), (2, 16, 7, 50, 3)])
def test_prefix_trees_of_nbest_lists(B, beam, cap, V, seed):
    from paper_2506_00185_amd import nbest_tree
    g = np.random.default_rng(seed)
    tokens = g.integers(0, V, (B, beam, cap)).astype(np.int32)
    lens = g.integers(-1, cap + 1, (B, beam)).astype(np.int32)  # -1: empty slot, 0: empty transcript
    t = nbest_tree(tokens, lens)
    for b in range(B):
        tok, par, leaf = brute_tree(tokens[b], lens[b])
        n = t["n_nodes"][b]
        assert n == len(tok)
        np.testing.assert_array_equal(t["tokens"][b, :n], tok)
        np.testing.assert_array_equal(t["parents"][b, :n], par)
        assert np.all(t["parents"][b, n:] == -2)
        np.testing.assert_array_equal(t["leaf"][b], leaf)
    assert t["parents"].shape[1] == max(1, t["n_nodes"].max())


def test_prefix_tree_that_does_not_fit_is_refused():
    from paper_2506_00185_amd import RnntBeamError, nbest_tree
    tokens, lens = np.arange(6, dtype=np.int32).reshape(1, 2, 3), np.array([[3, 3]], np.int32)
    assert nbest_tree(tokens, lens, max_nodes=6)["n_nodes"][0] == 6
    with pytest.raises(RnntBeamError, match="max_nodes"):
        nbest_tree(tokens, lens, max_nodes=5)
    with pytest.raises(RnntBeamError, match="beyond cap"):
        nbest_tree(tokens, lens + 1)


# ---------------------------------------------------------------- refusals
def a_select(**over):
    from paper_2506_00185_amd.tokens import _Select
    s = _Select(struct_size=C.sizeof(_Select), type=0, B=2, beam=4, V=100, eos=-1, logits=FAKE, stride_b=400, stride_k=100, scores=FAKE, done=None,
                out_scores=FAKE, out_parent=FAKE, out_token=FAKE, out_done=None, workspace=FAKE, workspace_bytes=1 << 30)
    for k, v in over.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("over,what", [
    (dict(struct_size=8), "struct_size"), (dict(type=3), "type"), (dict(type=-1), "type"), (dict(B=0), "B and V"), (dict(V=0), "B and V"), (dict(beam=0), "beam"),
    (dict(beam=17), "beam"), (dict(beam=16, V=1 << 27), "2^31"), (dict(beam=1, V=0x7fffffff), "2^31"), (dict(beam=2, V=0x3fff8001), "2^31"), (dict(eos=100), "eos"), (dict(eos=-2), "eos"), (dict(eos=3), "out_done"),
    (dict(done=FAKE), "done"), (dict(out_done=FAKE), "done"), (dict(logits=None), "NULL"), (dict(scores=None), "NULL"), (dict(out_token=None), "NULL"),
    (dict(V=1 << 20, workspace=None), "workspace"), (dict(V=1 << 20, workspace_bytes=100), "workspace"), (dict(V=1 << 20, workspace=FAKE + 8), "workspace")])
def test_selection_refuses(lib, over, what):
    assert lib.rnnt_select_tokens(C.byref(a_select(**over)), None) == E_ARG
    assert what in message(lib)


def test_selection_workspace(lib):
    assert lib.rnnt_select_tokens_workspace(1, 4, 1024) == 0
    assert lib.rnnt_select_tokens_workspace(1, 4, 1 << 20) > 0
    assert lib.rnnt_select_tokens_workspace(1, 17, 1 << 20) == 0
    assert lib.rnnt_select_tokens(None, None) == E_ARG


def a_state(**over):
    from paper_2506_00185_amd.tokens import _States
    s = _States(data=FAKE, lead_stride=0, b_stride=4000, slot_stride=1000, inner_stride=0, row_bytes=1000, lead=1, inner=1)
    for k, v in over.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("over,what", [
    (dict(slot_stride=999), "overlap"), (dict(b_stride=3999), "overlap"), (dict(slot_stride=0), "overlap"), (dict(inner=2, inner_stride=500), "overlap"),
    (dict(lead=2), "overlap"), (dict(slot_stride=-1000), "overlap"), (dict(row_bytes=-1), "negative"), (dict(inner=-1), "negative"), (dict(data=None), "NULL"),
    (dict(row_bytes=1 << 50, slot_stride=1 << 50, b_stride=1 << 52), "more work")])
def test_reordering_refuses(lib, over, what):
    v = (type(a_state()) * 1)(a_state(**over))
    assert lib.rnnt_reorder_states(C.c_void_p(FAKE), 2, 4, v, 1, None) == E_ARG
    assert what in message(lib)


def test_reordering_refuses_counts_and_repeats(lib):
    two = (type(a_state()) * 2)(a_state(), a_state())
    assert lib.rnnt_reorder_states(C.c_void_p(FAKE), 2, 4, two, 2, None) == E_ARG and "twice" in message(lib)
    many = (type(a_state()) * 17)(*[a_state() for _ in range(17)])
    assert lib.rnnt_reorder_states(C.c_void_p(FAKE), 2, 4, many, 17, None) == E_ARG and "16" in message(lib)
    assert lib.rnnt_reorder_states(C.c_void_p(FAKE), 2, 17, two, 1, None) == E_ARG and "beam" in message(lib)
    assert lib.rnnt_reorder_states(C.c_void_p(FAKE), 0, 4, two, 1, None) == E_ARG
    assert lib.rnnt_reorder_states(None, 2, 4, two, 1, None) == E_ARG
    # nothing to move: nothing is launched
    assert lib.rnnt_reorder_states(C.c_void_p(FAKE), 2, 4, None, 0, None) == 0
    assert lib.rnnt_reorder_states(C.c_void_p(FAKE), 2, 1, two, 1, None) == 0
    empty = (type(a_state()) * 1)(a_state(row_bytes=0, data=None))
    assert lib.rnnt_reorder_states(C.c_void_p(FAKE), 2, 4, empty, 1, None) == 0


def test_reordering_refuses_parents_that_it_would_move(lib):
    """(Other tensors' blocks would read parents while they are rewritten.)  A second tensor is more work than one launch takes, so that what is not refused for
    its parents is refused for that, behind it."""
    far = a_state(data=1 << 45, row_bytes=16, lead=2**30 - 1, lead_stride=16, slot_stride=1 << 34, b_stride=1 << 36)

    def refused(at, **over):
        assert lib.rnnt_reorder_states(C.c_void_p(at), 2, 4, (type(far) * 2)(a_state(**over), far), 2, None) == E_ARG
        assert message(lib) in ("parents lie in a tensor that is reordered", "more work than one launch takes")
        return "parents" in message(lib)

    for at in (FAKE, FAKE + 400, FAKE + 7999, FAKE - 31):  # 2 x 4 rows of 1000 bytes, 32 bytes of parents
        assert refused(at, lead=2, lead_stride=8000)
    # every place next to rows with gaps
    g = np.random.default_rng(0)
    for _ in range(60):
        row, span, strides = int(g.integers(1, 40)), 0, {}
        sizes = dict(inner=int(g.integers(1, 4)), lead=int(g.integers(2, 4)), b=2, slot=4)
        span = row
        for name in g.permutation(list(sizes)):
            strides[str(name)] = span + int(g.integers(0, 90))
            span += strides[str(name)] * (sizes[str(name)] - 1)
        v = dict(inner=sizes["inner"], lead=sizes["lead"], row_bytes=row, **{f"{k}_stride": x for k, x in strides.items()})
        held = np.zeros(span + 128, bool)
        for i in np.ndindex(*sizes.values()):
            at = 64 + sum(n * strides[k] for n, k in zip(i, sizes))
            held[at:at + row] = True
        for at in range(24, len(held) - 32, 4):
            assert refused(FAKE + at - 64, **v) == bool(held[at:at + 32].any())


def a_cache(**over):
    from paper_2506_00185_amd.tokens import _Cache
    c = _Cache(struct_size=C.sizeof(_Cache), format=0, n_pages=10, page_size=16, heads=2, dim=64, k=FAKE, v=FAKE, k_exp=FAKE, v_exp=FAKE, table=FAKE,
               table_stride=5, width=5)
    for k, v in over.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [(dict(struct_size=1), "struct_size"), (dict(format=2), "format"), (dict(page_size=12), "page_size"), (dict(page_size=0), "page_size"),
              (dict(page_size=8192), "page_size"), (dict(dim=0), "dim"), (dict(dim=72), "dim"), (dict(dim=272), "dim"), (dict(heads=0), "heads"), (dict(n_pages=0), "n_pages"),
              (dict(width=0), "width"), (dict(k=FAKE + 8), "aligned"), (dict(v_exp=None), "NULL"), (dict(table=None), "NULL"),
              (dict(n_pages=1 << 30, page_size=4096), "2^32"), (dict(width=1 << 30), "2^30")]


@pytest.mark.parametrize("over,what", BAD_CACHES)
def test_caches_that_are_refused(lib, over, what):
    from paper_2506_00185_amd.tokens import _Rows
    c, rows = a_cache(**over), _Rows(FAKE, 1, 1, 1)
    for call in (lib.rnnt_cache_write, lib.rnnt_cache_read):
        assert call(C.byref(c), C.byref(rows), C.byref(rows), 0, 1, 1, C.c_void_p(FAKE), None, None) == E_ARG
        assert what in message(lib)
    assert lib.rnnt_cache_attend(C.byref(c), C.byref(an_attend()), None) == E_ARG and what in message(lib)
    assert lib.rnnt_cache_attend_workspace(C.byref(c), C.byref(an_attend())) == E_ARG


def test_rows_that_are_refused(lib):
    from paper_2506_00185_amd.tokens import _Rows
    c, rows, none = a_cache(), _Rows(FAKE, 1, 1, 1), _Rows(None, 1, 1, 1)
    for call in (lib.rnnt_cache_write, lib.rnnt_cache_read):
        assert call(C.byref(c), C.byref(rows), C.byref(rows), 3, 1, 1, C.c_void_p(FAKE), None, None) == E_ARG and "type" in message(lib)
        assert call(C.byref(c), C.byref(rows), C.byref(rows), 0, 0, 1, C.c_void_p(FAKE), None, None) == E_ARG
        assert call(C.byref(c), C.byref(rows), C.byref(rows), 0, 1, -1, C.c_void_p(FAKE), None, None) == E_ARG
        assert call(C.byref(c), C.byref(rows), C.byref(rows), 0, 1, 1, None, None, None) == E_ARG
        assert call(C.byref(c), C.byref(none), C.byref(rows), 0, 1, 1, C.c_void_p(FAKE), None, None) == E_ARG
        assert call(C.byref(c), C.byref(rows), C.byref(rows), 0, 1 << 30, 1 << 30, C.c_void_p(FAKE), None, None) == E_ARG and "more work" in message(lib)
        assert call(C.byref(c), C.byref(rows), C.byref(rows), 0, 1, 0, C.c_void_p(FAKE), None, None) == 0  # no rows


def an_attend(**over):
    from paper_2506_00185_amd.tokens import _Attend, _Rows
    a = _Attend(struct_size=C.sizeof(_Attend), type=0, B=2, n=3, tree=3, q_heads=4, scale=1.0, max_len=80, q=_Rows(FAKE, 1, 1, 1), out=FAKE, lens=FAKE,
                parents=None, workspace=FAKE, workspace_bytes=1 << 30)
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("over,what", [
    (dict(struct_size=4), "struct_size"), (dict(type=7), "type"), (dict(B=0), "at least 1"), (dict(n=0), "at least 1"), (dict(tree=2), "tree"),
    (dict(parents=FAKE, tree=1025), "1024"), (dict(q_heads=3), "q_heads"), (dict(q_heads=0), "q_heads"), (dict(max_len=-1), "max_len"), (dict(out=None), "NULL"),
    (dict(lens=None), "NULL"), (dict(n=1 << 30, tree=1 << 30), "more work"), (dict(B=1 << 30), "more work")])
def test_attention_refuses(lib, over, what):
    assert lib.rnnt_cache_attend(C.byref(a_cache()), C.byref(an_attend(**over)), None) == E_ARG
    assert what in message(lib)


def test_attention_workspace(lib):
    long = a_cache(n_pages=1000, width=1000)
    need = lib.rnnt_cache_attend_workspace(C.byref(long), C.byref(an_attend(max_len=16000)))
    assert need > 0
    for over in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=FAKE + 4)):
        assert lib.rnnt_cache_attend(C.byref(long), C.byref(an_attend(max_len=16000, **over)), None) == E_ARG and "workspace" in message(lib)


def test_python_side_refuses_host_tensors():
    import torch
    from paper_2506_00185_amd import KVCache, RnntBeamError, reorder_states, select_tokens
    with pytest.raises(RnntBeamError, match="GPU"):
        select_tokens(torch.zeros(1, 2, 8), torch.zeros(1, 2, dtype=torch.float64))
    with pytest.raises(RnntBeamError, match="GPU"):
        reorder_states(torch.zeros(1, 2, dtype=torch.int32), [torch.zeros(1, 2, 3)])
    with pytest.raises(RnntBeamError, match="GPU"):
        KVCache(1, 16, 1, 64, device="cpu")


def a_meta_cache(n_pages=4, page_size=16, heads=2, dim=64):
    """A cache whose tensors have shapes and no memory: calls get as far as the check of the device."""
    import torch
    from paper_2506_00185_amd import KVCache
    from paper_2506_00185_amd.tokens import _Cache
    c = KVCache.__new__(KVCache)
    c.k = c.v = torch.empty(n_pages, heads, page_size, dim, dtype=torch.float16, device="meta")
    c.k_exp = c.v_exp = torch.empty(n_pages, heads, page_size, dtype=torch.uint8, device="meta")
    c.n_pages, c.heads, c.page_size, c.dim, c.device, c.format = n_pages, heads, page_size, dim, c.k.device, "f16"
    c._c = _Cache(struct_size=C.sizeof(_Cache), format=1, n_pages=n_pages, page_size=page_size, heads=heads, dim=dim)
    return c


def test_sizes_that_32_bits_do_not_hold_are_refused(lib):
    """(The library counts in 32 bits: passed on, 2^32 + 5 would be 5.)"""
    import torch
    from paper_2506_00185_amd import KVCache, RnntBeamError, nbest_tree, reorder_states, select_tokens
    big = 2**32 + 5
    meta = lambda *shape, dtype=torch.float16: torch.empty(shape, dtype=dtype, device="meta")  # noqa: E731
    i32, f64 = torch.int32, torch.float64
    c = a_meta_cache()
    table, start, rows = meta(3, 8, dtype=i32), meta(3, dtype=i32), meta(3, 5, 2, 64)
    states = [(meta(2, 3, big), 0), (meta(2, 3, big, 2)[..., :1], 0), (meta(big, 2, 3, 4), 1)]
    calls = [lambda: select_tokens(meta(2, 3, big), meta(2, 3, dtype=f64)), lambda: select_tokens(meta(big, 3, 7), meta(big, 3, dtype=f64)),
             lambda: KVCache.from_tensors(meta(big, 1, 1, 16), meta(big, 1, 1, 16), meta(big, 1, 1), meta(big, 1, 1)),
             lambda: KVCache.from_tensors(meta(1, 1, 2**32 + 16, 16), meta(1, 1, 2**32 + 16, 16), meta(1, 1, 2**32 + 16), meta(1, 1, 2**32 + 16)),
             lambda: KVCache.from_tensors(meta(1, 1, 16, 2**32 + 16), meta(1, 1, 16, 2**32 + 16), meta(1, 1, 16), meta(1, 1, 16)),
             lambda: KVCache.from_tensors(meta(1, big, 1, 16), meta(1, big, 1, 16), meta(1, big, 1), meta(1, big, 1)),
             lambda: c.write(meta(3, big, 2, 64), meta(3, big, 2, 64), table, start), lambda: c.read(table, start, big),
             lambda: c.write(rows, rows, meta(3, big, dtype=i32), start), lambda: c.write(meta(big, 1, 2, 64), meta(big, 1, 2, 64), meta(big, 8, dtype=i32), meta(big, dtype=i32)),
             lambda: c.attend(meta(3, big, 2, 64), table, start), lambda: c.attend(meta(3, 1, big - 1, 64), table, start),
             lambda: c.attend(rows, table, start, parents=meta(3, big, dtype=i32)),
             lambda: nbest_tree(np.zeros((1, 1, 4), np.int32), np.ones((1, 1), np.int32), max_nodes=big),
             lambda: nbest_tree(np.broadcast_to(np.int32(0), (1, 0, big)), np.zeros((1, 0), np.int32))]
    calls += [lambda t=t, lead=lead: reorder_states(meta(2, 3, dtype=i32), [t], lead=lead) for t, lead in states[1:]]
    for i, call in enumerate(calls):
        with pytest.raises(RnntBeamError, match="2\\^31"):
            call()
            raise AssertionError(i)
    with pytest.raises(RnntBeamError, match="GPU"):  # one run of so many elements is counted in 64 bits
        reorder_states(meta(2, 3, dtype=i32), [states[0][0]])
    for eos in (2**32 + 3, 3 - 2**32, 7, -2):
        with pytest.raises(RnntBeamError, match="eos"):
            select_tokens(meta(2, 3, 7), meta(2, 3, dtype=f64), eos=eos)
    with pytest.raises(RnntBeamError, match="max_len"):
        c.attend(rows, table, start, max_len=3 - 2**32)


def differentiable_calls():
    """(call, floating tensors by name) for each call; ``call`` takes what replaces one of them."""
    import torch
    from paper_2506_00185_amd import reorder_states, select_tokens
    meta = lambda *shape, dtype=torch.float16: torch.empty(shape, dtype=dtype, device="meta")  # noqa: E731
    i32, f64 = torch.int32, torch.float64
    table, start, parents = meta(3, 8, dtype=i32), meta(3, dtype=i32), meta(2, 3, dtype=i32)

    def cache_call(name):
        def call(kk=None, vv=None, a=None, b=None, out=None):
            c = a_meta_cache()
            c.k, c.v = c.k if kk is None else kk, c.v if vv is None else vv
            rows = [meta(3, 5, 2, 64) if t is None else t for t in (a, b)]
            if name == "write":
                c.write(*rows, table, start)
            elif name == "read":
                c.read(table, start, 5)
            else:
                c.attend(rows[0], table, start, out=out)
        return call

    cache, rows = dict(kk=meta(4, 2, 16, 64), vv=meta(4, 2, 16, 64)), meta(3, 5, 2, 64)
    return {"select": (lambda x=meta(2, 3, 7), s=meta(2, 3, dtype=f64), o=meta(2, 3, dtype=f64): select_tokens(x, s, out=(o, parents, parents, None)),
                       dict(x=meta(2, 3, 7), s=meta(2, 3, dtype=f64), o=meta(2, 3, dtype=f64))),
            "reorder": (lambda x=meta(2, 3, 4): reorder_states(parents, [meta(2, 3), x]), dict(x=meta(2, 3, 4))),
            "write": (cache_call("write"), dict(cache, a=rows, b=rows)), "read": (cache_call("read"), cache),
            "attend": (cache_call("attend"), dict(cache, a=rows, out=rows))}


@pytest.mark.parametrize("name", ["select", "reorder", "write", "read", "attend"])
def test_tensors_that_require_a_gradient_are_refused(name):
    import torch
    from paper_2506_00185_amd import RnntBeamError
    call, tensors = differentiable_calls()[name]
    for k, t in tensors.items():
        leaf = torch.empty_like(t, requires_grad=True)
        for x in (leaf, leaf * 1.0, leaf.view_as(leaf)):
            with pytest.raises(RnntBeamError, match="gradient"):
                call(**{k: x})
            with torch.no_grad(), pytest.raises(RnntBeamError, match="GPU"):
                call(**{k: x})
            with pytest.raises(RnntBeamError, match="GPU"):
                call(**{k: x.detach()})


@pytest.mark.parametrize("name", ["select", "reorder", "write", "read", "attend"])
def test_forward_tangents_are_refused(name):
    import torch
    import torch.autograd.forward_ad as fw
    from paper_2506_00185_amd import RnntBeamError
    call, tensors = differentiable_calls()[name]
    for k, t in tensors.items():
        with fw.dual_level():
            dual = fw.make_dual(t, torch.empty_like(t))
            for guard in (torch.enable_grad, torch.no_grad):
                with guard(), pytest.raises(RnntBeamError, match="tangent"):
                    call(**{k: dual})
            with pytest.raises(RnntBeamError, match="GPU"):
                call(**{k: t})


def test_prefix_trees_of_other_integers():
    from paper_2506_00185_amd import RnntBeamError, nbest_tree
    tokens, lens = np.array([[[1, 2], [1, 3]]]), np.array([[2, 2]])
    want = nbest_tree(tokens.astype(np.int32), lens.astype(np.int32))
    for dtype in (np.int64, np.uint8, np.int16, np.float32):
        got = nbest_tree(tokens.astype(dtype), lens.astype(dtype))
        assert all(np.array_equal(got[k], want[k]) for k in want)
    for t, n in [(tokens + 2**32, lens), (tokens, lens + 2**32), (tokens + 0.5, lens), (tokens, lens * 0.75), (tokens * np.nan, lens)]:
        with pytest.raises(RnntBeamError, match="int32"):
            nbest_tree(t, n)
    with pytest.raises(RnntBeamError, match="beyond cap"):  # (and no room is made for such a length)
        nbest_tree(tokens, lens + 2**30)


def test_the_current_device_comes_back_when_a_stream_or_an_input_is_refused(monkeypatch):
    """Without a GPU: the device's and the stream's scopes are stand-ins that write down when they are entered and left."""
    import contextlib
    from types import SimpleNamespace
    import torch
    from paper_2506_00185_amd import RnntBeamError, tokens
    log = []

    @contextlib.contextmanager
    def scope(what):
        log.append(("in", what))
        try:
            yield
        finally:
            log.append(("out", what))

    def tensor(device, fails=False):
        def record_stream(stream):
            if fails:
                raise RuntimeError("no")
        device = torch.device(device)
        return SimpleNamespace(is_cuda=device.type == "cuda", get_device=lambda: device.index, device=device, record_stream=record_stream)

    monkeypatch.setattr(torch.cuda, "device", lambda i: scope(f"device {i}"))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: scope("stream"))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda i: SimpleNamespace(device=torch.device("cuda", i), cuda_stream=0))
    T = SimpleNamespace(device_of=lambda: 0)
    mine, other = (SimpleNamespace(device=torch.device("cuda", i), cuda_stream=7) for i in (1, 0))
    here = tensor("cuda:1")
    for stream, inputs, error in [(other, [here], RnntBeamError), (mine, [here, None, tensor("cpu")], RnntBeamError), (mine, [here, tensor("cuda:0")], RnntBeamError),
                                  (mine, [here, tensor("cuda:1", fails=True)], RuntimeError)]:
        with pytest.raises(error):
            tokens._enter(T, here, stream, inputs)
        assert sorted(w for e, w in log if e == "in") == sorted(w for e, w in log if e == "out"), log
    raw, close = tokens._enter(T, here, mine, [here, None])
    assert raw.value == 7 and log[-2:] == [("in", "device 1"), ("in", "stream")]
    close.close()
    assert log[-2:] == [("out", "stream"), ("out", "device 1")]


# ---------------------------------------------------------------- the plain implementations themselves
def test_plain_formats():
    import torch
    g = np.random.default_rng(0)
    for fmt, dtype, top in (("e4m3", torch.float8_e4m3fn, 448.0), ("f16", torch.float16, 2.0**15)):
        for e in (-140, -126, -20, 0, 5, 127):
            x = np.float32(g.standard_normal(64) * 2.0**e) if e < 127 else np.float32(g.uniform(-3.4e38, 3.4e38, 64))
            y, b = R.quantise(x, fmt)
            assert np.abs(y).max() <= top
            assert b == 1 or np.abs(y).max() > top / 2 - 2.0**9 * (fmt == "f16") - 16
            np.testing.assert_array_equal(torch.from_numpy(y).float().to(dtype).double().numpy(), y)  # representable
            np.testing.assert_array_equal(torch.ldexp(torch.from_numpy(x).double(), torch.tensor(127 - b)).float().to(dtype).double().numpy(), y)
        assert R.quantise(np.array([448.0, 1.0]), "e4m3")[1] == 127 and R.quantise(np.array([449.0, 1.0]), "e4m3")[1] == 128
        assert R.quantise(np.zeros(4), fmt)[1] == 127 and R.quantise(np.array([1.0, math.nan]), fmt)[1] == 255


def test_plain_selection_and_paths():
    s, p, t, d = R.select(np.log(np.array([[[0.5, 0.25, 0.25], [0.1, 0.8, 0.1]]])), np.array([[0.0, -0.1]]), eos=1)
    np.testing.assert_array_equal(p, [[1, 0]])
    np.testing.assert_array_equal(t, [[1, 0]])
    np.testing.assert_allclose(s, [[-0.1 + math.log(0.8), math.log(0.5)]], rtol=1e-12)
    np.testing.assert_array_equal(d, [[True, False]])
    assert R.path_of([-1, 0, 0, 1], 3) == [3, 1, 0] and R.path_of([-1, -2, 1], 2) is None and R.path_of([0], 0) is None
