"""Selection of a beam's best tokens from a caller's logits and the reordering of states, against a plain implementation in 64 bits."""
import numpy as np
import pytest

import token_ref as R

pytestmark = pytest.mark.gpu

# A key is score + (x - lse).  The polynomial of the exponentials is off by at most 5.5e-11 of each term, so of their sum and so of lse; what is left are
# roundings to 53 bits of numbers below 1e3 (sums of positive terms: 64 lanes' shares of a few hundred each, 2^-53 a step).
KEY_ATOL = 6e-11 + 1e3 * 2.0**-52


def run(logits, scores, done=None, eos=-1, **kw):
    import torch
    from paper_2506_00185_amd import select_tokens
    g = select_tokens(logits, torch.from_numpy(scores).cuda(), None if done is None else torch.from_numpy(done).cuda(), eos, **kw)
    torch.cuda.synchronize()
    return [None if t is None else t.cpu().numpy() for t in g]


def check(logits, scores, done=None, eos=-1, **kw):
    """logits: a CUDA tensor."""
    x = logits.double().cpu().numpy()
    want = R.select(x, scores, done, eos)
    # different keys are far enough apart for the tolerance not to decide between them
    assert R.select_margin(x, scores, done, eos) > 2 * KEY_ATOL
    got = run(logits, scores, done, eos, **kw)
    np.testing.assert_array_equal(got[1], want[1])
    np.testing.assert_array_equal(got[2], want[2])
    assert np.array_equal(np.isinf(got[0]), np.isinf(want[0]))
    np.testing.assert_allclose(got[0], want[0], rtol=0, atol=KEY_ATOL)
    if eos >= 0:
        np.testing.assert_array_equal(got[3], want[3])
    else:
        assert got[3] is None
    return got


def make(B, K, V, dtype, seed, spread=2.5):
    import torch
    g = np.random.default_rng(seed)
    logits = torch.from_numpy(g.standard_normal((B, K, V)) * spread).to(R.torch_type(dtype)).cuda()
    return logits, -20 - 3 * g.random((B, K))


# one launch and two, tiles that end anywhere, rows that start anywhere (odd V of 16-bit types), every beam's number of lists
SIZES = [(1, 1, 1), (2, 3, 1), (1, 4, 2), (3, 16, 2), (2, 5, 17), (1, 1, 63), (4, 2, 64), (7, 7, 65), (1, 4, 1024), (3, 16, 1023), (2, 16, 1025), (2, 4, 4096),
         (2, 4, 4097), (1, 1, 16384), (1, 1, 16385), (2, 13, 5000), (1, 10, 8192), (2, 8, 8193), (1, 12, 32003), (1, 16, 60001), (1, 3, 100003), (130, 1, 300),
         (40, 9, 2000), (1, 1, 1000003)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,K,V", SIZES)
def test_sizes_and_types(B, K, V, dtype):
    check(*make(B, K, V, dtype, B + 31 * K + V))


@pytest.mark.parametrize("V", [1, 50, 5000, 40000])
@pytest.mark.parametrize("K", [1, 6, 16])
def test_finished_hypotheses_and_empty_slots(K, V):
    logits, scores = make(4, K, V, "f32", 5 * V + K)
    g = np.random.default_rng(V)
    done = g.random((4, K)) < 0.4
    done[1] = True  # all finished: the beam in order of its scores
    scores[2, K // 2:] = -np.inf  # empty slots
    scores[3] = -np.inf
    scores[3, 0] = 0.0  # a search's first step
    done[3] = False
    for eos in (0, V - 1):
        got = check(logits, scores, done, eos)
        assert got[3][1].all() and (got[2][1] == eos).all()
    # nothing at all to choose from
    s, p, t, d = run(logits, np.full((4, K), -np.inf), np.zeros((4, K), bool), 0)
    assert np.isneginf(s).all() and (p == -1).all() and (t == -3).all() and not d.any()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,K,V", [(4, 4, 1024), (3, 16, 900), (1, 1, 16000), (2, 10, 8192), (1, 12, 32003), (3, 5, 12345)])
def test_keys_have_the_bits_of_float64(B, K, V, dtype):
    """Against 64-bit mantissas.  The sum is off by the polynomial's 3.3e-16, four half steps of its evaluation, n times what ln 2 in float64 leaves of it (2.4e-17,
    n up to 145 for terms of e^-100, what is below weighs nothing) and up to 64 additions of a lane and 16 of lanes and parts: 1.3e-14.  Three more
    roundings, of numbers below 64."""
    logits, scores = make(B, K, V, dtype, 3 * B + K + V)
    x = logits.double().cpu().numpy().astype(np.longdouble)
    assert np.finfo(np.longdouble).nmant >= 63
    top = x.max(-1, keepdims=True)
    keys = scores.astype(np.longdouble)[..., None] + (x - (top + np.log(np.exp(x - top).sum(-1, keepdims=True))))
    got = run(logits, scores)
    assert np.abs(got[0]).max() < 64 and np.abs(x).max() < 64
    there = np.take_along_axis(keys.reshape(B, -1), got[1].astype(np.int64) * V + got[2], 1)
    assert np.abs(got[0] - there).max() <= 1.3e-14 + 3 * 64 * 2.0**-53


def run_in(fill, logits, scores, done=None, eos=-1):
    """The C call with a workspace of the caller's that holds ``fill`` in every byte."""
    import ctypes as C
    import torch
    from paper_2506_00185_amd import load_library
    from paper_2506_00185_amd.tokens import _Select
    lib, (B, K, V) = load_library(), logits.shape
    assert logits.is_contiguous()
    need = lib.rnnt_select_tokens_workspace(B, K, V)
    assert need > 0
    work = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
    s, d = torch.from_numpy(scores).cuda(), None if done is None else torch.from_numpy(done).cuda()
    out = [torch.empty(B, K, dtype=t, device="cuda") for t in (torch.float64, torch.int32, torch.int32, torch.bool)]
    code = [torch.float32, torch.float16, torch.bfloat16].index(logits.dtype)
    a = _Select(C.sizeof(_Select), code, B, K, V, eos, logits.data_ptr(), K * V, V, s.data_ptr(), None if d is None else d.data_ptr(),
                *(t.data_ptr() for t in out[:3]), out[3].data_ptr() if eos >= 0 else None, work.data_ptr(), need)
    assert lib.rnnt_select_tokens(C.byref(a), C.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in (out if eos >= 0 else out[:3])]


# two launches with 1024 rows and more, so that lists are few: one to a row for beams from 3 on
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,K,V", [(342, 3, 5462), (400, 3, 8192), (1025, 1, 16400), (513, 2, 8200), (260, 4, 4200), (128, 9, 2000), (104, 10, 8192), (64, 16, 1100),
                                   (64, 16, 8193)])
def test_what_a_workspace_held_does_not_matter(B, K, V, dtype):
    """Words that read as no candidate, as logits of 1.5 and 48.6, above most and all of the logits, and as NaN."""
    logits, scores = make(B, K, V, dtype, B + K + V)
    eos = V // 2
    done = np.random.default_rng(V).random((B, K)) < 0.1
    want = check(logits, scores, done, eos)
    for fill in (0x00, 0xbf, 0xc2, 0xff):
        for a, b in zip(run_in(fill, logits, scores, done, eos), want):
            np.testing.assert_array_equal(a, b)


def test_finished_hypotheses_logits_are_not_read():
    logits, scores = make(2, 4, 3000, "f32", 1)
    logits[:, 1] = float("nan")
    done = np.zeros((2, 4), bool)
    done[:, 1] = True
    check(logits, scores, done, 7)


@pytest.mark.parametrize("V", [40, 6000])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_without_candidates(V, dtype):
    import torch
    logits, scores = make(6, 4, V, dtype, V)
    logits[0, 1, V // 2] = float("nan")
    logits[1, 0, V - 1] = float("inf")
    logits[2, 3] = -float("inf")
    logits[3, :, 1:] = -float("inf")         # one token left
    logits[4, :, V // 3:] = -float("inf")    # tiles of nothing
    logits[5] = -float("inf")                # an utterance of nothing
    scores[0, 2], scores[1, 2] = np.nan, -np.inf
    want = R.select(logits.double().cpu().numpy(), np.where(np.isnan(scores), -np.inf, scores))
    got = run(logits, scores)
    np.testing.assert_array_equal(got[1], want[1])
    np.testing.assert_array_equal(got[2], want[2])
    assert (got[1][5] == -1).all() and (got[2][5] == -3).all() and np.isneginf(got[0][5]).all()
    assert (got[1][3] >= 0).sum() == 4  # each hypothesis' one token
    # masks of the type's lowest value: candidates behind all others
    low = float(torch.finfo(logits.dtype).min)
    logits, scores = make(2, 4, V, dtype, V + 1)
    logits[0, :, 2:] = low
    logits[1, 1:] = -float("inf")
    logits[1, 0, 2:] = low
    scores[:] = [[0.0, -1.0, -2.5, -3.25]] * 2
    got = run(logits, scores)
    assert (got[2][0] < 2).all()
    want = R.select(logits.double().cpu().numpy(), scores)
    np.testing.assert_array_equal(got[2], want[2])
    np.testing.assert_array_equal(got[1], want[1])


@pytest.mark.parametrize("K,V", [(1, 900), (4, 900), (16, 900), (4, 30000), (16, 30000)])
@pytest.mark.parametrize("kind", ["equal", "blocks", "rising", "falling", "few"])
def test_ties_and_orders(K, V, kind):
    """Equal keys go to the smallest index; logits that rise with it change a list at every tile."""
    import torch
    g = np.random.default_rng(K + V)
    x = {"equal": np.zeros((2, K, V)), "blocks": np.repeat(g.integers(0, 3, (2, K, V // 50)), 50, 2), "rising": np.arange(V) / 64.0 + np.zeros((2, K, V)),
         "falling": -np.arange(V) / 64.0 + np.zeros((2, K, V)), "few": g.integers(0, 4, (2, K, V))}[kind]
    # keys of two rows are equal (scores[0]), or far apart
    scores = np.stack([np.zeros(K), -np.arange(K) * 0.37])
    logits = torch.from_numpy(x.astype(np.float32)).cuda()
    got = run(logits, scores)
    want = R.select(x, scores)
    if kind in ("equal", "rising", "falling"):  # rows alike: sums alike, keys equal on both sides
        np.testing.assert_array_equal(got[1], want[1])
        np.testing.assert_array_equal(got[2], want[2])
    else:  # scores[1]'s rows; of those of equal score the order hangs on their sums
        np.testing.assert_array_equal(got[1][1], want[1][1])
        np.testing.assert_array_equal(got[2][1], want[2][1])
    np.testing.assert_allclose(got[0], want[0], rtol=0, atol=KEY_ATOL)
    again = run(logits, scores)
    for a, b in zip(got[:3], again[:3]):
        np.testing.assert_array_equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [333, 20011])
def test_strides_and_places(V, dtype):
    """Rows apart, batches apart, in another order, from an odd element on."""
    import torch
    base, scores = make(3, 5, V + 9, dtype, V)
    check(base[:, :, 3:V + 3], scores)
    wide, _ = make(6, 11, V, dtype, V + 1)
    check(wide[::2, 1::2], scores)
    turned, _ = make(5, 3, V, dtype, V + 2)
    check(turned.transpose(0, 1), scores)
    one, _ = make(3, 1, V, dtype, V + 3)
    check(one.expand(3, 5, V), -np.arange(15.0).reshape(3, 5) * 0.7)  # hypotheses that share a row


def test_values_far_from_zero():
    import torch
    for shift, spread in ((3e4, 2.0), (-3e4, 2.0), (0.0, 300.0), (0.0, 1e-6)):
        logits, scores = make(2, 4, 9000, "f32", 3, spread)
        # (float32 logits at 3e4 are 2^-9 apart: many equal)
        check(logits + shift, scores)
    logits, scores = make(2, 4, 9000, "f32", 4)
    logits[:, :, 4000:] += 900.0  # a tile far above the first one's largest
    check(logits, scores)
    logits[:, :, :4000] += 1900.0
    check(logits, scores)


@pytest.mark.parametrize("V", [60, 9000])
def test_scores_that_float32_does_not_hold(V):
    logits, _ = make(4, 4, V, "f32", 12)
    # (next to such a score a logit is nothing: the keys of a hypothesis are equal, its largest logits win)
    scores = np.array([[-1e300, -2e300, -3e300, -4e300], [-1e39, -1e300, -5.0, -1e40], [1e300, 2e300, 1e39, -1e39], [-np.inf, -1e300, -np.inf, -1e300]])
    got = check(logits, scores)
    assert got[1][0].tolist() == [0] * 4 and got[1][1].tolist() == [2] * 4
    assert got[2][0].tolist() == logits[0, 0].topk(4).indices.tolist()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("K,V", [(1, 50), (5, 900), (4, 9000), (16, 1500)])
def test_zeros_of_both_signs_are_equal(K, V, dtype):
    import torch
    g = np.random.default_rng(V)
    x = np.where(g.random((3, K, V)) < 0.5, -0.0, 0.0)
    x[g.random(x.shape) < 0.4] = -1.0
    x[1] = np.where(g.random((K, V)) < 0.01, x[1], -1.0)  # few of them
    logits = torch.from_numpy(x).to(R.torch_type(dtype)).cuda()
    scores = np.sort(g.random((3, K)))
    want, got = R.select(x, scores), run(logits, scores)
    np.testing.assert_array_equal(got[1], want[1])
    np.testing.assert_array_equal(got[2], want[2])


def test_the_longest_row():
    """Indices up to the last that is allowed; equal logits everywhere else."""
    import math
    import torch
    V = 2**31 - 2**16
    logits = torch.zeros(1, 1, V, dtype=torch.bfloat16, device="cuda")
    for at in (V - 1, V // 2 + 1, 0):
        logits[0, 0, at] = 12.0
        got = run(logits, np.array([[-3.0]]))
        logits[0, 0, at] = 0.0
        assert got[1][0, 0] == 0 and got[2][0, 0] == at
        # (a lane adds V / 64 / 256 terms, less than 2^17, each sum off by up to half a step)
        assert abs(got[0][0, 0] - (9.0 - math.log(V - 1 + math.exp(12.0)))) <= KEY_ATOL + (2**17 + 64) * 2.0**-53
    del logits
    torch.cuda.empty_cache()


def test_in_place_and_on_another_stream():
    import torch
    from paper_2506_00185_amd import select_tokens
    for V in (700, 50000):
        logits, scores = make(3, 6, V, "f32", V)
        done = np.zeros((3, 6), bool)
        done[:, 2] = True
        want = R.select(logits.double().cpu().numpy(), scores, done, 4)
        s, d = torch.from_numpy(scores).cuda(), torch.from_numpy(done).cuda()
        p, t = torch.empty(3, 6, dtype=torch.int32, device="cuda"), torch.empty(3, 6, dtype=torch.int32, device="cuda")
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        out = select_tokens(logits, s, d, 4, out=(s, p, t, d), stream=side)
        assert out[0] is s and out[3] is d
        side.synchronize()
        np.testing.assert_array_equal(p.cpu().numpy(), want[1])
        np.testing.assert_array_equal(t.cpu().numpy(), want[2])
        np.testing.assert_array_equal(d.cpu().numpy(), want[3])
        np.testing.assert_allclose(s.cpu().numpy(), want[0], rtol=0, atol=KEY_ATOL)


def test_two_graphs_replayed_in_turn():
    import torch
    from paper_2506_00185_amd import reorder_states, select_tokens
    graphs = []
    for V in (900, 40000):
        logits, scores = make(2, 5, V, "bf16", V)
        s = torch.from_numpy(scores).cuda()
        state = torch.randn(2, 5, 33, device="cuda")
        select_tokens(logits, s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = select_tokens(logits, s)
            reorder_states(out[1], [state])
        graphs.append((g, logits, s, state, out, V))
    for turn in range(3):
        for g, logits, s, state, out, V in graphs:
            fresh, scores = make(2, 5, V, "bf16", 100 * turn + V % 7)
            logits.copy_(fresh)
            s.copy_(torch.from_numpy(scores))
            before = state.clone()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            want = R.select(fresh.double().cpu().numpy(), scores)
            np.testing.assert_array_equal(out[1].cpu().numpy(), want[1])
            np.testing.assert_array_equal(out[2].cpu().numpy(), want[2])
            np.testing.assert_array_equal(state.cpu().numpy(), before.cpu().numpy()[np.arange(2)[:, None], want[1]])


def test_what_python_refuses():
    import torch
    from paper_2506_00185_amd import RnntBeamError, select_tokens
    x, s = torch.zeros(2, 3, 10, device="cuda"), torch.zeros(2, 3, dtype=torch.float64, device="cuda")
    d = torch.zeros(2, 3, dtype=torch.bool, device="cuda")
    bad = [(x[0], s), (x.double(), s), (x.transpose(1, 2), s), (x, s.float()), (x, s[:1]), (x, s.t()), (x, s.cpu()), (x[:, :, ::2], s), (x, s, d), (x, s, d, 10),
           (x, s, d.int(), 3), (x, s, d[:1], 3), (x[:, :, :0], s)]
    for args in bad:
        with pytest.raises(RnntBeamError):
            select_tokens(*args)
    with pytest.raises(RnntBeamError, match="gradient"):
        select_tokens(x.clone().requires_grad_(), s)
    with torch.no_grad():
        select_tokens(x.clone().requires_grad_(), s)
    with pytest.raises(RnntBeamError, match="beam"):
        select_tokens(torch.zeros(1, 17, 5, device="cuda"), torch.zeros(1, 17, dtype=torch.float64, device="cuda"))
    with pytest.raises(RnntBeamError):
        select_tokens(x, s, out=(s, s, s, None))


# ---------------------------------------------------------------- reordering
def check_reorder(states, parents, lead=0, **kw):
    import torch
    from paper_2506_00185_amd import reorder_states
    B, K = parents.shape
    at = np.where((parents >= 0) & (parents < K), parents, np.arange(K))
    rows = torch.arange(B)[:, None]
    want = [(t.cpu()[:, rows, torch.from_numpy(at)] if lead else t.cpu()[rows, torch.from_numpy(at)]) for t in states]
    reorder_states(torch.from_numpy(parents.astype(np.int32)).cuda(), states, lead=lead, **kw)
    torch.cuda.synchronize()
    for t, w in zip(states, want):
        assert torch.equal(t.cpu().contiguous().view(torch.uint8), w.contiguous().view(torch.uint8))


@pytest.mark.parametrize("K", [1, 2, 4, 5, 8, 9, 16])
@pytest.mark.parametrize("tail", [(), (1,), (7,), (640,), (3, 33), (2, 5, 1000)])
def test_reorder_shapes(K, tail):
    import torch
    g = np.random.default_rng(K)
    for B in (1, 3, 33):
        for dtype in (torch.float32, torch.uint8, torch.bfloat16, torch.float64, torch.int32):
            t = (torch.rand(B, K, *tail) * 200).to(dtype).cuda()
            check_reorder([t], g.integers(-1, K, (B, K)))


def test_reorder_orders():
    """Cycles, exchanges, one parent for all, empty slots, parents that are none."""
    import torch
    K = 8
    parents = np.array([np.roll(np.arange(K), 1), np.arange(K)[::-1], np.zeros(K, int), np.arange(K), np.full(K, -1), np.full(K, 7), [100, -5, 3, 2, 1, 0, 8, 7]])
    for n in (1, 1000, 40000):
        check_reorder([torch.randn(len(parents), K, n, device="cuda")], parents)


def test_reorder_of_views():
    import torch
    g = np.random.default_rng(0)
    B, K, L = 3, 6, 2
    parents = g.integers(0, K, (B, K))
    cache = torch.randn(L, B, K, 4, 50, 16, device="cuda").half()
    whole = cache.clone()
    check_reorder([cache[:, :, :, :, :37], torch.randn(L, B, K, 11, device="cuda")], parents, lead=1)
    assert torch.equal(cache[..., 37:, :], whole[..., 37:, :])
    table = torch.arange(B * K * 40, dtype=torch.int32, device="cuda").reshape(B, K, 40)
    whole = table.clone()
    check_reorder([table[:, :, 1:14]], parents)
    assert torch.equal(table[:, :, 14:], whole[:, :, 14:]) and torch.equal(table[:, :, 0], whole[:, :, 0])
    turned = torch.randn(K, 9, B, device="cuda")
    check_reorder([turned.permute(2, 0, 1)], parents)  # slots outermost, rows of single elements
    both = torch.randn(B, K, 20, 2, device="cuda")
    check_reorder([both[..., 0], both[..., 1]], parents)  # interleaved, not overlapping
    odd = torch.zeros(B * K * 100 + 1, dtype=torch.uint8, device="cuda").random_()
    check_reorder([odd[1:].view(B, K, 100)], parents)
    # many tensors of different widths at once
    check_reorder([torch.randn(B, K, n, device="cuda").to(d) for n in (1, 5, 64, 999) for d in (torch.float32, torch.half, torch.float64, torch.int8)], parents)
    check_reorder([torch.randn(B, K, 0, device="cuda"), torch.randn(B, K, 3, device="cuda")], parents)
    check_reorder([], parents)


def test_reorder_far_apart():
    """Offsets beyond 32 bits."""
    import torch
    from paper_2506_00185_amd import reorder_states
    big = torch.empty(3, 2, 1 << 30, dtype=torch.uint8, device="cuda")
    view = big[:, :, -4099:]
    view.random_()
    want = view.flip(1).cpu()
    reorder_states(torch.tensor([[1, 0]] * 3, dtype=torch.int32, device="cuda"), [view])
    assert torch.equal(view.cpu(), want)


def test_reorder_on_another_stream_and_refusals():
    import torch
    from paper_2506_00185_amd import RnntBeamError, reorder_states
    side = torch.cuda.Stream()
    t = torch.randn(2, 3, 500, device="cuda")
    torch.cuda.synchronize()
    check_reorder([t], np.array([[1, 2, 0], [2, 2, 2]]), stream=side)
    p = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    x = torch.zeros(2, 3, 4, 5, 6, device="cuda")
    for parents, states, kw in [(p.long(), [x], {}), (p[0], [x], {}), (p, [x[:1]], {}), (p, [x.cpu()], {}), (p, [x], dict(lead=1)), (p, [x], dict(lead=2)), (p, [x] * 17, {}),
                                (p, [x, x], {}), (p, [torch.zeros(3, device="cuda").expand(2, 3)], {}), (p, [x[:, :, :, ::2, ::2]], {}), (p.t().contiguous().t(), [x], {})]:
        with pytest.raises(RnntBeamError):
            reorder_states(parents, states, **kw)
