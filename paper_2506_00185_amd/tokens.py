"""Operators for networks that the caller runs itself: ctypes binding of rnnt_select_tokens, rnnt_reorder_states,
rnnt_cache_write / read / attend and rnnt_nbest_tree.  Argument checks and marshalling only; include/rnnt_beam.h says what each does.

Tensors live on one GPU; work goes to ``stream`` (default: the current stream of that GPU) and the calls return without
waiting.  Outputs and workspaces are torch tensors of that stream, so that all calls may be captured into a graph.  The calls are for
inference: a tensor that requires a gradient is refused, among the outputs and what is overwritten too, unless gradients are off; one with a tangent of
forward differentiation always.  What a call overwrites counts as changed in place: a backward pass that saved it says so."""
from __future__ import annotations

import contextlib
import ctypes as C

import numpy as np

from .binding import RnntBeamError, _check, load_library

_FORMATS = {"e4m3": 0, "f16": 1}


class _Select(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("type", C.c_int32), ("B", C.c_int32), ("beam", C.c_int32), ("V", C.c_int32),
                ("eos", C.c_int32), ("logits", C.c_void_p), ("stride_b", C.c_int64), ("stride_k", C.c_int64),
                ("scores", C.c_void_p), ("done", C.c_void_p), ("out_scores", C.c_void_p), ("out_parent", C.c_void_p),
                ("out_token", C.c_void_p), ("out_done", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class _States(C.Structure):
    _fields_ = [("data", C.c_void_p), ("lead_stride", C.c_int64), ("b_stride", C.c_int64), ("slot_stride", C.c_int64),
                ("inner_stride", C.c_int64), ("row_bytes", C.c_int64), ("lead", C.c_int32), ("inner", C.c_int32)]


class _Cache(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("format", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32),
                ("heads", C.c_int32), ("dim", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p),
                ("v_exp", C.c_void_p), ("table", C.c_void_p), ("table_stride", C.c_int64), ("width", C.c_int32)]


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_b", C.c_int64), ("stride_n", C.c_int64), ("stride_h", C.c_int64)]


class _Attend(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("type", C.c_int32), ("B", C.c_int32), ("n", C.c_int32), ("tree", C.c_int32),
                ("q_heads", C.c_int32), ("scale", C.c_float), ("max_len", C.c_int32), ("q", _Rows), ("out", C.c_void_p),
                ("lens", C.c_void_p), ("parents", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


def _refuse(ok, what):
    if not ok:
        raise RnntBeamError(what)


_MOST = 0x7fffffff


def _sizes(a, b=0, c=0):
    """The library counts in 32 bits, and ctypes passes on the last 32 bits of what does not fit."""
    if a > _MOST or b > _MOST or c > _MOST:
        raise RnntBeamError(f"sizes must be below 2^31, not {max(a, b, c)}")


class _Torch:
    """What the calls below need of torch, looked up once: a call is a few microseconds in all."""

    def __init__(self):
        import torch
        import torch.autograd.forward_ad as forward
        # (of equals the faster one: a tensor like another, the device's number without a check that there is a device)
        self.empty, self.empty_like = torch.empty, torch.empty_like
        self.device_of = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
        self.f64, self.f32, self.i32, self.u8, self.bool = torch.float64, torch.float32, torch.int32, torch.uint8, torch.bool
        self.grads, self.forward = torch.is_grad_enabled, forward
        self.types = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
        self.changed = getattr(torch._C, "_increment_version", None) or torch.autograd.graph.increment_version
        # (the pointer alone where this torch gives it without an object around it)
        self.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        self.lib = load_library()


_loaded = None


def _torch():
    global _loaded
    if _loaded is None:
        _loaded = _Torch()
    return _loaded


def _type_of(T, t, what):
    code = T.types.get(t.dtype)
    if code is None:
        raise RnntBeamError(f"{what} must be float32, float16 or bfloat16")
    return code


def _no_derivatives(T, *tensors):
    if T.grads():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise RnntBeamError("a tensor requires a gradient, of which this call has none: detach it, or call under torch.no_grad()")
    if T.forward._current_level >= 0:
        for t in tensors:
            if t is not None and T.forward.unpack_dual(t).tangent is not None:
                raise RnntBeamError("a tensor has a tangent, of which this call has none: take its primal")


def _array(t, what, dtype, shape, device):
    """Pointer of a contiguous tensor of that type, shape and device."""
    if t.dtype != dtype or t.device != device or t.shape != shape or not t.is_contiguous():
        _refuse(t.dtype == dtype, f"{what} must be {dtype}")
        _refuse(t.device == device, f"{what} is on {t.device}, not on {device}")
        _refuse(t.shape == shape, f"{what} must have shape {tuple(shape)}, not {tuple(t.shape)}")
        raise RnntBeamError(f"{what} must be contiguous")
    return t.data_ptr()


def _enter(T, t, stream, inputs):
    """(pointer of the stream, what to close behind the call): the call's device and stream are the current ones in between, so that what
    it allocates belongs to them."""
    if not t.is_cuda:
        raise RnntBeamError("tensors must be on the GPU: there is no CPU fallback")
    index = t.get_device()
    if stream is None and index == T.device_of():
        return C.c_void_p(T.raw_stream(index)), None
    import torch
    with contextlib.ExitStack() as stack:  # (closed here only if something below is refused)
        stack.enter_context(torch.cuda.device(index))
        if stream is not None and stream != torch.cuda.current_stream(index):
            _refuse(stream.device == t.device, f"the stream is of {stream.device}, the tensors are on {t.device}")
            for x in inputs:  # of another stream: not to be given away before this call has used them
                if x is not None:
                    _refuse(x.device == t.device, f"a tensor is on {x.device}, not on {t.device}")
                    x.record_stream(stream)
            stack.enter_context(torch.cuda.stream(stream))
        scope = stack.pop_all()
    return C.c_void_p((stream or torch.cuda.current_stream(index)).cuda_stream), scope


def select_tokens(logits, scores, done=None, eos=-1, out=None, stream=None):
    """rnnt_select_tokens: one step of a beam search over logits [B, beam, V] (float32, float16 or bfloat16, last dimension contiguous) with
    the hypotheses' scores float64 [B, beam].  Returns (scores float64, parents int32, tokens int32, done bool or None), each [B, beam].
    ``eos``: the token that finishes a hypothesis (-1: none), ``done`` bool [B, beam]: which have finished.  ``out``: such a tuple to write
    to; it may hold ``scores`` and ``done`` themselves."""
    T = _torch()
    if logits.dim() != 3:
        raise RnntBeamError("logits must be [B, beam, V]")
    B, beam, V = logits.shape
    stride_b, stride_k, stride_v = logits.stride()
    if V < 1 or (V > 1 and stride_v != 1):
        raise RnntBeamError("the last dimension of logits must be contiguous")
    _sizes(B, beam, V)
    if not -1 <= eos < V:
        raise RnntBeamError("eos must be a token, or -1")
    _no_derivatives(T, logits, scores, *(out or ()))
    dev, shape = logits.device, (B, beam)
    s = _Select(C.sizeof(_Select), _type_of(T, logits, "logits"), B, beam, V, eos, logits.data_ptr(), stride_b, stride_k,
                _array(scores, "scores", T.f64, shape, dev))
    if done is not None:
        s.done = _array(done, "done", T.bool, shape, dev)
    raw, scope = _enter(T, logits, stream, (logits, scores, done) + tuple(out or ()))
    given = out
    try:
        if out is None:
            whole = T.empty_like(scores, dtype=T.i32)
            out = (T.empty_like(scores), whole, T.empty_like(whole), T.empty_like(scores, dtype=T.bool) if eos >= 0 else None)
            s.out_scores, s.out_parent, s.out_token = out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr()
        else:
            _refuse(len(out) == 4, "out must be (scores, parents, tokens, done)")
            s.out_scores = _array(out[0], "out scores", T.f64, shape, dev)
            s.out_parent = _array(out[1], "out parents", T.i32, shape, dev)
            s.out_token = _array(out[2], "out tokens", T.i32, shape, dev)
            if out[3] is not None:
                _array(out[3], "out done", T.bool, shape, dev)
        if out[3] is not None:
            s.out_done = out[3].data_ptr()
        need = T.lib.rnnt_select_tokens_workspace(B, beam, V)
        if need:
            work = T.empty(need, dtype=T.u8, device=dev)
            s.workspace, s.workspace_bytes = work.data_ptr(), need
        _check(T.lib.rnnt_select_tokens(C.byref(s), raw))
        if given is not None:
            T.changed([t for t in out if t is not None])
    finally:
        if scope:
            scope.close()
    return out


def _rows_of(shape, strides, which):
    """(rows, stride, run) of trailing dimensions: a run of contiguous elements, repeated at one stride."""
    if len(shape) == 1 and strides[0] == 1:
        return 1, 0, shape[0]
    run, dims = 1, list(zip(shape, strides))
    while dims and (dims[-1][0] == 1 or dims[-1][1] == run):
        run *= dims.pop()[0]
    dims = [d for d in dims if d[0] != 1]
    if not dims:
        return 1, 0, run
    rows, stride = dims.pop()
    while dims and dims[-1][1] == stride * rows:
        rows *= dims.pop()[0]
    _refuse(not dims, f"state {which}: the dimensions behind the slots must be one run of elements or runs at one stride")
    return rows, stride, run


def reorder_states(parents, states, lead=0, stream=None):
    """rnnt_reorder_states: state[b, k] = state[b, parents[b, k]] in place, for each of up to 16 tensors of any type, [B, beam, ...] behind
    ``lead`` (0 or 1) dimensions, e.g. of layers.  parents int32 [B, beam]; those outside 0 .. beam - 1 leave their slot as it is."""
    T = _torch()
    if parents.dim() != 2 or parents.numel() == 0:
        raise RnntBeamError("parents must be [B, beam]")
    shape, dev = parents.shape, parents.device
    ptr = _array(parents, "parents", T.i32, shape, dev)
    _refuse(lead in (0, 1), "lead must be 0 or 1")
    _refuse(len(states) <= 16, "at most 16 tensors")
    _no_derivatives(T, *states)
    _sizes(shape[0])
    views = (_States * max(len(states), 1))()
    for i, t in enumerate(states):
        full, strides, size = t.shape, t.stride(), t.element_size()
        if t.device != dev or full[lead:lead + 2] != shape:
            _refuse(t.device == dev, f"state {i} is on {t.device}, not on {dev}")
            raise RnntBeamError(f"state {i} must be [{'layers, ' * lead}B, beam, ...]")
        rows, stride, run = _rows_of(full[lead + 2:], strides[lead + 2:], i)
        outer, outer_stride = (full[0], strides[0]) if lead else (1, 0)
        _sizes(outer, rows)
        views[i] = _States(t.data_ptr(), outer_stride * size, strides[lead] * size, strides[lead + 1] * size, stride * size, run * size, outer, rows)
    raw, scope = _enter(T, parents, stream, (parents, *states))
    try:
        _check(T.lib.rnnt_reorder_states(C.c_void_p(ptr), shape[0], shape[1], views, len(states), raw))
        T.changed(states)
    finally:
        if scope:
            scope.close()


class KVCache:
    """The paged cache of one attention layer (rnnt_cache_t): ``k`` and ``v`` [n_pages, heads, page_size, dim], torch.float8_e4m3fn
    (format "e4m3") or torch.float16 ("f16"), ``k_exp`` and ``v_exp`` uint8 [n_pages, heads, page_size]; a row's values are
    k 2^(k_exp - 127).  Which pages belong to a sequence is the caller's to say, by a table int32 [B, width] with each call.  Sequences may
    share pages, hypotheses of a beam those of their common prefix; with pages of one token a table lists each hypothesis' tokens."""

    def __init__(self, n_pages, page_size, heads, dim, format="e4m3", device="cuda:0"):
        import torch
        _refuse(format in _FORMATS, "format must be 'e4m3' or 'f16'")
        dtype = torch.float16 if format == "f16" else torch.float8_e4m3fn
        shape = (n_pages, heads, page_size)
        # (zeros that are written as bytes: a row that was never written reads as zeros)
        k, v = (torch.zeros(shape + (dim * (2 if format == "f16" else 1),), dtype=torch.uint8, device=device).view(dtype) for _ in range(2))
        self._set(k, v, torch.full(shape, 127, dtype=torch.uint8, device=device), torch.full(shape, 127, dtype=torch.uint8, device=device))

    @classmethod
    def from_tensors(cls, k, v, k_exp, v_exp):
        """A cache over arrays that the caller holds."""
        self = cls.__new__(cls)
        self._set(k, v, k_exp, v_exp)
        return self

    def _set(self, k, v, k_exp, v_exp):
        import torch
        _refuse(k.dim() == 4 and k.dtype in (torch.float16, torch.float8_e4m3fn), "k must be [n_pages, heads, page_size, dim], float8_e4m3fn or float16")
        for size in k.shape:
            _sizes(size)
        _refuse(k.is_cuda, "tensors must be on the GPU: there is no CPU fallback")
        self.k, self.v, self.k_exp, self.v_exp, self.device = k, v, k_exp, v_exp, k.device
        self.n_pages, self.heads, self.page_size, self.dim = k.shape
        self._written = (k, v, k_exp, v_exp)
        self.format = "f16" if k.dtype == torch.float16 else "e4m3"
        self._c = _Cache(struct_size=C.sizeof(_Cache), format=_FORMATS[self.format], n_pages=self.n_pages, page_size=self.page_size,
                         heads=self.heads, dim=self.dim)
        self._c.k = _array(k, "k", k.dtype, tuple(k.shape), self.device)
        self._c.v = _array(v, "v", k.dtype, tuple(k.shape), self.device)
        self._c.k_exp = _array(k_exp, "k_exp", torch.uint8, tuple(k.shape[:3]), self.device)
        self._c.v_exp = _array(v_exp, "v_exp", torch.uint8, tuple(k.shape[:3]), self.device)

    def _view(self, T, table, B):
        shape, strides = table.shape, table.stride()
        if len(shape) != 2 or table.dtype != T.i32 or shape[0] != B or shape[1] < 1 or table.device != self.device or (shape[1] > 1 and strides[1] != 1):
            _refuse(len(shape) == 2 and table.dtype == T.i32 and shape[0] == B and shape[1] >= 1, f"table must be int32 [{B}, width]")
            _refuse(table.device == self.device, f"table is on {table.device}, not on {self.device}")
            raise RnntBeamError("rows of table must be contiguous")
        _sizes(B, shape[1])
        c = _Cache.from_buffer_copy(self._c)
        c.table, c.table_stride, c.width = table.data_ptr(), strides[0], shape[1]
        return c

    def _rows(self, t, what, heads):
        shape, strides = t.shape, t.stride()
        if len(shape) != 4 or shape[2] != heads or shape[3] != self.dim or t.device != self.device or strides[3] != 1:
            _refuse(len(shape) == 4 and shape[2] == heads and shape[3] == self.dim, f"{what} must be [B, n, {heads}, {self.dim}]")
            _refuse(t.device == self.device, f"{what} is on {t.device}, not on {self.device}")
            raise RnntBeamError(f"the last dimension of {what} must be contiguous")
        return _Rows(t.data_ptr(), strides[0], strides[1], strides[2])

    def _counts(self, T, start, count, B):
        return (C.c_void_p(_array(start, "start", T.i32, (B,), self.device)),
                C.c_void_p(_array(count, "count", T.i32, (B,), self.device)) if count is not None else None)

    def write(self, k, v, table, start, count=None, stream=None):
        """rnnt_cache_write: rows k, v [B, n, heads, dim] (float32, float16 or bfloat16) to positions start[b] + i, i < count[b] (None: n)."""
        T = _torch()
        shape = k.shape
        if k.dtype != v.dtype or shape != v.shape or len(shape) != 4:
            raise RnntBeamError(f"k and v must be [B, n, {self.heads}, {self.dim}] of one type and shape")
        B, n = shape[0], shape[1]
        _sizes(n)
        code, c = _type_of(T, k, "k"), self._view(T, table, B)
        _no_derivatives(T, k, v, self.k, self.v)
        rk, rv = self._rows(k, "k", self.heads), self._rows(v, "v", self.heads)
        first, many = self._counts(T, start, count, B)
        raw, scope = _enter(T, k, stream, (k, v, table, start, count, self.k, self.v, self.k_exp, self.v_exp))
        try:
            _check(T.lib.rnnt_cache_write(C.byref(c), C.byref(rk), C.byref(rv), code, B, n, first, many, raw))
            T.changed(self._written)
        finally:
            if scope:
                scope.close()

    def read(self, table, start, n, dtype=None, count=None, stream=None):
        """rnnt_cache_read: (k, v) [B, n, heads, dim] of ``dtype`` (default float32), the rows at positions start[b] + i; zeros from count[b] on and
        where there is no page."""
        T = _torch()
        dtype = dtype or T.f32
        code, B = T.types.get(dtype), table.shape[0]
        _refuse(code is not None, "dtype must be float32, float16 or bfloat16")
        _sizes(n)
        _no_derivatives(T, self.k, self.v)
        c = self._view(T, table, B)
        first, many = self._counts(T, start, count, B)
        raw, scope = _enter(T, self.k, stream, (table, start, count, self.k, self.v, self.k_exp, self.v_exp))
        try:
            heads, dim = self.heads, self.dim
            k = T.empty((B, n, heads, dim), dtype=dtype, device=self.device)
            out = (k, T.empty_like(k))
            if n:
                rk, rv = (_Rows(t.data_ptr(), n * heads * dim, heads * dim, dim) for t in out)
                _check(T.lib.rnnt_cache_read(C.byref(c), C.byref(rk), C.byref(rv), code, B, n, first, many, raw))
        finally:
            if scope:
                scope.close()
        return out

    def attend(self, q, table, lens, parents=None, scale=None, max_len=None, out=None, stream=None):
        """rnnt_cache_attend: attention of queries q [B, n, q_heads, dim] over lens[b] tokens (int32 [B]) and the new nodes behind them, whose
        rows have been written to positions lens[b] + i.  ``parents`` int32 [B, tree], tree >= n: the queries are the last n nodes of a tree,
        each sees its ancestors (-1: none) and itself; less than -1: padding.  None: each node follows the one before it, n = 1 is a step of
        a search.  ``scale``: default dim ** -0.5.  ``max_len``: a bound of lens + tree, by which work is split (default: all that
        the table holds).  Returns [B, n, q_heads, dim] of q's type; ``out``: contiguous, such a tensor to write to."""
        T = _torch()
        shape = q.shape
        if len(shape) != 4:
            raise RnntBeamError("q must be [B, n, q_heads, dim]")
        B, n, heads, dim = shape
        _sizes(n, heads)
        _no_derivatives(T, q, self.k, self.v, out)
        c = self._view(T, table, B)
        rows = self._rows(q, "q", heads)
        bound = self.page_size * c.width if max_len is None else max_len
        if bound < 0:
            raise RnntBeamError("max_len must not be negative")
        a = _Attend(C.sizeof(_Attend), _type_of(T, q, "q"), B, n, n, heads, dim ** -0.5 if scale is None else scale, min(bound, _MOST), rows)
        a.lens = _array(lens, "lens", T.i32, (B,), self.device)
        if parents is not None:
            _refuse(parents.dim() == 2, "parents must be [B, tree]")
            _sizes(parents.shape[1])
            a.tree = parents.shape[1]
            a.parents = _array(parents, "parents", T.i32, (B, a.tree), self.device)
        lib = T.lib
        raw, scope = _enter(T, q, stream, (q, table, lens, parents, out, self.k, self.v, self.k_exp, self.v_exp))
        try:
            given = out
            need = lib.rnnt_cache_attend_workspace(C.byref(c), C.byref(a))
            if need < 0:
                _check(need)
            if out is None:
                out = T.empty_like(q) if q.is_contiguous() else T.empty(shape, dtype=q.dtype, device=self.device)
                a.out = out.data_ptr()
            else:
                a.out = _array(out, "out", q.dtype, shape, self.device)
            if need:
                work = T.empty(need, dtype=T.u8, device=self.device)
                a.workspace, a.workspace_bytes = work.data_ptr(), need
            _check(lib.rnnt_cache_attend(C.byref(c), C.byref(a), raw))
            if given is not None:
                T.changed((out,))
        finally:
            if scope:
                scope.close()
        return out


def _int32(a, what):
    """A contiguous int32 array of the same numbers."""
    a = np.asarray(a)
    with np.errstate(invalid="ignore"):
        out = np.ascontiguousarray(a, np.int32)
    _refuse(a.dtype == np.int32 or bool((out == a).all()), f"{what} must be int32, or numbers that it holds")
    return out


def nbest_tree(tokens, lens, max_nodes=None) -> dict:
    """rnnt_nbest_tree: the prefix trees of the n-best lists of BeamDecoder.results (tokens [B, beam, cap], lens [B, beam], numpy), to be
    rescored by one KVCache.attend: tokens and parents [B, nodes] (parent -1: first token, -2: padding), leaf [B, beam]: the node at which each
    hypothesis ends (-1: empty), n_nodes [B]."""
    tokens, lens = _int32(tokens, "tokens"), _int32(lens, "lens")
    _refuse(tokens.ndim == 3 and lens.shape == tokens.shape[:2], "tokens must be [B, beam, cap], lens [B, beam]")
    B, beam, cap = tokens.shape
    _sizes(B, beam, cap)
    # (lengths beyond cap are refused below)
    room = max(1, int(np.clip(lens, 0, cap).sum(1, dtype=np.int64).max(initial=0))) if max_nodes is None else max_nodes
    _sizes(room)
    tok, par = (np.empty((B, room), np.int32) for _ in range(2))
    leaf, n_nodes = np.empty((B, beam), np.int32), np.empty(B, np.int32)
    most = _check(load_library().rnnt_nbest_tree(*(C.c_void_p(x.ctypes.data) for x in (tokens, lens)), B, beam, cap, room,
                                                 *(C.c_void_p(x.ctypes.data) for x in (tok, par, leaf, n_nodes))))
    width = max(1, most) if max_nodes is None else max_nodes
    return dict(tokens=np.ascontiguousarray(tok[:, :width]), parents=np.ascontiguousarray(par[:, :width]), leaf=leaf, n_nodes=n_nodes)
