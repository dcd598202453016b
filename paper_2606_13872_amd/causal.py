"""Causal attention of packed prompts with grouped heads (include/sra.h, sra_causal_*): argument marshalling.

    plan = CausalPlan(q_lens, heads, kv_heads, head_dim)       # once per set of lengths
    o, lse = causal_forward(q, k, v, plan)                     # every layer
    g = causal_backward(q, k, v, o, lse, do, plan)             # g["dq"], g["dk"], g["dv"]
"""
from __future__ import annotations

import ctypes
import weakref
from typing import Dict, Optional, Sequence

import numpy as np

from . import sra as _s

INT32_MAX = 2**31 - 1  # sizes reach the library in 32 bits, which ctypes would cut them to

_handles_declared = False


class _CausalProblem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("num_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("q_lens", ctypes.c_void_p), ("k_lens", ctypes.c_void_p)]


def _lib():
    global _handles_declared
    L = _s.lib()
    if not _handles_declared:
        vp, i32, i64, sz, f = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        psz = ctypes.POINTER(sz)
        for name, args in {
            "sra_causal_plan_create": [ctypes.POINTER(_CausalProblem), ctypes.c_int, ctypes.POINTER(vp)],
            "sra_causal_plan_destroy": [vp],
            "sra_causal_plan_sizes": [vp, psz, psz, psz],
            "sra_causal_plan_tables": [vp, vp, sz],
            "sra_causal_plan_mask": [vp, ctypes.c_int, i32, i32, vp],
            "sra_causal_forward": [vp] * 5 + [i64] * 3 + [vp, vp, f, vp, sz, vp],
            "sra_causal_backward": [vp] * 5 + [i64] * 3 + [vp] * 6 + [f, vp, sz, vp],
        }.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = ctypes.c_int
        _handles_declared = True
    return L


def _lens(x, name) -> np.ndarray:
    a = np.asarray(x.detach().cpu() if hasattr(x, "detach") else x)
    if a.ndim != 1 or a.size == 0 or a.dtype.kind not in "iu":
        raise _s._bad(f"{name} must be a non-empty sequence of integers")
    if a.min() < 0 or a.max() > INT32_MAX:
        raise _s._bad(f"{name}: lengths must be between 0 and 2^31 - 1")
    return np.ascontiguousarray(a.astype(np.int32))


class _PlanHandle(ctypes.c_void_p):
    """An sra_causal_plan, destroyed with the last object that holds it (copies of a CausalPlan share it)."""


class CausalPlan:
    """The tile schedule of causal attention for one set of lengths, with its tables on `device` (default: the
    current GPU; without a GPU only the host hooks work). Made once, used by every layer and call with these lengths.
    A plan is made outside a graph's capture, and kept as long as graphs that hold calls with it (they read its tables).
    Making it, and the first call on another GPU, copies the tables and waits for the current stream: make plans for coming
    lengths ahead.

    q_lens: tokens of each packed sequence. k_lens: its keys, where they differ (the sequence continues earlier
    keys: token i of nq sees the keys j <= i + nk - nq). backward=False plans the forward alone.
    """

    def __init__(self, q_lens: Sequence[int], heads: int, kv_heads: int, head_dim: int,
                 k_lens: Optional[Sequence[int]] = None, backward: bool = True, device=None):
        L = _lib()
        self.q_lens = _lens(q_lens, "q_lens")
        self.k_lens = self.q_lens if k_lens is None else _lens(k_lens, "k_lens")
        if self.k_lens.shape != self.q_lens.shape:
            raise _s._bad("q_lens and k_lens must have one length per sequence each")
        self.heads, self.kv_heads, self.head_dim, self.backward = int(heads), int(kv_heads), int(head_dim), bool(backward)
        if max(len(self.q_lens), abs(self.heads), abs(self.kv_heads), abs(self.head_dim)) > INT32_MAX:
            raise _s._bad("sequences, heads and head_dim must be below 2^31")
        p = _CausalProblem(len(self.q_lens), self.heads, self.kv_heads, self.head_dim, self.q_lens.ctypes.data,
                           self.k_lens.ctypes.data)
        h = _PlanHandle()
        _s._check(L.sra_causal_plan_create(ctypes.byref(p), 1 if backward else 0, ctypes.byref(h)))
        weakref.finalize(h, L.sra_causal_plan_destroy, h.value)
        self._handle = h
        t, f, b = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
        _s._check(L.sra_causal_plan_sizes(h, ctypes.byref(t), ctypes.byref(f), ctypes.byref(b)))
        self._table_bytes, self.forward_workspace, self.backward_workspace = t.value, f.value, b.value
        self.n_q, self.n_k = int(self.q_lens.sum(dtype=np.int64)), int(self.k_lens.sum(dtype=np.int64))
        self.q_shape = (self.n_q, self.heads, self.head_dim)
        self.k_shape = (self.n_k, self.kv_heads, self.head_dim)
        self.lse_shape = (self.heads, self.n_q)
        self._tables = {}
        torch = _s._tm()
        if device is not None or torch.cuda.is_available():
            dev = torch.device("cuda" if device is None else device)
            if dev.type != "cuda":
                raise _s._bad(f"a plan's tables must be on a GPU (HIP device), got {dev}")
            self._upload(torch.cuda.current_device() if dev.index is None else dev.index)

    def _upload(self, index: int):
        """The tables on GPU `index` (its address and the stream that they were copied on)."""
        torch = _s._tm()
        if torch.cuda.is_current_stream_capturing():
            raise _s._bad(f"the plan's tables are not on GPU {index}: make the plan, for this GPU, before the capture")
        host = np.zeros(max(1, self._table_bytes), dtype=np.uint8)
        _s._check(_lib().sra_causal_plan_tables(self._handle, host.ctypes.data, self._table_bytes))
        with torch.cuda.device(index):
            t = torch.from_numpy(host).to(torch.device("cuda", index))
            torch.cuda.current_stream().synchronize()  # any stream may read them from now on
            self._tables[index] = (t, torch.cuda.current_stream().cuda_stream)
        return self._tables[index]

    def _device_tables(self, dev, stream):
        """Address of the tables on `dev`, kept for the work that is enqueued on `stream` now."""
        t, home = self._tables.get(dev.index) or self._upload(dev.index)
        if stream.value != home and (stream.value or home):
            t.record_stream(_s._tm().cuda.current_stream(dev))
        return t.data_ptr()

    def mask(self, which: int, sequence: int, head: int) -> np.ndarray:
        """sra_causal_plan_mask: how often launch `which` (SCHED_*) computes each (token, key) pair."""
        ok = 0 <= sequence < len(self.q_lens)
        out = np.zeros((self.q_lens[sequence], self.k_lens[sequence]) if ok else (1, 1), dtype=np.uint8)
        buf = out if out.size else np.zeros(1, dtype=np.uint8)
        _s._check(_lib().sra_causal_plan_mask(self._handle, which, sequence, head, buf.ctypes.data))
        return out


def _rows(t, name, shape):
    """Checks an input, bf16 [tokens, heads, head_dim] with contiguous heads; its token stride (0: at most one token)."""
    torch = _s._tm()
    if not isinstance(t, torch.Tensor) or t.dtype != torch.bfloat16 or t.shape != shape:
        _s._expect(t, name, shape, torch.bfloat16, False)  # says what is wrong
    st = t.stride()
    if shape[0] and (st[2] != 1 or (shape[1] > 1 and st[1] != shape[2])):
        raise _s._bad(f"{name} must be [tokens, heads, head_dim] with contiguous heads")
    if shape[0] <= 1:
        return 0
    if st[0] < shape[1] * shape[2]:
        raise _s._bad(f"{name}: tokens overlap (stride {st[0]})")
    return st[0]


def _addr(t):
    """Its address (None without elements)."""
    return None if t is None else t.data_ptr() or None


def _qkv(q, k, v, plan):
    if not isinstance(plan, CausalPlan):
        raise _s._bad("plan must be a CausalPlan")
    return _rows(q, "q", plan.q_shape), _rows(k, "k", plan.k_shape), _rows(v, "v", plan.k_shape)


def _no_alias(out, named):
    """Output buffers must not share memory with inputs or each other (they are written while inputs are read)."""
    spans = []
    for name, t in named:
        if t is None or t.numel() == 0:
            continue
        a = t.data_ptr()
        b = a + t.element_size() * (sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1)
        for other, c, d, w in spans:
            if a < d and c < b and (w or name in out):
                raise _s._bad(f"output {name if name in out else other} overlaps {other if name in out else name}")
        spans.append((name, a, b, name in out))


def _call(dev, fn):
    """fn(stream) with `dev` as the current device."""
    torch = _s._tm()
    if torch.cuda.current_device() == dev.index:
        return fn(_s._stream_ptr(dev))
    with torch.cuda.device(dev):
        return fn(_s._stream_ptr(dev))


def causal_forward(q, k, v, plan: CausalPlan, scale: Optional[float] = None, out: Optional[Dict] = None):
    """Causal attention of packed prompts. Returns (o, lse).

    q: bf16 [tokens, heads, head_dim], k, v: bf16 [keys, kv_heads, head_dim], heads contiguous, a token stride each
    (views of one packed buffer work); query head h reads K/V head h // (heads // kv_heads). o: bf16 like q, dense;
    lse: fp32 [heads, tokens], natural log. Rows that see no key have o = 0 and lse = -inf. An infinity or NaN in v
    may reach any row of its sequence. scale: None or <= 0 selects 1 / sqrt(head_dim). `out` may hold caller buffers
    o, lse (dense) and workspace (uint8), which must not overlap the inputs. A wrong dtype, shape, layout or
    device raises SRAError (SRA_ERR_INVALID_ARGUMENT) before anything reaches the library.
    """
    torch = _s._tm()
    qs, ks, vs = _qkv(q, k, v, plan)
    dev = q.device
    if out:
        _s._precheck_outs(out, [("o", plan.q_shape, torch.bfloat16), ("lse", plan.lse_shape, torch.float32)])
    _s._same_device((("q", q), ("k", k), ("v", v)), dev)
    need = plan.forward_workspace
    if out:
        o = _s._out(out, "o", plan.q_shape, torch.bfloat16, dev)
        lse = _s._out(out, "lse", plan.lse_shape, torch.float32, dev)
        ws = _s._workspace(out, need, dev)
        _no_alias(out, (("q", q), ("k", k), ("v", v), ("o", o), ("lse", lse), ("workspace", ws)))
    else:
        o = torch.empty(plan.q_shape, dtype=torch.bfloat16, device=dev)
        lse = torch.empty(plan.lse_shape, dtype=torch.float32, device=dev)
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _s._check(_call(dev, lambda s: _lib().sra_causal_forward(
        plan._handle, plan._device_tables(dev, s), _addr(q), _addr(k), _addr(v), qs, ks, vs, _addr(o), _addr(lse),
        0.0 if scale is None else float(scale), _addr(ws), 0 if ws is None else ws.numel(), s)))
    return o, lse


def causal_backward(q, k, v, o, lse, do, plan: CausalPlan, scale: Optional[float] = None, out: Optional[Dict] = None):
    """Gradients of causal_forward. Returns dict dq, dk, dv (bf16, dense, overwritten).

    o and lse as causal_forward wrote them, do: bf16 like o, dense. dk and dv are summed over the query heads that
    share a K/V head. An infinity or NaN in an input may reach any gradient of its sequence. `out` may hold caller
    buffers dq, dk, dv (dense) and workspace (uint8).
    """
    torch = _s._tm()
    qs, ks, vs = _qkv(q, k, v, plan)
    if not plan.backward:
        raise _s._bad("the plan was made with backward=False")
    bf = torch.bfloat16
    dense = (("o", o, plan.q_shape, bf), ("do", do, plan.q_shape, bf), ("lse", lse, plan.lse_shape, torch.float32))
    for name, t, shape, dtype in dense:
        _s._expect(t, name, shape, dtype, True)
    dev = q.device
    grads = (("dq", plan.q_shape), ("dk", plan.k_shape), ("dv", plan.k_shape))
    ins = (("q", q), ("k", k), ("v", v), ("o", o), ("lse", lse), ("do", do))
    if out:
        _s._precheck_outs(out, [(n, shape, bf) for n, shape in grads])
    _s._same_device(ins, dev)
    need = plan.backward_workspace
    if out:
        g = {n: _s._out(out, n, shape, bf, dev) for n, shape in grads}
        ws = _s._workspace(out, need, dev)
        _no_alias(out, ins + (*g.items(), ("workspace", ws)))
    else:
        g = {n: torch.empty(shape, dtype=bf, device=dev) for n, shape in grads}
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _s._check(_call(dev, lambda s: _lib().sra_causal_backward(
        plan._handle, plan._device_tables(dev, s), _addr(q), _addr(k), _addr(v), qs, ks, vs, _addr(o), _addr(lse),
        _addr(do), _addr(g["dq"]), _addr(g["dk"]), _addr(g["dv"]), 0.0 if scale is None else float(scale), _addr(ws),
        0 if ws is None else ws.numel(), s)))
    return g
