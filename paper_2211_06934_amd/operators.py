"""Python binding of the language-model operators of the C ABI (include/diffopt.h).

Argument marshalling only, as in ``diffopt``: every function is the C entry
point ``diffopt_<name>``, takes device tensors, writes into tensors that the
caller owns and enqueues on the current torch stream unless one is given.
Activations are fp32 or bf16, one type per call; weights, tables, statistics
and states are fp32.  [B, T, heads, width] tensors may have any strides but
that of their last axis; rows of logits may lie any distance apart.

Where a call needs scratch memory it is allocated on the current stream;
``workspace`` takes a uint8 tensor of ``*_workspace`` bytes instead (as a
program that captures its step into a graph keeps it).
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from .diffopt import _check, _done, _lib, _native, _stream

F32, BF16 = 0, 1
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}

_vp, _i64, _i32, _f64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double


class _Heads(ctypes.Structure):
    _fields_ = [("data", _vp), ("stride_b", _i64), ("stride_t", _i64), ("stride_h", _i64)]


_hp = ctypes.POINTER(_Heads)
_QK = [_vp, _vp, _vp, _vp, _i64, _vp, _i32, _i64, _i64, _i64, _i64, _i64, _i64, _i64, _i32, _i32, _f64]
_ROWS = [_vp, _i64, _i64, _i64, _i32, _vp, _i32, _vp, _i64, _f64]
_SIGNATURES = {
    "diffopt_linattn_fwd": (_i32, [_hp, _hp, _hp, _vp, _vp, _vp, *[_i64] * 6, _i32, _f64, _hp, _vp, _vp, _i64, _vp]),
    "diffopt_linattn_bwd": (_i32, [_hp, _vp, _hp, _hp, _hp, _vp, _vp, _vp, *[_i64] * 6, _i32, _f64, _hp, _hp, _hp, _vp, _vp, _i64,
                                   _vp]),
    "diffopt_linattn_workspace": (_i64, [*[_i64] * 6, _i32, _i32]),
    "diffopt_linattn_step": (_i32, [_hp, _hp, _hp, _vp, *[_i64] * 5, _i32, _f64, _vp, _hp, _vp]),
    "diffopt_qknorm_rope_fwd": (_i32, [_hp, _hp, *_QK, _hp, _hp, _vp]),
    "diffopt_qknorm_rope_bwd": (_i32, [_hp, _hp, _hp, _hp, *_QK, _hp, _hp, _vp, _vp, _vp, _i64, _vp]),
    "diffopt_qknorm_rope_bwd_bwd": (_i32, [_hp, _hp, _vp, _vp, _hp, _hp, _hp, _hp, *_QK, _hp, _hp, _hp, _hp, _vp, _vp, _vp, _i64,
                                           _vp]),
    "diffopt_qknorm_rope_workspace": (_i64, [_i64] * 5),
    "diffopt_distill_fwd": (_i32, [*_ROWS, _vp, _vp, _vp, _i64, _vp]),
    "diffopt_distill_bwd": (_i32, [_vp, *_ROWS, _vp, _vp, _i64, _vp, _vp]),
    "diffopt_distill_fwd_bwd": (_i32, [_vp, *_ROWS, _vp, _vp, _vp, _i64, _vp, _vp, _i64, _vp]),
    "diffopt_distill_bwd_bwd": (_i32, [_vp, _i64, _vp, _vp, *_ROWS, _vp, _vp, _vp, _i64, _vp, _vp, _i64, _vp]),
    "diffopt_distill_workspace": (_i64, [_i64, _i64, _i32, _i64]),
}
for _name, (_res, _args) in _SIGNATURES.items():
    if not hasattr(_lib, _name):
        raise ImportError("the library lacks %s: it is older than its sources; rebuild with "
                          "`python paper_2211_06934_amd/build.py`" % _name)
    getattr(_lib, _name).restype, getattr(_lib, _name).argtypes = _res, _args


def _tensor(x, what: str, dtype, shape, device=None) -> torch.Tensor:
    if not isinstance(x, torch.Tensor):
        raise TypeError("%s: expected a torch.Tensor" % what)
    if not x.is_cuda:
        raise ValueError("%s: tensor must live in device memory" % what)
    if device is not None and x.device != device:
        raise ValueError("%s: expected a tensor on %s, got %s" % (what, device, x.device))
    if x.dtype != dtype:
        raise ValueError("%s: expected dtype %s, got %s" % (what, dtype, x.dtype))
    if tuple(x.shape) != tuple(shape):
        raise ValueError("%s: expected shape %s, got %s" % (what, tuple(shape), tuple(x.shape)))
    return x


def _heads(x, what: str, like: torch.Tensor, shape, optional: bool = False):
    """A [B, T, heads, width] tensor of the call's type as the C struct."""
    if x is None and optional:
        return None
    _tensor(x, what, like.dtype, shape, like.device)
    if x.shape[3] > 1 and x.stride(3) != 1 and x.numel() > 0:
        raise ValueError("%s: the elements of a head must be contiguous" % what)
    return _Heads(x.data_ptr() or None, x.stride(0), x.stride(1), x.stride(2))


def _ref(h):
    return None if h is None else ctypes.byref(h)


def _apart(x, what: str) -> None:
    """A result's elements must not overlap one another."""
    at = 1
    for stride, size in sorted((s, n) for s, n in zip(x.stride(), x.shape) if n > 1):
        if stride < at:
            raise ValueError("%s: elements of a result overlap" % what)
        at += stride * (size - 1)


def _flat(x, what: str, like: torch.Tensor, shape, optional: bool = False, dtype=torch.float32) -> Optional[int]:
    """Address of a contiguous tensor of this shape."""
    if x is None:
        if optional:
            return None
        raise TypeError("%s: expected a torch.Tensor" % what)
    _tensor(x, what, dtype, shape, like.device)
    if not x.is_contiguous():
        raise ValueError("%s: tensor must be contiguous" % what)
    return x.data_ptr() or None


def _type_of(x, what: str) -> int:
    if not isinstance(x, torch.Tensor):
        raise TypeError("%s: expected a torch.Tensor" % what)
    if not x.is_cuda:
        raise ValueError("%s: tensor must live in device memory" % what)
    if x.dtype not in _DTYPES:
        raise ValueError("%s: expected dtype torch.float32 or torch.bfloat16, got %s" % (what, x.dtype))
    return _DTYPES[x.dtype]


def _here(workspace, stream) -> bool:
    """Whether scratch memory that the call allocates may be allocated on the current stream."""
    return stream is None or workspace is not None


def _scratch(given, need: int, device, stream):
    """(tensor kept alive, address, bytes) of a call's workspace, allocated on the call's stream: it returns to that stream's
    pool, so nothing enqueued elsewhere takes it while the call still uses it."""
    if given is None and need > 0:
        if stream is None:
            given = torch.empty(need, dtype=torch.uint8, device=device)
        else:
            with torch.cuda.stream(torch.cuda.ExternalStream(_stream(stream), device=device)):
                given = torch.empty(need, dtype=torch.uint8, device=device)
    elif given is None:
        pass
    elif not isinstance(given, torch.Tensor) or given.dtype != torch.uint8 or not given.is_cuda or not given.is_contiguous():
        raise ValueError("workspace: expected a contiguous uint8 tensor in device memory")
    elif given.device != device:
        raise ValueError("workspace: expected a tensor on %s, got %s" % (device, given.device))
    elif given.numel() < need:
        raise ValueError("workspace: expected at least %d bytes, got %d" % (need, given.numel()))
    return given, (None if given is None else given.data_ptr() or None), 0 if given is None else given.numel()


# ---- linear attention -------------------------------------------------------


def _dims(q, k, v, axes: int):
    for x, what in ((q, "q"), (k, "k"), (v, "v")):
        if not isinstance(x, torch.Tensor) or x.dim() != axes:
            raise ValueError("%s: expected a tensor of %d axes" % (what, axes))
    return q.shape[-2], k.shape[-2], q.shape[-1], v.shape[-1]


def linattn_workspace(B: int, T: int, H: int, Hk: int, Dk: int, Dv: int, dtype=torch.float32, backward: bool = False) -> int:
    """diffopt_linattn_workspace: bytes that linattn_fwd (linattn_bwd) needs for these sizes."""
    n = int(_lib.diffopt_linattn_workspace(B, T, H, Hk, Dk, Dv, _DTYPES[dtype], int(backward)))
    if n < 0:
        raise ValueError("linattn: sizes that the operator refuses")
    return n


def linattn_fwd(q, k, v, log_decay, out, state=None, state_out=None, lengths=None, scale: float = 1.0, workspace=None,
                stream=None) -> None:
    """diffopt_linattn_fwd: out_t = scale S_t^T q_t with S_t = exp(log_decay) S_{t-1} + k_t v_t^T.

    q [B, T, H, Dk], k [B, T, Hk, Dk], v [B, T, Hk, Dv] -> out [B, T, H, Dv]; log_decay [Hk]; state, state_out
    [B, Hk, Dk, Dv]; lengths int32 [B] (tokens from there on are padding)."""
    if _here(workspace, stream) and _done(_native.linattn_fwd(
            q, k, v, log_decay, out, state, state_out, lengths, scale, workspace, _stream(stream))):
        return
    dt = _type_of(q, "q")
    H, Hk, Dk, Dv = _dims(q, k, v, 4)
    B, T = q.shape[:2]
    cq, ck, cv = _heads(q, "q", q, (B, T, H, Dk)), _heads(k, "k", q, (B, T, Hk, Dk)), _heads(v, "v", q, (B, T, Hk, Dv))
    co = _heads(out, "out", q, (B, T, H, Dv))
    _apart(out, "out")
    lg, ln = _flat(log_decay, "log_decay", q, (Hk,)), _flat(lengths, "lengths", q, (B,), True, torch.int32)
    s0, s1 = _flat(state, "state", q, (B, Hk, Dk, Dv), True), _flat(state_out, "state_out", q, (B, Hk, Dk, Dv), True)
    keep, ws, nws = _scratch(workspace, _lib.diffopt_linattn_workspace(B, T, H, Hk, Dk, Dv, dt, 0), q.device, stream)
    _check(_lib.diffopt_linattn_fwd(_ref(cq), _ref(ck), _ref(cv), lg, ln, s0, B, T, H, Hk, Dk, Dv, dt, float(scale), _ref(co), s1,
                                    ws, nws, _stream(stream)))


def linattn_bwd(dout, q, k, v, log_decay, dq, dk, dv, state=None, dstate_out=None, dstate=None, lengths=None, scale: float = 1.0,
                workspace=None, stream=None) -> None:
    """diffopt_linattn_bwd: gradients of linattn_fwd for the cotangents dout and dstate_out; any of dq, dk, dv, dstate may be
    None."""
    if _here(workspace, stream) and _done(_native.linattn_bwd(
            dout, q, k, v, log_decay, dq, dk, dv, state, dstate_out, dstate, lengths, scale, workspace, _stream(stream))):
        return
    dt = _type_of(q, "q")
    H, Hk, Dk, Dv = _dims(q, k, v, 4)
    B, T = q.shape[:2]
    cq, ck, cv = _heads(q, "q", q, (B, T, H, Dk)), _heads(k, "k", q, (B, T, Hk, Dk)), _heads(v, "v", q, (B, T, Hk, Dv))
    cdo = _heads(dout, "dout", q, (B, T, H, Dv))
    cdq, cdk, cdv = (_heads(x, w, q, s, True) for x, w, s in ((dq, "dq", (B, T, H, Dk)), (dk, "dk", (B, T, Hk, Dk)),
                                                              (dv, "dv", (B, T, Hk, Dv))))
    for x, w in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        if x is not None:
            _apart(x, w)
    lg, ln = _flat(log_decay, "log_decay", q, (Hk,)), _flat(lengths, "lengths", q, (B,), True, torch.int32)
    s0, ds1, ds0 = (_flat(x, w, q, (B, Hk, Dk, Dv), True) for x, w in ((state, "state"), (dstate_out, "dstate_out"),
                                                                       (dstate, "dstate")))
    keep, ws, nws = _scratch(workspace, _lib.diffopt_linattn_workspace(B, T, H, Hk, Dk, Dv, dt, 1), q.device, stream)
    _check(_lib.diffopt_linattn_bwd(_ref(cdo), ds1, _ref(cq), _ref(ck), _ref(cv), lg, ln, s0, B, T, H, Hk, Dk, Dv, dt, float(scale),
                                    _ref(cdq), _ref(cdk), _ref(cdv), ds0, ws, nws, _stream(stream)))


def linattn_step(q, k, v, log_decay, state, out, scale: float = 1.0, stream=None) -> None:
    """diffopt_linattn_step: one token per sequence, q [B, H, Dk], k [B, Hk, Dk], v [B, Hk, Dv] -> out [B, H, Dv]; state
    [B, Hk, Dk, Dv] is updated in place."""
    if _done(_native.linattn_step(q, k, v, log_decay, state, out, scale, _stream(stream))):
        return
    dt = _type_of(q, "q")
    H, Hk, Dk, Dv = _dims(q, k, v, 3)
    B = q.shape[0]
    ops = []
    for x, w, s in ((q, "q", (B, H, Dk)), (k, "k", (B, Hk, Dk)), (v, "v", (B, Hk, Dv)), (out, "out", (B, H, Dv))):
        _tensor(x, w, q.dtype, s, q.device)
        ops.append(_heads(x.unsqueeze(1), w, q, (s[0], 1, s[1], s[2])))
    _apart(out, "out")
    lg, st = _flat(log_decay, "log_decay", q, (Hk,)), _flat(state, "state", q, (B, Hk, Dk, Dv))
    _check(_lib.diffopt_linattn_step(_ref(ops[0]), _ref(ops[1]), _ref(ops[2]), lg, B, H, Hk, Dk, Dv, dt, float(scale), st,
                                     _ref(ops[3]), _stream(stream)))


# ---- norms of queries and keys, rotation ------------------------------------


def qknorm_rope_workspace(B: int, T: int, H: int, Hk: int, D: int) -> int:
    """diffopt_qknorm_rope_workspace: bytes that the backwards need where a weight's gradient is wanted."""
    n = int(_lib.diffopt_qknorm_rope_workspace(B, T, H, Hk, D))
    if n < 0:
        raise ValueError("qknorm_rope: sizes that the operator refuses")
    return n


def _qk_shape(q, k, q_weight, k_weight, cos, sin, positions, first, eps, interleaved):
    """(element type, shapes of q and k, the C arguments they share)."""
    dt = _type_of(q, "q")
    if q.dim() != 4:
        raise ValueError("q: expected a tensor of 4 axes")
    B, T, H, D = q.shape
    Hk = 0 if k is None else k.shape[-2] if isinstance(k, torch.Tensor) and k.dim() == 4 else -1
    if Hk < 0:
        raise ValueError("k: expected a tensor of 4 axes")
    rows = half = 0
    pc = ps = None
    if cos is not None:
        if not isinstance(cos, torch.Tensor) or cos.dim() != 2:
            raise ValueError("cos: expected a tensor of 2 axes")
        rows, half = cos.shape
        pc, ps = _flat(cos, "cos", q, (rows, half)), _flat(sin, "sin", q, (rows, half))
    pos, pbytes = None, 0
    if positions is not None:
        if not isinstance(positions, torch.Tensor) or positions.dtype not in (torch.int32, torch.int64):
            raise ValueError("positions: expected an int32 or int64 tensor")
        pos, pbytes = _flat(positions, "positions", q, (B, T), dtype=positions.dtype), positions.element_size()
    args = [_flat(q_weight, "q_weight", q, (D,), True), _flat(k_weight, "k_weight", q, (D,), True), pc, ps, rows, pos, pbytes,
            int(first), B, T, H, Hk, D, 2 * half, int(bool(interleaved)), dt, float(eps)]
    return (B, T, H, D), (B, T, Hk, D), args


def _qk_pair(xq, xk, what, q, sq, sk, optional=False, result=False):
    out = []
    for x, side, shape in ((xq, "q", sq), (xk, "k", sk)):
        name = what % side
        if shape[2] == 0 and side == "k":
            out.append(None)
            continue
        out.append(_heads(x, name, q, shape, optional))
        if result:
            _apart(x, name)
    return out


def qknorm_rope_fwd(q, k, q_weight, k_weight, cos, sin, q_out, k_out, positions=None, first: int = 0, eps: float = 1e-6,
                    interleaved: bool = False, stream=None) -> None:
    """diffopt_qknorm_rope_fwd: q [B, T, H, D] and k [B, T, Hk, D] (or None) normed for each head, scaled by the weights [D]
    (None: ones) and rotated by row positions[b, t] (None: first + t) of cos and sin [rows, rot/2] (None: no rotation)."""
    if _done(_native.qknorm_rope_fwd(q, k, q_weight, k_weight, cos, sin, q_out, k_out, positions, first, eps, bool(interleaved),
                                     _stream(stream))):
        return
    sq, sk, args = _qk_shape(q, k, q_weight, k_weight, cos, sin, positions, first, eps, interleaved)
    x = _qk_pair(q, k, "%s", q, sq, sk)
    y = _qk_pair(q_out, k_out, "%s_out", q, sq, sk, result=True)
    _check(_lib.diffopt_qknorm_rope_fwd(_ref(x[0]), _ref(x[1]), *args, _ref(y[0]), _ref(y[1]), _stream(stream)))


def qknorm_rope_bwd(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, dq, dk, dq_weight=None, dk_weight=None, positions=None,
                    first: int = 0, eps: float = 1e-6, interleaved: bool = False, workspace=None, stream=None) -> None:
    """diffopt_qknorm_rope_bwd: gradients of qknorm_rope_fwd; the weights' may be None."""
    if _here(workspace, stream) and _done(_native.qknorm_rope_bwd(
            dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, dq, dk, dq_weight, dk_weight, positions, first, eps,
            bool(interleaved), workspace, _stream(stream))):
        return
    sq, sk, args = _qk_shape(q, k, q_weight, k_weight, cos, sin, positions, first, eps, interleaved)
    x, dy = _qk_pair(q, k, "%s", q, sq, sk), _qk_pair(dq_out, dk_out, "d%s_out", q, sq, sk)
    dx = _qk_pair(dq, dk, "d%s", q, sq, sk, result=True)
    wq, wk = _flat(dq_weight, "dq_weight", q, sq[3:], True), _flat(dk_weight, "dk_weight", q, sq[3:], True)
    need = _lib.diffopt_qknorm_rope_workspace(*sq[:3], sk[2], sq[3]) if wq or wk else 0
    keep, ws, nws = _scratch(workspace, need, q.device, stream)
    _check(_lib.diffopt_qknorm_rope_bwd(_ref(dy[0]), _ref(dy[1]), _ref(x[0]), _ref(x[1]), *args, _ref(dx[0]), _ref(dx[1]), wq, wk, ws,
                                        nws, _stream(stream)))


def qknorm_rope_bwd_bwd(ddq, ddk, ddq_weight, ddk_weight, dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, out_dq_out, out_dk_out,
                        out_q, out_k, out_q_weight=None, out_k_weight=None, positions=None, first: int = 0, eps: float = 1e-6,
                        interleaved: bool = False, workspace=None, stream=None) -> None:
    """diffopt_qknorm_rope_bwd_bwd: gradients of qknorm_rope_bwd for cotangents of its results (None: zero)."""
    if _here(workspace, stream) and _done(_native.qknorm_rope_bwd_bwd(
            ddq, ddk, ddq_weight, ddk_weight, dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, out_dq_out, out_dk_out, out_q, out_k,
            out_q_weight, out_k_weight, positions, first, eps, bool(interleaved), workspace, _stream(stream))):
        return
    sq, sk, args = _qk_shape(q, k, q_weight, k_weight, cos, sin, positions, first, eps, interleaved)
    x, dy = _qk_pair(q, k, "%s", q, sq, sk), _qk_pair(dq_out, dk_out, "d%s_out", q, sq, sk)
    a = _qk_pair(ddq, ddk, "dd%s", q, sq, sk, optional=True)
    oy = _qk_pair(out_dq_out, out_dk_out, "out_d%s_out", q, sq, sk, result=True)
    ox = _qk_pair(out_q, out_k, "out_%s", q, sq, sk, result=True)
    b = [_flat(w, n, q, sq[3:], True) for w, n in ((ddq_weight, "ddq_weight"), (ddk_weight, "ddk_weight"))]
    wq, wk = _flat(out_q_weight, "out_q_weight", q, sq[3:], True), _flat(out_k_weight, "out_k_weight", q, sq[3:], True)
    need = _lib.diffopt_qknorm_rope_workspace(*sq[:3], sk[2], sq[3]) if wq or wk else 0
    keep, ws, nws = _scratch(workspace, need, q.device, stream)
    _check(_lib.diffopt_qknorm_rope_bwd_bwd(_ref(a[0]), _ref(a[1]), *b, _ref(dy[0]), _ref(dy[1]), _ref(x[0]), _ref(x[1]), *args,
                                            _ref(oy[0]), _ref(oy[1]), _ref(ox[0]), _ref(ox[1]), wq, wk, ws, nws, _stream(stream)))


# ---- distillation -----------------------------------------------------------


def distill_workspace(N: int, V: int, K: int, dtype=torch.float32) -> int:
    """diffopt_distill_workspace: bytes that distill_fwd, distill_fwd_bwd and distill_bwd_bwd need."""
    n = int(_lib.diffopt_distill_workspace(N, V, _DTYPES[dtype], K))
    if n < 0:
        raise ValueError("distill: sizes that the operator refuses")
    return n


def _rows(x, what, like, shape, result=False):
    _tensor(x, what, like.dtype, shape, like.device)
    if x.shape[1] > 1 and x.stride(1) != 1 and x.numel() > 0:
        raise ValueError("%s: the elements of a row must be contiguous" % what)
    if result:
        _apart(x, what)
    return x.data_ptr() or None, x.stride(0)


def _logits(logits, ids, teacher, temperature):
    dt = _type_of(logits, "logits")
    if logits.dim() != 2:
        raise ValueError("logits: expected a tensor of 2 axes")
    if not isinstance(ids, torch.Tensor) or ids.dtype not in (torch.int32, torch.int64) or ids.dim() != 2:
        raise ValueError("ids: expected an int32 or int64 tensor of 2 axes")
    N, V = logits.shape
    K = ids.shape[1]
    p, stride = _rows(logits, "logits", logits, (N, V))
    args = [p, stride, N, V, dt, _flat(ids, "ids", logits, (N, K), dtype=ids.dtype), ids.element_size(),
            _flat(teacher, "teacher", logits, (N, K)), K, float(temperature)]
    return N, V, K, dt, args


def distill_fwd(logits, ids, teacher, loss, stats, temperature: float = 1.0, workspace=None, stream=None) -> None:
    """diffopt_distill_fwd: loss [N] of logits [N, V] against the teacher's logits [N, K] at tokens ids [N, K]; stats [N, 2] is
    what the backwards take."""
    if _here(workspace, stream) and _done(_native.distill_fwd(
            logits, ids, teacher, loss, stats, temperature, workspace, _stream(stream))):
        return
    N, V, K, dt, args = _logits(logits, ids, teacher, temperature)
    pl, ps = _flat(loss, "loss", logits, (N,)), _flat(stats, "stats", logits, (N, 2))
    keep, ws, nws = _scratch(workspace, _lib.diffopt_distill_workspace(N, V, dt, K), logits.device, stream)
    _check(_lib.diffopt_distill_fwd(*args, pl, ps, ws, nws, _stream(stream)))


def distill_bwd(dloss, logits, ids, teacher, stats, dlogits, dteacher=None, temperature: float = 1.0, stream=None) -> None:
    """diffopt_distill_bwd: gradients of distill_fwd for the cotangent dloss [N]; dlogits may be logits."""
    if _done(_native.distill_bwd(dloss, logits, ids, teacher, stats, dlogits, dteacher, temperature, _stream(stream))):
        return
    N, V, K, dt, args = _logits(logits, ids, teacher, temperature)
    pg, ps = _flat(dloss, "dloss", logits, (N,)), _flat(stats, "stats", logits, (N, 2))
    pd, dstride = _rows(dlogits, "dlogits", logits, (N, V), True)
    _check(_lib.diffopt_distill_bwd(pg, *args, ps, pd, dstride, _flat(dteacher, "dteacher", logits, (N, K), True), _stream(stream)))


def distill_fwd_bwd(dloss, logits, ids, teacher, loss, stats, dlogits, dteacher=None, temperature: float = 1.0, workspace=None,
                    stream=None) -> None:
    """diffopt_distill_fwd_bwd: the loss and its gradients for a dloss known beforehand, the logits read once."""
    if _here(workspace, stream) and _done(_native.distill_fwd_bwd(
            dloss, logits, ids, teacher, loss, stats, dlogits, dteacher, temperature, workspace, _stream(stream))):
        return
    N, V, K, dt, args = _logits(logits, ids, teacher, temperature)
    pg, pl, ps = _flat(dloss, "dloss", logits, (N,)), _flat(loss, "loss", logits, (N,)), _flat(stats, "stats", logits, (N, 2))
    pd, dstride = _rows(dlogits, "dlogits", logits, (N, V), True)
    keep, ws, nws = _scratch(workspace, _lib.diffopt_distill_workspace(N, V, dt, K), logits.device, stream)
    _check(_lib.diffopt_distill_fwd_bwd(pg, *args, pl, ps, pd, dstride, _flat(dteacher, "dteacher", logits, (N, K), True), ws, nws,
                                        _stream(stream)))


def distill_bwd_bwd(ddlogits, ddteacher, dloss, logits, ids, teacher, stats, out_dloss, out_logits, out_teacher,
                    temperature: float = 1.0, workspace=None, stream=None) -> None:
    """diffopt_distill_bwd_bwd: gradients of distill_bwd for cotangents of dlogits and dteacher (None: zero); out_dloss and
    out_teacher may be None."""
    if _here(workspace, stream) and _done(_native.distill_bwd_bwd(
            ddlogits, ddteacher, dloss, logits, ids, teacher, stats, out_dloss, out_logits, out_teacher, temperature, workspace,
            _stream(stream))):
        return
    N, V, K, dt, args = _logits(logits, ids, teacher, temperature)
    pa, astride = (None, 0) if ddlogits is None else _rows(ddlogits, "ddlogits", logits, (N, V))
    po, ostride = _rows(out_logits, "out_logits", logits, (N, V), True)
    pg, ps = _flat(dloss, "dloss", logits, (N,)), _flat(stats, "stats", logits, (N, 2))
    keep, ws, nws = _scratch(workspace, _lib.diffopt_distill_workspace(N, V, dt, K), logits.device, stream)
    _check(_lib.diffopt_distill_bwd_bwd(pa, astride, _flat(ddteacher, "ddteacher", logits, (N, K), True), pg, *args, ps,
                                        _flat(out_dloss, "out_dloss", logits, (N,), True), po, ostride,
                                        _flat(out_teacher, "out_teacher", logits, (N, K), True), ws, nws, _stream(stream)))
