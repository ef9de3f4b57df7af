"""ctypes binding of the sequence operators (the C ABI of include/evconv_ops.h, in libevconv.so).

Argument marshalling only: PyTorch owns the memory and names the stream (the current one of the
tensors' device); every value is computed by the library's kernels.  A refused call raises
`EvConvError` with the library's status, as the net's calls do.

    o, state = delta_rule(q, k, v, gate, beta, state)            the gated delta rule
    r = block_norm(x, branch, z, ...)                            norms around a block: r.x, r.h, r.q
    y = quant_matmul(quantize_rows(x), quantize_rows(weight))    product in 8-bit integers
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from .evconv import (ERR_INVALID_ARG, ERR_SHAPE, OK, EvConvError, lib)

ABI_VERSION = 1
EXPORTS = ["evconv_delta_rule_workspace", "evconv_delta_rule", "evconv_block_norm", "evconv_quant_matmul_workspace",
           "evconv_quant_matmul"]
DELTA_NORMALIZE, DELTA_RAW_GATES = 1, 2
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}
_NORMS = {"rms": 0, "layer": 1}
_GATES = {"none": 0, "sigmoid": 1, "silu": 2}
_ACTS = {"none": 0, "relu": 1, "sigmoid": 2, "tanh": 3}
_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class Heads(ctypes.Structure):
    _fields_ = [("data", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class DeltaArgs(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("dtype", _i32), ("gate_dtype", _i32), ("flags", ctypes.c_uint32),
                ("heads_k", _i32), ("heads_v", _i32), ("d_k", _i32), ("d_v", _i32), ("n_seq", _i32), ("n_slots", _i32),
                ("n_tokens", _i64), ("scale", _f32),
                ("q", Heads), ("k", Heads), ("v", Heads), ("gate", Heads), ("beta", Heads),
                ("o", _vp), ("o_token_stride", _i64), ("o_head_stride", _i64), ("a_scale", _vp), ("dt_bias", _vp),
                ("seq_offsets", _vp), ("slots", _vp), ("state_in", _vp), ("state_out", _vp)]


class NormArgs(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("dtype", _i32), ("norm", _i32), ("gate_act", _i32), ("pre_norm", _i32),
                ("dim", _i32), ("group", _i32), ("eps", _f32), ("rows", _i64), ("x", _vp), ("branch", _vp), ("gate", _vp),
                ("x_stride", _i64), ("branch_stride", _i64), ("gate_stride", _i64),
                ("post_weight", _vp), ("post_bias", _vp), ("res_scale", _vp), ("pre_weight", _vp), ("pre_bias", _vp),
                ("x_out", _vp), ("h_out", _vp), ("x_out_stride", _i64), ("h_out_stride", _i64),
                ("q", _vp), ("q_stride", _i64), ("q_scale", _vp)]


class QuantArgs(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("dtype", _i32), ("act", _i32), ("n", _i32), ("k", _i32), ("m", _i64),
                ("a", _vp), ("b", _vp), ("a_stride", _i64), ("b_stride", _i64), ("a_scale", _vp), ("b_scale", _vp),
                ("bias", _vp), ("y", _vp), ("y_stride", _i64)]


class QuantRows(NamedTuple):
    """Rows of 8-bit integers: row i stands for scale[i] * q[i, :k].  q: int8 [rows, stride] with zeros from
    column k on, stride a multiple of 128; scale: fp32 [rows]."""
    q: torch.Tensor
    scale: torch.Tensor
    k: int


class NormResult(NamedTuple):
    x: Optional[torch.Tensor]
    h: Optional[torch.Tensor]
    q: Optional[QuantRows]


_entry = None


def _calls():
    global _entry
    if _entry is None:
        L = lib()
        size = ctypes.POINTER(ctypes.c_size_t)
        L.evconv_delta_rule_workspace.argtypes = [ctypes.POINTER(DeltaArgs), size]
        L.evconv_delta_rule.argtypes = [ctypes.POINTER(DeltaArgs), _vp, ctypes.c_size_t, _vp]
        L.evconv_block_norm.argtypes = [ctypes.POINTER(NormArgs), _vp]
        L.evconv_quant_matmul_workspace.argtypes = [ctypes.POINTER(QuantArgs), size]
        L.evconv_quant_matmul.argtypes = [ctypes.POINTER(QuantArgs), _vp, ctypes.c_size_t, _vp]
        _entry = L
    return _entry


def _check(status):
    if status != OK:
        raise EvConvError(status, lib().evconv_last_error(None).decode())


def _refuse(status, text):
    raise EvConvError(status, text)


def _tensor(t, name, device, dtype, shape):
    """A tensor of this device, type and shape with contiguous rows; None passes."""
    if t is None:
        return
    if t.device != device or device.type != "cuda":
        _refuse(ERR_INVALID_ARG, f"{name} is on {t.device}, expected one GPU ({device})")
    if t.dtype != dtype:
        _refuse(ERR_INVALID_ARG, f"{name} is {t.dtype}, expected {dtype}")
    if t.shape != shape:
        _refuse(ERR_SHAPE, f"{name} is {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse(ERR_SHAPE, f"{name}: the last dimension must be contiguous")


def _packed(t, name, device, dtype, shape):
    _tensor(t, name, device, dtype, shape)
    if t is not None and not t.is_contiguous():
        _refuse(ERR_SHAPE, f"{name} must be contiguous")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dtype(t, name):
    if t.dtype not in _DTYPES:
        _refuse(ERR_INVALID_ARG, f"{name} is {t.dtype}, expected float32 or bfloat16")
    return _DTYPES[t.dtype]


def _enqueue(call, args, device, workspace_of=None):
    """The call on the device's current stream, with a workspace of its own from the caching allocator
    (which keeps it for this stream until the call's kernels are done)."""
    with torch.cuda.device(device):
        stream = torch.cuda.current_stream().cuda_stream
        if workspace_of is None:
            _check(call(ctypes.byref(args), stream))
            return
        n = ctypes.c_size_t(0)
        _check(workspace_of(ctypes.byref(args), ctypes.byref(n)))
        ws = torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None
        _check(call(ctypes.byref(args), _ptr(ws), n.value, stream))


def _set_heads(to, t):
    to.data, to.token_stride, to.head_stride = t.data_ptr(), t.stride(0), t.stride(1)


def delta_rule(q, k, v, gate, beta, state=None, *, state_out=None, out=None, seq_offsets=None, slots=None, n_seq=None,
               scale=None, normalize=False, a_scale=None, dt_bias=None):
    """The gated delta rule (evconv_delta_rule): (o, states after the last tokens).

    q, k: [tokens, heads_k, d_k]; v: [tokens, heads_v, d_v]; gate, beta: [tokens, heads_v], log decays and
    strengths, or with a_scale and dt_bias ([heads_v] fp32) what a projection gave for them.  The last dimension is
    contiguous, the others may be strided (slices of one projection).  state: fp32 [slots, heads_v, d_k, d_v], None:
    zeros.  Sequences: seq_offsets (int32 [n_seq + 1]), or n_seq of equal length (by default as many as `slots`,
    else as states, else one).  slots: int32 [n_seq], which state a sequence continues, negative: none.
    state_out: where the states go, may be `state`; by default a new tensor, with `slots` `state` itself.  scale: of o,
    by default d_k ** -0.5.  normalize: q and k are divided by their norms first."""
    if q.dim() != 3 or v.dim() != 3 or gate.dim() != 2:
        _refuse(ERR_SHAPE, f"q {tuple(q.shape)}, v {tuple(v.shape)}, gate {tuple(gate.shape)}: expected three, three and two dimensions")
    device, (n, hk, dk), (hv, dv) = v.device, q.shape, v.shape[1:]
    a = DeltaArgs(abi_version=ABI_VERSION, dtype=_dtype(v, "v"), gate_dtype=_dtype(gate, "gate"),
                  flags=(DELTA_NORMALIZE if normalize else 0) | (DELTA_RAW_GATES if a_scale is not None or dt_bias is not None else 0),
                  heads_k=hk, heads_v=hv, d_k=dk, d_v=dv, n_tokens=n, scale=dk ** -0.5 if scale is None else scale)
    for t, name, dtype, shape in ((q, "q", v.dtype, q.shape), (k, "k", v.dtype, q.shape), (v, "v", v.dtype, (n, hv, dv)),
                                  (gate, "gate", gate.dtype, (n, hv)), (beta, "beta", gate.dtype, (n, hv)), (out, "out", v.dtype, v.shape)):
        if name in ("gate", "beta"):  # (single values: any strides)
            if t.device != device or t.dtype != dtype or t.shape != shape:
                _refuse(ERR_SHAPE, f"{name} is {tuple(t.shape)} {t.dtype} on {t.device}, expected {shape} {dtype} on {device}")
        else:
            _tensor(t, name, device, dtype, shape)
    _packed(a_scale, "a_scale", device, torch.float32, (hv,))
    _packed(dt_bias, "dt_bias", device, torch.float32, (hv,))
    if seq_offsets is not None:
        n_seq = seq_offsets.numel() - 1
        _packed(seq_offsets, "seq_offsets", device, torch.int32, (n_seq + 1,))
    elif n_seq is None:
        n_seq = slots.numel() if slots is not None else state.shape[0] if state is not None else 1
    _packed(slots, "slots", device, torch.int32, (n_seq,))
    some = state if state is not None else state_out
    n_slots = some.shape[0] if some is not None and some.dim() else n_seq
    for t, name in ((state, "state"), (state_out, "state_out")):
        _packed(t, name, device, torch.float32, (n_slots, hv, dk, dv))
    if state_out is None:
        state_out = state if state is not None and slots is not None else \
            torch.empty(n_slots, hv, dk, dv, dtype=torch.float32, device=device)
    if out is None:
        out = torch.empty(n, hv, dv, dtype=v.dtype, device=device)
    a.n_seq, a.n_slots = n_seq, n_slots
    for to, t in ((a.q, q), (a.k, k), (a.v, v), (a.gate, gate), (a.beta, beta)):
        _set_heads(to, t)
    a.o, a.o_token_stride, a.o_head_stride = out.data_ptr(), out.stride(0), out.stride(1)
    a.a_scale, a.dt_bias, a.seq_offsets, a.slots = _ptr(a_scale), _ptr(dt_bias), _ptr(seq_offsets), _ptr(slots)
    a.state_in, a.state_out = _ptr(state), state_out.data_ptr()
    L = _calls()
    _enqueue(L.evconv_delta_rule, a, device, L.evconv_delta_rule_workspace)
    return out, state_out


def _quant_rows(rows, dim, device):
    stride = -(-dim // 128) * 128
    return QuantRows(torch.empty(rows, stride, dtype=torch.int8, device=device),
                     torch.empty(rows, dtype=torch.float32, device=device), dim)


def block_norm(x=None, branch=None, gate=None, *, post_weight=None, post_bias=None, gate_act=None, group=None, res_scale=None,
               pre_norm=None, pre_weight=None, pre_bias=None, kind="rms", eps=1e-6, want=None, x_out=None, h_out=None):
    """The norms around a block (evconv_block_norm), per row of the last dimension: with
    t = norm(branch) * post_weight + post_bias (in groups of `group` values), times act(gate),
    x' = x + res_scale * t;  h = norm(x') * pre_weight + pre_bias (pre_norm; by default if pre_weight is given).

    x, branch, gate: [rows, dim] with contiguous rows; gate_act: "none", "sigmoid" or "silu" (default: "silu" if there is a
    gate).  want: which outputs, letters of "xhq": x', h, and h as rows of 8-bit integers; by default "xh" (without
    pre_norm "x").  Returns NormResult(x, h, q), None for what is not wanted.  x_out may be x."""
    rows_of = x if x is not None else branch
    if rows_of is None or rows_of.dim() != 2:
        _refuse(ERR_SHAPE, "block norm: x or branch as [rows, dim]")
    device, dtype, (rows, dim) = rows_of.device, rows_of.dtype, rows_of.shape
    group = dim if group is None else group
    if pre_norm is None:
        pre_norm = pre_weight is not None or pre_bias is not None
    gate_act = ("none" if gate is None else "silu") if gate_act is None else gate_act
    if want is None:
        want = "xh" if pre_norm else "x"
    if kind not in _NORMS or gate_act not in _GATES or not want or set(want) - set("xhq"):
        _refuse(ERR_INVALID_ARG, f"block norm: kind {kind!r}, gate_act {gate_act!r}, want {want!r}")
    for t, name in ((x, "x"), (branch, "branch"), (gate, "gate"), (x_out, "x_out"), (h_out, "h_out")):
        _tensor(t, name, device, dtype, (rows, dim))
    for t, name, size in ((post_weight, "post_weight", group), (post_bias, "post_bias", group), (res_scale, "res_scale", dim),
                          (pre_weight, "pre_weight", dim), (pre_bias, "pre_bias", dim)):
        _packed(t, name, device, torch.float32, (size,))
    if "x" in want and x_out is None:
        x_out = torch.empty(rows, dim, dtype=dtype, device=device)
    if "h" in want and h_out is None:
        h_out = torch.empty(rows, dim, dtype=dtype, device=device)
    q = _quant_rows(rows, dim, device) if "q" in want else None
    a = NormArgs(abi_version=ABI_VERSION, dtype=_dtype(rows_of, "x"), norm=_NORMS[kind], gate_act=_GATES[gate_act],
                 pre_norm=1 if pre_norm else 0, dim=dim, group=group, eps=eps, rows=rows, x=_ptr(x), branch=_ptr(branch), gate=_ptr(gate),
                 post_weight=_ptr(post_weight), post_bias=_ptr(post_bias), res_scale=_ptr(res_scale),
                 pre_weight=_ptr(pre_weight), pre_bias=_ptr(pre_bias))
    for name, t in (("x", x), ("branch", branch), ("gate", gate)):
        if t is not None:
            setattr(a, name + "_stride", t.stride(0))
    if "x" in want:
        a.x_out, a.x_out_stride = x_out.data_ptr(), x_out.stride(0)
    if "h" in want:
        a.h_out, a.h_out_stride = h_out.data_ptr(), h_out.stride(0)
    if q is not None:
        a.q, a.q_stride, a.q_scale = q.q.data_ptr(), q.q.stride(0), q.scale.data_ptr()
    _enqueue(_calls().evconv_block_norm, a, device)
    return NormResult(x_out if "x" in want else None, h_out if "h" in want else None, q)


def quantize_rows(x) -> QuantRows:
    """Rows [rows, k] as 8-bit integers with a scale each (tokens of activations, output channels of a weight)."""
    return block_norm(x, want="q").q


def quant_matmul(a: QuantRows, b: QuantRows, *, bias=None, act="none", out_dtype=torch.float32, out=None):
    """act(a b' + bias) of rows of 8-bit integers (evconv_quant_matmul): [rows of a, rows of b].  act: "none",
    "relu", "sigmoid" or "tanh"."""
    (m, sa), (n, sb), device = a.q.shape, b.q.shape, a.q.device
    if a.k != b.k:
        _refuse(ERR_SHAPE, f"quantised product: rows of {a.k} and {b.k} values")
    if act not in _ACTS:
        _refuse(ERR_INVALID_ARG, f"quantised product: act {act!r}")
    for r, name, rows in ((a, "a", m), (b, "b", n)):
        _tensor(r.q, name + ".q", device, torch.int8, r.q.shape)
        _packed(r.scale, name + ".scale", device, torch.float32, (rows,))
    _packed(bias, "bias", device, torch.float32, (n,))
    if out is None:
        out = torch.empty(m, n, dtype=out_dtype, device=device)
    _tensor(out, "out", device, out.dtype, (m, n))
    args = QuantArgs(abi_version=ABI_VERSION, dtype=_dtype(out, "out"), act=_ACTS[act], n=n, k=a.k, m=m, a=a.q.data_ptr(), b=b.q.data_ptr(),
                     a_stride=a.q.stride(0), b_stride=b.q.stride(0), a_scale=a.scale.data_ptr(), b_scale=b.scale.data_ptr(),
                     bias=_ptr(bias), y=out.data_ptr(), y_stride=out.stride(0))
    L = _calls()
    _enqueue(L.evconv_quant_matmul, args, device, L.evconv_quant_matmul_workspace)
    return out
