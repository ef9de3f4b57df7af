"""ctypes binding of the sequence operators (the C ABI of include/evconv_ops.h, in libevconv.so).

Argument marshalling only: PyTorch owns the memory and names the stream (the current one of the
tensors' device); every value is computed by the library's kernels.  A refused call raises
`EvConvError` with the library's status, as the net's calls do.  No operator has a gradient: a tensor that
wants one is refused where gradients are recorded.

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
EXPORTS = ["evconv_delta_rule_workspace", "evconv_delta_rule", "evconv_block_norm", "evconv_quant_matmul"]
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


class _FlatDeltaArgs(ctypes.Structure):
    """DeltaArgs with the fields of its Heads in their place: filled in by position, without five more structures a call."""
    _fields_ = [(name + part, kind) for name, of in DeltaArgs._fields_
                for part, kind in ([("_" + p, t) for p, t in Heads._fields_] if of is Heads else [("", of)])]


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
_byref, _empty, _empty_like, _grad_enabled = ctypes.byref, torch.empty, torch.empty_like, torch.is_grad_enabled
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)  # (without the wrapper's own checks)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda gpu: torch.cuda.current_stream(gpu).cuda_stream)


def _calls():
    global _entry
    if _entry is None:
        L = lib()
        L.evconv_delta_rule_workspace.argtypes = [_vp, _vp]  # (byref() of the structures above)
        L.evconv_delta_rule.argtypes = [_vp, _vp, ctypes.c_size_t, _vp]
        L.evconv_block_norm.argtypes = [_vp, _vp]
        L.evconv_quant_matmul.argtypes = [_vp, _vp]
        _entry = L
    return _entry


def _check(status):
    if status != OK:
        raise EvConvError(status, lib().evconv_last_error(None).decode())


def _refuse(status, text):
    raise EvConvError(status, text)


# The checks run before every launch, and a launch of few tokens takes a few microseconds: one comparison of each
# property, the reasons only once one has failed.

def _explain(t, name, gpu, dtype, shape):
    if gpu < 0 or t.get_device() != gpu:
        _refuse(ERR_INVALID_ARG, f"{name} is on {t.device}, expected " + (f"cuda:{gpu}" if gpu >= 0 else "a GPU"))
    if t.dtype != dtype:
        _refuse(ERR_INVALID_ARG, f"{name} is {t.dtype}, expected {dtype}")
    if t.shape != shape:
        _refuse(ERR_SHAPE, f"{name} is {tuple(t.shape)}, expected {tuple(shape)}")
    if t.requires_grad and _grad_enabled():
        _refuse(ERR_INVALID_ARG, f"{name} wants a gradient, which these operators do not have: call them under torch.no_grad()")
    _refuse(ERR_SHAPE, f"{name}: strides {t.stride()}: rows (parameters and states: the whole tensor) must be contiguous")


def _rows(t, name, gpu, dtype, shape):
    """(address, strides) of a tensor of this GPU, type and shape whose last dimension is contiguous."""
    stride = t.stride()
    if t.get_device() != gpu or t.dtype is not dtype or t.shape != shape or (stride[-1] != 1 and shape[-1] > 1) \
            or (t.requires_grad and _grad_enabled()):
        _explain(t, name, gpu, dtype, shape)
    return t.data_ptr(), stride


def _packed(t, name, gpu, dtype, shape):
    """Address of a contiguous tensor; None of None."""
    if t is None:
        return None
    if t.get_device() != gpu or t.dtype is not dtype or t.shape != shape or not t.is_contiguous() \
            or (t.requires_grad and _grad_enabled()):
        _explain(t, name, gpu, dtype, shape)
    return t.data_ptr()


def _like(t, shape, dtype, gpu):
    """A new contiguous tensor of this shape and type, those of `t` unless that is None.  (Making one like another takes less
    time than making one from its shape.)"""
    if t is not None and t.is_contiguous():
        return _empty_like(t)
    return _empty(*shape, dtype=dtype, device=gpu)


def _dtype(t, name):
    code = _DTYPES.get(t.dtype)
    if code is None:
        _refuse(ERR_INVALID_ARG, f"{name} is {t.dtype}, expected float32 or bfloat16")
    return code


def _enqueue(call, args, gpu, workspace_of=None):
    """The call on the GPU's current stream, with a workspace of its own from the caching allocator (which
    keeps it for this stream until the call's kernels are done)."""
    if _current_device() != gpu:
        with torch.cuda.device(gpu):
            return _enqueue(call, args, gpu, workspace_of)
    stream, args = _current_stream(gpu), _byref(args)
    if workspace_of is None:
        status = call(args, stream)
    else:
        n = ctypes.c_size_t(0)
        _check(workspace_of(args, _byref(n)))
        if n.value:
            ws = torch.empty(n.value, dtype=torch.uint8, device=gpu)
            status = call(args, ws.data_ptr(), n.value, stream)
        else:
            status = call(args, None, 0, stream)
    if status != OK:
        _check(status)


def delta_rule(q, k, v, gate, beta, state=None, *, state_out=None, out=None, seq_offsets=None, slots=None, n_seq=None,
               scale=None, normalize=False, a_scale=None, dt_bias=None):
    """The gated delta rule (evconv_delta_rule): (o, states after the last tokens).

    q, k: [tokens, heads_k, d_k]; v: [tokens, heads_v, d_v]; gate, beta: [tokens, heads_v], log decays and
    strengths, or with a_scale and dt_bias ([heads_v] fp32) what a projection gave for them.  The last dimension is
    contiguous, the others may be strided (slices of one projection).  state: fp32 [slots, heads_v, d_k, d_v], None:
    zeros.  Sequences: seq_offsets (int32 [n_seq + 1]), or n_seq of equal length (by default as many as `slots`,
    else as states, else one).  slots: int32 [n_seq], which state a sequence continues, negative: none.
    state_out: where the states go, may be `state`; by default a new tensor (states of no sequence as in `state`), with
    `slots` `state` itself.  Slots need one of the two.  scale: of o, by default d_k ** -0.5.  normalize: q and k are divided by their norms first."""
    if q.dim() != 3 or v.dim() != 3 or gate.dim() != 2:
        _refuse(ERR_SHAPE, f"q {tuple(q.shape)}, v {tuple(v.shape)}, gate {tuple(gate.shape)}: expected three, three and two dimensions")
    gpu, dtype, gate_dtype, q_shape, v_shape = v.get_device(), v.dtype, gate.dtype, q.shape, v.shape
    (n, hk, dk), (hv, dv) = q_shape, v_shape[1:]
    if gpu < 0 or v_shape[0] != n:
        _explain(v, "v", gpu, dtype, (n, hv, dv))
    raw = a_scale is not None or dt_bias is not None
    flags, f32 = (DELTA_NORMALIZE if normalize else 0) | (DELTA_RAW_GATES if raw else 0), torch.float32
    q_at, (q_token, q_head, _) = _rows(q, "q", gpu, dtype, q_shape)
    k_at, (k_token, k_head, _) = _rows(k, "k", gpu, dtype, q_shape)
    v_at, (v_token, v_head, _) = _rows(v, "v", gpu, dtype, v_shape)
    gates = (n, hv)
    if gate.get_device() != gpu or gate.shape != gates or (gate.requires_grad and _grad_enabled()):  # (single values: any strides)
        _explain(gate, "gate", gpu, gate_dtype, gates)
    if beta.get_device() != gpu or beta.dtype is not gate_dtype or beta.shape != gates or (beta.requires_grad and _grad_enabled()):
        _explain(beta, "beta", gpu, gate_dtype, gates)
    if raw:
        a_scale, dt_bias = _packed(a_scale, "a_scale", gpu, f32, (hv,)), _packed(dt_bias, "dt_bias", gpu, f32, (hv,))
    if seq_offsets is not None:
        if n_seq is not None and n_seq != seq_offsets.numel() - 1:
            _refuse(ERR_SHAPE, f"{seq_offsets.numel()} offsets for {n_seq} sequences")
        n_seq = seq_offsets.numel() - 1
        seq_offsets = _packed(seq_offsets, "seq_offsets", gpu, torch.int32, (n_seq + 1,))
    elif n_seq is None:
        n_seq = slots.numel() if slots is not None else state.shape[0] if state is not None and state.dim() else 1
    slots_at = _packed(slots, "slots", gpu, torch.int32, (n_seq,))
    some = state if state is not None else state_out
    if some is None and slots is not None:
        _refuse(ERR_INVALID_ARG, "slots without state and state_out: of how many states?")
    n_slots = some.shape[0] if some is not None and some.dim() else n_seq
    shape = (n_slots, hv, dk, dv)
    state_at = _packed(state, "state", gpu, f32, shape)
    if state_out is None:
        if slots is not None:
            state_out = state
        else:  # (the call writes the sequences' states; where there are more, the others are as they were)
            state_out = state.clone() if n_slots > n_seq else _like(state, shape, f32, gpu)
        to_at = state_out.data_ptr()
    else:
        to_at = state_at if state_out is state else _packed(state_out, "state_out", gpu, f32, shape)
    if out is None:
        out = _like(v, v_shape, dtype, gpu)
        o_at, (o_token, o_head, _) = out.data_ptr(), out.stride()
    else:
        o_at, (o_token, o_head, _) = _rows(out, "out", gpu, dtype, v_shape)
    a = _FlatDeltaArgs(ABI_VERSION, _dtype(v, "v"), _dtype(gate, "gate"), flags, hk, hv, dk, dv, n_seq, n_slots, n,
                  dk ** -0.5 if scale is None else scale, q_at, q_token, q_head, k_at, k_token, k_head, v_at, v_token, v_head,
                  gate.data_ptr(), *gate.stride(), beta.data_ptr(), *beta.stride(), o_at, o_token, o_head, a_scale, dt_bias,
                  seq_offsets, slots_at, state_at, to_at)  # (in the order of _fields_)
    L = _calls()
    _enqueue(L.evconv_delta_rule, a, gpu, L.evconv_delta_rule_workspace)
    return out, state_out


def block_norm(x=None, branch=None, gate=None, *, post_weight=None, post_bias=None, gate_act=None, group=None, res_scale=None,
               pre_norm=None, pre_weight=None, pre_bias=None, kind="rms", eps=1e-6, want=None, x_out=None, h_out=None):
    """The norms around a block (evconv_block_norm), per row of the last dimension: with
    t = norm(branch) * post_weight + post_bias (in groups of `group` values), times act(gate),
    x' = x + res_scale * t;  h = norm(x') * pre_weight + pre_bias (pre_norm; by default if pre_weight is given).

    x, branch, gate: [rows, dim] with contiguous rows; gate_act: "none", "sigmoid" or "silu" (default: "silu" if there is a
    gate).  want: which outputs, letters of "xhq": x', h, and h as rows of 8-bit integers; by default "xh" (without
    pre_norm "x").  Returns NormResult(x, h, q), None for what is not wanted.  x_out may be x."""
    first = x if x is not None else branch
    if first is None or first.dim() != 2:
        _refuse(ERR_SHAPE, "block norm: x or branch as [rows, dim]")
    gpu, dtype, shape = first.get_device(), first.dtype, first.shape
    if gpu < 0:
        _explain(first, "x" if x is not None else "branch", gpu, dtype, shape)
    rows, dim = shape
    if group is None:
        group = dim
    if pre_norm is None:
        pre_norm = pre_weight is not None or pre_bias is not None
    if gate_act is None:
        gate_act = "none" if gate is None else "silu"
    if want is None:
        want = "xh" if pre_norm else "x"
    if kind not in _NORMS or gate_act not in _GATES or not want or want.strip("xhq"):
        _refuse(ERR_INVALID_ARG, f"block norm: kind {kind!r}, gate_act {gate_act!r}, want {want!r}")
    f32 = torch.float32
    x_at = branch_at = gate_at = x_to = h_to = q_to = scale_to = None
    x_step = branch_step = gate_step = x_to_step = h_to_step = q_step = 0
    if x is not None:
        x_at, (x_step, _) = _rows(x, "x", gpu, dtype, shape)
    if branch is not None:
        branch_at, (branch_step, _) = _rows(branch, "branch", gpu, dtype, shape)
    if gate is not None:
        gate_at, (gate_step, _) = _rows(gate, "gate", gpu, dtype, shape)
    if post_weight is not None:
        post_weight = _packed(post_weight, "post_weight", gpu, f32, (group,))
    if post_bias is not None:
        post_bias = _packed(post_bias, "post_bias", gpu, f32, (group,))
    if res_scale is not None:
        res_scale = _packed(res_scale, "res_scale", gpu, f32, (dim,))
    if pre_weight is not None:
        pre_weight = _packed(pre_weight, "pre_weight", gpu, f32, (dim,))
    if pre_bias is not None:
        pre_bias = _packed(pre_bias, "pre_bias", gpu, f32, (dim,))
    if "x" not in want:
        x_out = None
    elif x_out is None:
        x_out = _like(first, shape, dtype, gpu)
        x_to, x_to_step = x_out.data_ptr(), dim
    else:
        x_to, (x_to_step, _) = _rows(x_out, "x_out", gpu, dtype, shape)
    if "h" not in want:
        h_out = None
    elif h_out is None:
        h_out = _like(first, shape, dtype, gpu)
        h_to, h_to_step = h_out.data_ptr(), dim
    else:
        h_to, (h_to_step, _) = _rows(h_out, "h_out", gpu, dtype, shape)
    q = None
    if "q" in want:
        q_step = -(-dim // 128) * 128
        q = QuantRows(_empty(rows, q_step, dtype=torch.int8, device=gpu), _empty(rows, dtype=f32, device=gpu), dim)
        q_to, scale_to = q.q.data_ptr(), q.scale.data_ptr()
    a = NormArgs(ABI_VERSION, _dtype(first, "x"), _NORMS[kind], _GATES[gate_act], 1 if pre_norm else 0, dim, group, eps, rows,
                 x_at, branch_at, gate_at, x_step, branch_step, gate_step, post_weight, post_bias, res_scale, pre_weight, pre_bias,
                 x_to, h_to, x_to_step, h_to_step, q_to, q_step, scale_to)  # (in the order of _fields_)
    _enqueue(_calls().evconv_block_norm, a, gpu)
    return NormResult(x_out, h_out, q)


def quantize_rows(x) -> QuantRows:
    """Rows [rows, k] as 8-bit integers with a scale each (tokens of activations, output channels of a weight): block_norm's
    "q" of x alone."""
    if x.dim() != 2:
        _refuse(ERR_SHAPE, "block norm: x or branch as [rows, dim]")
    gpu, dtype, shape = x.get_device(), x.dtype, x.shape
    if gpu < 0:
        _explain(x, "x", gpu, dtype, shape)
    rows, dim = shape
    at, (step, _) = _rows(x, "x", gpu, dtype, shape)
    q_step = -(-dim // 128) * 128
    q, scale = _empty(rows, q_step, dtype=torch.int8, device=gpu), _empty(rows, dtype=torch.float32, device=gpu)
    a = NormArgs(ABI_VERSION, _dtype(x, "x"), 0, 0, 0, dim, dim, 0.0, rows, at, None, None, step, 0, 0, None, None, None, None, None,
                 None, None, 0, 0, q.data_ptr(), q_step, scale.data_ptr())
    _enqueue(_calls().evconv_block_norm, a, gpu)
    return QuantRows(q, scale, dim)


def quant_matmul(a: QuantRows, b: QuantRows, *, bias=None, act="none", out_dtype=torch.float32, out=None):
    """act(a b' + bias) of rows of 8-bit integers (evconv_quant_matmul): [rows of a, rows of b].  act: "none",
    "relu", "sigmoid" or "tanh"."""
    aq, a_scale, k = a
    bq, b_scale, bk = b
    if aq.dim() != 2 or bq.dim() != 2 or k != bk:
        _refuse(ERR_SHAPE, f"quantised product: rows {tuple(aq.shape)} of {k} and {tuple(bq.shape)} of {bk} values")
    if act not in _ACTS:
        _refuse(ERR_INVALID_ARG, f"quantised product: act {act!r}")
    gpu, m, n, f32 = aq.get_device(), aq.shape[0], bq.shape[0], torch.float32
    if gpu < 0:
        _explain(aq, "a.q", gpu, torch.int8, aq.shape)
    a_at, (a_step, _) = _rows(aq, "a.q", gpu, torch.int8, aq.shape)
    b_at, (b_step, _) = _rows(bq, "b.q", gpu, torch.int8, bq.shape)
    if aq.shape[1] < -(-k // 128) * 128 or bq.shape[1] < -(-k // 128) * 128:
        _refuse(ERR_SHAPE, f"quantised product: rows of {aq.shape[1]} and {bq.shape[1]} bytes for {k} values")
    if bias is not None:
        bias = _packed(bias, "bias", gpu, f32, (n,))
    if out is None:
        out = _empty(m, n, dtype=out_dtype, device=gpu)
        y_at, y_step = out.data_ptr(), n
    else:
        y_at, (y_step, _) = _rows(out, "out", gpu, out.dtype, (m, n))
    args = QuantArgs(ABI_VERSION, _dtype(out, "out"), _ACTS[act], n, k, m, a_at, b_at, a_step, b_step,
                     _packed(a_scale, "a.scale", gpu, f32, (m,)), _packed(b_scale, "b.scale", gpu, f32, (n,)), bias, y_at, y_step)
    _enqueue(_calls().evconv_quant_matmul, args, gpu)
    return out
