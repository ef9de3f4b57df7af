"""The sequence operators in 64 bits, straight from their formulas (numpy, token by token)."""
import numpy as np


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-x))


def delta_rule(q, k, v, gate, beta, state, spans, scale, normalize=False, a_scale=None, dt_bias=None):
    """q, k [n, hk, dk], v [n, hv, dv], gate, beta [n, hv], state [n_seq, hv, dk, dv]; spans: (first, length) of every
    sequence.  Returns (o, states)."""
    q, k, v, gate, beta = (np.asarray(x, np.float64) for x in (q, k, v, gate, beta))
    state = np.array(state, np.float64)
    o = np.zeros(v.shape)
    if normalize:
        q = q / np.sqrt((q * q).sum(-1, keepdims=True) + 1e-6)
        k = k / np.sqrt((k * k).sum(-1, keepdims=True) + 1e-6)
    if a_scale is not None:
        gate = -np.asarray(a_scale, np.float64) * np.logaddexp(0.0, gate + np.asarray(dt_bias, np.float64))
        beta = sigmoid(beta)
    share = v.shape[1] // k.shape[1]
    q, k = np.repeat(q, share, axis=1), np.repeat(k, share, axis=1)
    with np.errstate(all="ignore"):
        for i, (first, length) in enumerate(spans):
            s = state[i]
            for t in range(first, first + length):
                s = s * np.exp(gate[t])[:, None, None]
                d = beta[t][:, None] * (v[t] - np.einsum("hkv,hk->hv", s, k[t]))
                s = s + k[t][:, :, None] * d[:, None, :]
                o[t] = scale * np.einsum("hkv,hk->hv", s, q[t])
            state[i] = s
    return o, state


def norm(x, kind, eps):
    if kind == "layer":
        x = x - x.mean(-1, keepdims=True)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def block_norm(x=None, branch=None, gate=None, post_weight=None, post_bias=None, gate_act="none", group=None, res_scale=None,
               pre_norm=False, pre_weight=None, pre_bias=None, kind="rms", eps=1e-6):
    """(x', h) of one call."""
    x, branch, gate, post_weight, post_bias, res_scale, pre_weight, pre_bias = (
        None if a is None else np.asarray(a, np.float64)
        for a in (x, branch, gate, post_weight, post_bias, res_scale, pre_weight, pre_bias))
    y = x
    if branch is not None:
        rows, dim = branch.shape
        t = norm(branch.reshape(rows, -1, group or dim), kind, eps)
        if post_weight is not None:
            t = t * post_weight
        if post_bias is not None:
            t = t + post_bias
        t = t.reshape(rows, dim)
        if gate is not None:
            t = t * sigmoid(gate) * (gate if gate_act == "silu" else 1.0)
        if res_scale is not None:
            t = t * res_scale
        y = t if x is None else x + t
    h = y
    if pre_norm:
        h = norm(y, kind, eps)
        if pre_weight is not None:
            h = h * pre_weight
        if pre_bias is not None:
            h = h + pre_bias
    return y, h


def quantize_rows(x):
    """(q, scale) of fp32 rows; the operator defines scale, inverse and their products in 32 bits."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        big = np.abs(x).max(axis=1)
        inverse = np.where(big > 0, np.float32(127) * (np.float32(1) / big), np.float32(0)).astype(np.float32)
        bad = ~np.isfinite(big)
        q = np.rint(x * inverse[:, None])
        q[bad | ~np.isfinite(inverse)] = 0
        scale = np.where(bad, np.float32(np.nan), big / np.float32(127)).astype(np.float32)
    return q.astype(np.int8), scale


def quant_matmul(qa, sa, qb, sb, bias=None, act="none"):
    y = (qa.astype(np.float64) @ qb.astype(np.float64).T) * np.asarray(sa, np.float64)[:, None] * np.asarray(sb, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return {"none": lambda v: v, "relu": lambda v: np.where(v < 0, 0.0, v), "sigmoid": sigmoid, "tanh": np.tanh}[act](y)
