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


# ---- the paged cache

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def head_rows(x, weight, eps, freqs, pairs, positions):
    """Norm and rotation of heads [n, heads, d]."""
    x = np.array(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    if freqs is not None and len(freqs):
        half = len(freqs)
        a, b = (slice(0, half), slice(half, 2 * half)) if pairs == "halves" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        turn = np.exp(1j * np.asarray(positions, np.float64)[:, None] * np.asarray(freqs, np.float64))[:, None]
        z = (x[..., a] + 1j * x[..., b]) * turn
        x[..., a], x[..., b] = z.real, z.imag
    return x


def fp4_rows(x):
    """Codes and scales of rows of fp32, in fp32 as the header has it."""
    x = np.asarray(x, np.float32)
    m = np.abs(x).max(-1)
    with np.errstate(all="ignore"):
        y = (np.float32(6) * x / np.where(m > 0, m, np.float32(1))[..., None]).astype(np.float64)
        scale = m / np.float32(6)
    middle = (LEVELS[1:] + LEVELS[:-1]) / 2
    up = np.where(np.arange(7) % 2 == 1, np.abs(y)[..., None] >= middle, np.abs(y)[..., None] > middle)
    code = up.sum(-1) + 8 * (y < 0)
    fine = np.isfinite(m)
    return np.where(fine[..., None], code, 0).astype(np.uint8), np.where(fine, scale, np.float32(np.nan))


def fp4_values(code, scale):
    return np.where(code & 8, -1.0, 1.0) * LEVELS[code & 7] * np.asarray(scale, np.float64)[..., None]


def attend(q, k, v, scale, seen):
    """One head's rows: q [n, d], k, v [t, d], seen [n, t].  (o, the weights' sum over |v|)."""
    with np.errstate(all="ignore"):
        x = np.where(seen, q @ k.T * scale, -np.inf)
        top = x.max(-1, keepdims=True, initial=-np.inf)
        p = np.where(seen, np.exp(x - np.where(np.isfinite(top), top, 0)), 0)
        p = p / np.maximum(p.sum(-1, keepdims=True), 1e-300)
        hidden = ~seen.any(0)
        v = np.where(hidden[:, None], 0, v)
        return p @ v, p @ np.abs(v)


def choose(score, count, first, last):
    """Pages 0 .. len(score) - 1, the last one the query's own: the first and last ones, then by score."""
    n = len(score)
    rank = [(0, 0, i) if i < first or i >= n - last else (1, -np.inf if np.isnan(score[i]) else -float(score[i]), i) for i in range(n)]
    chosen = sorted(i for _, _, i in sorted(rank)[:count])
    return chosen + [-1] * (count - len(chosen))
