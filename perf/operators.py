"""The sequence operators whose time counts: the gated delta rule over the tokens of independent
streams, the norms around a block with its gate and residual, and the product in 8-bit integers with
a scale per token and per channel, through the calls a program makes (`ops.delta_rule`,
`ops.block_norm`, `ops.quantize_rows`, `ops.quant_matmul`).

A stream's token is the feature vector of one time window; a whole recording is a sequence of them.
`run` computes the operators in elementary torch operations in 32 bits, or through the framework where
`own` is set.
"""
import math

import torch

own = False

CHUNK = 64  # tokens that the plain form of the delta rule takes at once
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    def delta(name, n_seq, length, hk, hv, dk, dv, dtype, ragged=False, fused=True):
        return dict(name=name, op="delta", n_seq=n_seq, length=length, ragged=ragged, hk=hk, hv=hv, dk=dk, dv=dv,
                    dtype=dtype, fused=fused)

    def norm(name, rows, dim, dtype, kind="rms", gate="sigmoid"):
        return dict(name=name, op="norm", rows=rows, dim=dim, dtype=dtype, kind=kind, gate=gate)

    def linear(name, rows, k, n, dtype, bias=False, act="none", heads=0):
        return dict(name=name, op="linear", rows=rows, k=k, n=n, dtype=dtype, bias=bias, act=act, heads=heads)

    return [
        # one new window of each of sixteen cameras: the latency of a step
        delta("delta_step_16", 16, 1, 4, 4, 64, 64, "f32"),
        # one new window of each of 256 streams, two value heads to a key head: the states' bytes
        delta("delta_step_256", 256, 1, 8, 16, 128, 128, "bf16"),
        # recordings of different lengths, empty ones and single windows among them, odd head sizes
        delta("delta_window_ragged", 24, 700, 3, 6, 80, 112, "f32", ragged=True, fused=False),
        # one long recording: few independent rows, a long axis
        delta("delta_history_32768", 1, 32768, 8, 16, 128, 128, "bf16"),
        # eight recordings at once: the largest call
        delta("delta_batch_8x4096", 8, 4096, 16, 32, 128, 128, "bf16"),
        # the norms around a block for sixteen tokens
        norm("norm_16x512", 16, 512, "f32"),
        # the same for a whole batch of recordings
        norm("norm_16384x2048", 16384, 2048, "bf16", gate="silu"),
        # mean and variance, a width and a count that are no multiple of anything
        norm("norm_layer_4099x1000", 4099, 1000, "f32", kind="layer", gate="none"),
        # a projection of sixteen tokens
        linear("linear_16x512x1536", 16, 512, 1536, "f32", bias=True),
        # odd sizes throughout
        linear("linear_1001x1000x777", 1001, 1000, 777, "f32", bias=True, act="tanh"),
        # the projection behind the delta rule: each head normed and gated, quantised in the same pass
        linear("linear_heads_2048x2048x1024", 2048, 2048, 1024, "bf16", heads=16),
        # the projection of a whole batch of recordings
        linear("linear_16384x2048x8192", 16384, 2048, 8192, "bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    dtype = rng.choice(["f32", "bf16"])
    op = rng.choice(["step", "window", "window", "norm", "linear", "linear"])
    if op in ("step", "window"):
        hk = rng.choice([1, 2, 3, 4, 8])
        hv = hk * rng.choice([1, 1, 2, 3])
        dk, dv = (rng.choice([32, 64, 96, 128, rng.randint(16, 128)]) for _ in range(2))
        if op == "step":
            n_seq, length, ragged = log_int(1, 256), rng.choice([1, 1, 1, 2, 5]), False
            n_seq = max(1, min(n_seq, 4096 // hv))
        else:
            length, ragged = log_int(9, 16384), rng.random() < 0.5
            n_seq = log_int(1, max(1, min(32, (1 << 18) // (length * hv))))
        return dict(op="delta", n_seq=n_seq, length=length, ragged=ragged, hk=hk, hv=hv, dk=dk, dv=dv, dtype=dtype,
                    fused=rng.random() < 0.5)
    if op == "norm":
        dim = rng.choice([256, 512, 1024, 2048, 4096, log_int(33, 4100)])
        return dict(op="norm", rows=log_int(1, max(2, (1 << 24) // dim)), dim=dim, dtype=dtype,
                    kind=rng.choice(["rms", "rms", "layer"]), gate=rng.choice(["none", "sigmoid", "silu"]))
    heads = rng.choice([0, 0, 0, 2, 8, 16]) if dtype == "bf16" else 0
    n = rng.choice([512, 1024, 2048, 4096, log_int(17, 4100)])
    k = heads * rng.choice([64, 112, 128]) if heads else rng.choice([512, 1024, 2048, 4096, log_int(33, 4100)])
    return dict(op="linear", rows=rng.choice([1, 16, log_int(1, 8192), log_int(1, 8192)]), k=k, n=n, dtype=dtype,
                bias=rng.random() < 0.5, act=rng.choice(["none", "none", "sigmoid", "tanh", "relu"]), heads=heads)


# ------------------------------------------------------------------- inputs

def _lengths(case):
    """Token counts of the sequences, the case's own: all alike, or spread from 0 to `length`."""
    if not case["ragged"]:
        return [case["length"]] * case["n_seq"]
    g = torch.Generator().manual_seed(case["n_seq"] * 65537 + case["length"])
    lens = (torch.rand(case["n_seq"], generator=g) * (case["length"] + 1)).long().tolist()
    lens[0] = case["length"]
    if case["n_seq"] > 2:
        lens[1], lens[2] = 0, 1
    return lens


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    if case["op"] == "delta":
        lens = _lengths(case)
        n, hk, hv, dk, dv = sum(lens), case["hk"], case["hv"], case["dk"], case["dv"]
        # the features of neighbouring windows are alike: a part of every key is the head's own
        k = 0.8 * normal(n, hk, dk) + 0.6 * normal(1, hk, dk)
        q = 0.8 * normal(n, hk, dk) + 0.6 * normal(1, hk, dk)
        s = dict(case, lens=lens, v=normal(n, hv, dv).to(t), state=0.3 * normal(case["n_seq"], hv, dk, dv))
        s["offsets"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda") \
            if case["ragged"] else None
        if case["fused"]:  # keys and queries as they come out of a projection, gates before their activations
            s.update(q=q.to(t), k=k.to(t), a=normal(n, hv).to(t), b=normal(n, hv).to(t),
                     a_scale=torch.exp(uniform(hv) * 4 - 5), dt_bias=0.5 * normal(hv))
        else:
            s.update(q=(q / q.norm(dim=-1, keepdim=True)).to(t), k=(k / k.norm(dim=-1, keepdim=True)).to(t),
                     a=-torch.exp(uniform(n, hv) * 6 - 7), b=torch.sigmoid(normal(n, hv)), a_scale=None, dt_bias=None)
        return s
    if case["op"] == "norm":
        r, d = case["rows"], case["dim"]
        s = dict(case, x=(2 * normal(r, d)).to(t), branch=(0.5 + normal(r, d)).to(t),
                 z=normal(r, d).to(t) if case["gate"] != "none" else None, post_weight=1 + 0.1 * normal(d),
                 pre_weight=1 + 0.1 * normal(d), res_scale=0.1 * uniform(d), post_bias=None, pre_bias=None)
        if case["kind"] == "layer":
            s.update(post_bias=0.1 * normal(d), pre_bias=0.1 * normal(d))
        return s
    r, k, n = case["rows"], case["k"], case["n"]
    # a weight of 8 bits as a program keeps it: rows of int8 padded with zeros to whole 128 bytes, one scale per row
    w = normal(n, k) / math.sqrt(k)
    big = w.abs().amax(dim=1)
    wq = torch.zeros(n, -(-k // 128) * 128, dtype=torch.int8, device="cuda")
    wq[:, :k] = torch.round(w * (127 / big)[:, None]).to(torch.int8)
    s = dict(case, x=normal(r, k).to(t), wq=wq, w_scale=big / 127, bias=0.1 * normal(n) if case["bias"] else None)
    if case["heads"]:
        s.update(z=normal(r, k).to(t), post_weight=1 + 0.1 * normal(k // case["heads"]))
    return s


# ------------------------------------------------------------------- one pass

def run(s):
    return {"delta": run_delta, "norm": run_norm, "linear": run_linear}[s["op"]](s)


def run_delta(s):
    if own:
        from paper_2303_04670_amd import ops
        o, state = ops.delta_rule(s["q"], s["k"], s["v"], s["a"], s["b"], s["state"], seq_offsets=s["offsets"],
                                  normalize=s["fused"], a_scale=s["a_scale"], dt_bias=s["dt_bias"])
        return {"o": o, "state": state}
    return plain_delta(s)


def run_norm(s):
    if own:
        from paper_2303_04670_amd import ops
        r = ops.block_norm(s["x"], s["branch"], s["z"], post_weight=s["post_weight"], post_bias=s["post_bias"],
                           gate_act=s["gate"], res_scale=s["res_scale"], pre_weight=s["pre_weight"],
                           pre_bias=s["pre_bias"], kind=s["kind"])
        return {"x": r.x, "h": r.h}
    t = s["x"].dtype
    b = plain_norm(s["branch"].float(), s["kind"], s["post_weight"], s["post_bias"])
    if s["gate"] != "none":
        b = b * plain_gate(s["z"].float(), s["gate"])
    x = s["x"].float() + s["res_scale"] * b
    h = plain_norm(x, s["kind"], s["pre_weight"], s["pre_bias"])
    return {"x": x.to(t), "h": h.to(t)}


def run_linear(s):
    if own:
        from paper_2303_04670_amd import ops
        if s["heads"]:
            rows = ops.block_norm(None, s["x"], s["z"], post_weight=s["post_weight"], gate_act="silu",
                                  group=s["k"] // s["heads"], want="q").q
        else:
            rows = ops.quantize_rows(s["x"])
        return ops.quant_matmul(rows, ops.QuantRows(s["wq"], s["w_scale"], s["k"]), bias=s["bias"], act=s["act"],
                                out_dtype=s["x"].dtype)
    x = s["x"].float()
    if s["heads"]:
        x = plain_norm(x.view(s["rows"], s["heads"], -1), "rms", s["post_weight"], None).view(s["rows"], -1)
        x = x * plain_gate(s["z"].float(), "silu")
    big = x.abs().amax(dim=1, keepdim=True)
    inverse = torch.where(big > 0, 127 / big, torch.zeros_like(big))
    q = torch.round(x * inverse)
    y = torch.matmul(q, s["wq"][:, :s["k"]].float().t()) * (big / 127) * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["act"] == "relu":
        y = torch.clamp(y, min=0)
    elif s["act"] == "sigmoid":
        y = 1 / (1 + torch.exp(-y))
    elif s["act"] == "tanh":
        y = torch.tanh(y)
    return y.to(s["x"].dtype)


def plain_norm(x, kind, weight, bias, eps=1e-6):
    if kind == "layer":
        x = x - x.mean(dim=-1, keepdim=True)
    x = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + eps) * weight
    return x if bias is None else x + bias


def plain_gate(z, act):
    y = 1 / (1 + torch.exp(-z))
    return z * y if act == "silu" else y


def plain_operands(s):
    q, k, v, a, b = (s[i].float() for i in ("q", "k", "v", "a", "b"))
    if s["fused"]:
        q = q / torch.sqrt((q * q).sum(dim=-1, keepdim=True) + 1e-6)
        k = k / torch.sqrt((k * k).sum(dim=-1, keepdim=True) + 1e-6)
        a = -s["a_scale"] * torch.log1p(torch.exp(a + s["dt_bias"]))
        b = 1 / (1 + torch.exp(-b))
    return q * s["dk"] ** -0.5, k, v, a, b


def plain_steps(s):
    """A few tokens of every sequence, one after the other."""
    n_seq, hv, share = s["n_seq"], s["hv"], s["hv"] // s["hk"]
    q, k, v, a, b = (x.view(n_seq, -1, *x.shape[1:]) for x in plain_operands(s))
    q, k = q.repeat_interleave(share, dim=2)[..., None], k.repeat_interleave(share, dim=2)[..., None]
    state, out = s["state"], []
    for i in range(v.shape[1]):
        state = state * torch.exp(a[:, i])[..., None, None]
        new = b[:, i, :, None] * (v[:, i] - (state * k[:, i]).sum(dim=2))
        state = state + k[:, i] * new[:, :, None]
        out.append((state * q[:, i]).sum(dim=2))
    o = torch.stack(out, dim=1).view(-1, hv, s["dv"])
    return {"o": o.to(s["v"].dtype), "state": state}


def plain_delta(s):
    """The delta rule a chunk of tokens at a time: within a chunk as products with the inverse of a
    unit lower triangular matrix, from chunk to chunk through the state."""
    n_seq, hk, hv, dk, dv, t = s["n_seq"], s["hk"], s["hv"], s["dk"], s["dv"], s["v"].dtype
    longest, lens = max(s["lens"]), s["lens"]
    if longest <= 8 and not s["ragged"]:
        return plain_steps(s)
    c = CHUNK
    length = -(-longest // c) * c
    q, k, v, a, b = plain_operands(s)
    # tokens of a sequence in a row of their own, [n_seq, heads, chunks, c, d]; what is behind its end is zero
    n = sum(lens)
    place = torch.full((n_seq, length), n, device=v.device)
    at = torch.arange(length, device=v.device)
    count = torch.tensor(lens, device=v.device)
    first = torch.cumsum(count, 0) - count
    place = torch.where(at < count[:, None], first[:, None] + at, place)

    def rows(x, heads):
        x = torch.cat([x, torch.zeros_like(x[:1])])[place]
        x = x.view(n_seq, length // c, c, x.shape[2], -1).permute(0, 3, 1, 2, 4)
        return x.repeat_interleave(hv // x.shape[1], dim=1).contiguous()

    q, k, v = rows(q, hk), rows(k, hk), rows(v, hv)
    g, b = torch.cumsum(rows(a[..., None], hv), dim=3), rows(b[..., None], hv)
    lower = torch.ones(c, c, device=v.device).tril()
    decay = torch.exp((g - g.transpose(3, 4)) * lower) * lower
    kt = k.transpose(3, 4).contiguous()
    m = torch.matmul(k, kt) * decay * b * (lower - torch.eye(c, device=v.device))
    p = torch.matmul(q, kt) * decay
    inv = torch.eye(c, device=v.device).expand_as(m).contiguous()
    size = 1
    while size < c:  # blocks of twice the size from the inverses on the diagonal and the block below
        for i in range(0, c, 2 * size):
            x, y, z = slice(i, i + size), slice(i + size, i + 2 * size), slice(i, i + size)
            inv[..., y, z] = -torch.matmul(torch.matmul(inv[..., y, y].contiguous(), m[..., y, x].contiguous()),
                                           inv[..., x, x].contiguous())
        size *= 2
    u = torch.matmul(inv, b * v)
    w = torch.matmul(inv, b * torch.exp(g) * k)
    q = q * torch.exp(g)
    last = g[:, :, :, -1:, :]
    kt = kt * torch.exp(last - g).transpose(3, 4)
    state, out = s["state"], []
    for i in range(length // c):
        new = u[:, :, i] - torch.matmul(w[:, :, i], state)
        out.append(torch.matmul(q[:, :, i], state) + torch.matmul(p[:, :, i], new))
        state = state * torch.exp(last[:, :, i]) + torch.matmul(kt[:, :, i], new)
    o = torch.stack(out, dim=2).permute(0, 2, 3, 1, 4).reshape(n_seq * length, hv, dv)
    keep = (place.view(-1) < n).nonzero()[:, 0]
    return {"o": o[keep].to(t), "state": state}


# ------------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "delta":
        n = sum(_lengths(case))
        hk, hv, dk, dv = (case[i] for i in ("hk", "hv", "dk", "dv"))
        gates = n * hv * 2 * (size if case["fused"] else 4)
        state = 2 * 4 * case["n_seq"] * hv * dk * dv
        # read, write and update of the state, a product and a sum for each of its values
        return {"bytes": n * (2 * hk * dk + 2 * hv * dv) * size + gates + state, "flops": 6.0 * n * hv * dk * dv}
    if case["op"] == "norm":
        values = case["rows"] * case["dim"]
        return {"bytes": values * size * (4 + (case["gate"] != "none")) + 12 * case["dim"], "flops": 16.0 * values}
    r, k, n = case["rows"], case["k"], case["n"]
    return {"bytes": r * k * size * (2 if case["heads"] else 1) + n * k + r * n * size + 4 * n * (2 if case["bias"] else 1),
            "flops": 2.0 * r * k * n}


# ------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "delta":
        return exact_delta(s)
    double = {i: x.double() for i, x in s.items() if torch.is_tensor(x) and x.is_floating_point()}
    if case["op"] == "norm":
        y = exact_norm(double["branch"], s["kind"]) * double["post_weight"]
        if s["post_bias"] is not None:
            y = y + double["post_bias"]
        if s["gate"] != "none":
            y = y * torch.sigmoid(double["z"]) * (double["z"] if s["gate"] == "silu" else 1)
        x = double["x"] + double["res_scale"] * y
        h = exact_norm(x, s["kind"]) * double["pre_weight"]
        return {"x": x, "h": h + double["pre_bias"] if s["pre_bias"] is not None else h}
    x = double["x"]
    if case["heads"]:
        x = exact_norm(x.view(s["rows"], s["heads"], -1), "rms") * double["post_weight"]
        x = (x.view(s["rows"], -1) * double["z"] * torch.sigmoid(double["z"])).float().double()
    # the operator's quantisation is defined in 32 bits: the scale, its inverse and the product with it
    big = x.abs().max(dim=1).values.float()
    inverse = torch.where(big > 0, 127 / big, torch.zeros_like(big))
    q = torch.round(x.float() * inverse[:, None]).double()
    y = q @ s["wq"][:, :s["k"]].double().t().contiguous() * (big / 127).double()[:, None] * double["w_scale"]
    if s["bias"] is not None:
        y = y + double["bias"]
    return {"none": lambda v: v, "relu": torch.relu, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[s["act"]](y)


def exact_norm(x, kind, eps=1e-6):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)


def exact_delta(s):
    """Token by token: S = exp(g) S; S += beta k (v - S' k)'; o = scale S' q."""
    q, k, v, g, b = (s[i].double() for i in ("q", "k", "v", "a", "b"))
    if s["fused"]:
        q = q * torch.rsqrt(q.square().sum(-1, keepdim=True) + 1e-6)
        k = k * torch.rsqrt(k.square().sum(-1, keepdim=True) + 1e-6)
        g = -s["a_scale"].double() * torch.nn.functional.softplus(g + s["dt_bias"].double())
        b = torch.sigmoid(b)
    share = s["hv"] // s["hk"]
    q, k = (x.repeat_interleave(share, dim=1) * f for x, f in ((q, s["dk"] ** -0.5), (k, 1)))
    state, o = s["state"].double(), torch.zeros_like(v)
    lens = s["lens"]
    first = [sum(lens[:i]) for i in range(len(lens))]
    count = torch.tensor(lens)
    start = torch.tensor(first, device=v.device)
    for step in range(max(lens)):
        live = (count > step).nonzero()[:, 0].to(v.device) if s["ragged"] else slice(None)
        row = start[live] + step
        x = state[live] * torch.exp(g[row])[..., None, None]
        kk = k[row][..., None]
        delta = b[row][..., None] * (v[row] - (x * kk).sum(2))
        x = x + kk * delta[:, :, None]
        o[row] = (x * q[row][..., None]).sum(2)
        if s["ragged"]:
            state[live] = x
        else:
            state = x
    return {"o": o, "state": state}
