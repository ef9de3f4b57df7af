"""The sequence operators on the GPU, through the C ABI's binding, against their formulas in 64 bits.

Tolerances, all set beforehand.  fp32 results: 2^-18 of the tensor's norm and 2^-15 of its largest
magnitude for any one value (64 roundings of 2^-24 in a row; a value is a sum of up to some hundred
terms, whose roundings add up to less than that for random signs).  bf16 results: 2^-8 of the value
(half a step is 2^-9) plus 2^-12 of the largest magnitude."""
import numpy as np
import pytest

import ops_ref
from paper_2303_04670_amd import evconv as ev

pytestmark = pytest.mark.gpu


def close(got, want, bf16=False):
    got, want = got.detach().float().cpu().numpy().astype(np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), "values that are not finite, elsewhere"
    if not fine.any():
        return
    d, w = np.abs(got - want)[fine], np.abs(want)[fine]
    if bf16:
        assert (d <= 2.0 ** -8 * w + 2.0 ** -12 * w.max()).all(), (d - 2.0 ** -8 * w).max() / w.max()
    else:
        assert np.linalg.norm(d) <= 2.0 ** -18 * np.linalg.norm(w), np.linalg.norm(d) / np.linalg.norm(w)
        assert d.max() <= 2.0 ** -15 * w.max(), d.max() / w.max()


def torch_ops():
    import torch
    from paper_2303_04670_amd import ops
    return torch, ops


def delta_inputs(seed, n, n_seq, hk, hv, dk, dv, dtype, raw):
    import torch
    g = torch.Generator().manual_seed(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    normal = lambda *s: torch.randn(*s, generator=g)
    k = normal(n, hk, dk) + 0.7 * normal(1, hk, dk)
    x = dict(q=normal(n, hk, dk), k=k if raw else k / k.norm(dim=-1, keepdim=True), v=normal(n, hv, dv),
             state=0.5 * normal(n_seq, hv, dk, dv), a_scale=None, dt_bias=None)
    if raw:
        x.update(gate=normal(n, hv).to(t), beta=normal(n, hv).to(t), a_scale=torch.exp(normal(hv) - 2), dt_bias=normal(hv))
    else:
        x.update(gate=-torch.exp(2 * normal(n, hv) - 2), beta=torch.sigmoid(normal(n, hv)))
    return {name: a.to(t) if name in ("q", "k", "v") else a for name, a in x.items()}


def spans_of(lens):
    first = np.concatenate([[0], np.cumsum(lens)])
    return [(int(first[i]), int(lens[i])) for i in range(len(lens))]


def numbers(x):
    return {n: None if a is None else a.float().numpy() for n, a in x.items()}


def offsets(lens):
    import torch
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()


def run_delta(x, lens, ragged=True, **kw):
    """(o, state, o and state in 64 bits) of one call."""
    torch, ops = torch_ops()
    raw = x["a_scale"] is not None
    d = {n: None if a is None else a.cuda() for n, a in x.items()}
    o, s = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], normalize=raw, a_scale=d["a_scale"],
                          dt_bias=d["dt_bias"], seq_offsets=offsets(lens) if ragged else None, **kw)
    torch.cuda.synchronize()
    c = numbers(x)
    scale = kw.get("scale", x["q"].shape[2] ** -0.5)
    want = ops_ref.delta_rule(c["q"], c["k"], c["v"], c["gate"], c["beta"], c["state"], spans_of(lens), scale, raw, c["a_scale"], c["dt_bias"])
    return o, s, want[0], want[1]


LENS = [0, 1, 2, 15, 16, 17, 63, 64, 65, 128, 129, 200]


@pytest.mark.parametrize("raw", [False, True], ids=["gates", "raw"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hk,hv,dk,dv", [(1, 1, 64, 64), (2, 6, 128, 128), (2, 2, 96, 40), (1, 2, 37, 51), (1, 1, 256, 256),
                                         (1, 1, 1, 1), (3, 3, 8, 17), (1, 1, 136, 20)])
def test_delta_rule_over_lengths(hk, hv, dk, dv, dtype, raw):
    x = delta_inputs(hash((hk, dk, dv)) % 1000, sum(LENS), len(LENS), hk, hv, dk, dv, dtype, raw)
    o, s, want_o, want_s = run_delta(x, LENS)
    close(o, want_o, dtype == "bf16")
    close(s, want_s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length", [1, 3, 16, 17, 64, 100])
def test_delta_rule_equal_lengths(length, dtype):
    x = delta_inputs(length, 3 * length, 3, 2, 4, 64, 48, dtype, True)
    o, s, want_o, want_s = run_delta(x, [length] * 3, ragged=False, scale=0.7)
    close(o, want_o, dtype == "bf16")
    close(s, want_s)


def test_delta_rule_long_sequence():
    x = delta_inputs(11, 3000, 1, 1, 2, 32, 24, "f32", True)
    o, s, want_o, want_s = run_delta(x, [3000], ragged=False)
    close(o, want_o)
    close(s, want_s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hk,hv,dk,dv", [(1, 2, 32, 16), (2, 2, 96, 128), (1, 2, 80, 112), (1, 1, 200, 30)])
def test_delta_rule_every_short_length(hk, hv, dk, dv, dtype):
    """Lengths on both sides of where tokens go one by one, alike and of their own."""
    calls = [([n, n, n], False) for n in range(1, 15)] + [(list(range(16)), True)]
    for lens, ragged in calls:
        x = delta_inputs(60 + len(lens) + lens[0], sum(lens), len(lens), hk, hv, dk, dv, dtype, True)
        o, s, want_o, want_s = run_delta(x, lens, ragged=ragged)
        close(o, want_o, dtype == "bf16")
        close(s, want_s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hk,hv,dk,dv", [(1, 2, 64, 64), (2, 2, 128, 128), (1, 1, 40, 24), (1, 1, 37, 70), (1, 1, 128, 17), (1, 1, 96, 128), (1, 2, 24, 72)])
def test_delta_rule_in_segments(hk, hv, dk, dv, dtype):
    """Sequences long enough, and heads few enough, to be worked on in segments side by side; states in place."""
    torch, ops = torch_ops()
    for lens in ([4500], [70, 9000, 0, 5, 3100]):
        x = delta_inputs(16 + dk, sum(lens), len(lens), hk, hv, dk, dv, dtype, True)
        d = {n: a.cuda() for n, a in x.items()}
        o, s = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], state_out=d["state"], seq_offsets=offsets(lens),
                              normalize=True, a_scale=d["a_scale"], dt_bias=d["dt_bias"])
        c = numbers(x)
        want_o, want_s = ops_ref.delta_rule(c["q"], c["k"], c["v"], c["gate"], c["beta"], c["state"], spans_of(lens), dk ** -0.5, True,
                                            c["a_scale"], c["dt_bias"])
        close(o, want_o, dtype == "bf16")
        close(s, want_s)
    # no state to begin with, none to leave, and a value that is not finite in one column of one segment
    n = 4500
    x = delta_inputs(17, n, 1, hk, hv, dk, dv, dtype, True)
    d = {name: a.cuda() for name, a in x.items()}
    kw = dict(normalize=True, a_scale=d["a_scale"], dt_bias=d["dt_bias"])
    o, s = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], 0 * d["state"], n_seq=1, **kw)
    p, t = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], **kw)
    assert torch.equal(o, p) and torch.equal(s, t)
    p, t = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], n_seq=1,
                          slots=torch.full((1,), -1, dtype=torch.int32, device="cuda"), state_out=torch.full_like(s, 5.0), **kw)
    assert torch.equal(o, p) and (t == 5.0).all()
    d["v"][2000, 0, 3] = np.nan
    p, t = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], **kw)
    rest = [i for i in range(dv) if i != 3]
    assert torch.equal(p[:, :, rest], o[:, :, rest]) and torch.equal(p[:2000], o[:2000]) and torch.equal(p[:, 1:], o[:, 1:])
    assert torch.equal(t[..., rest], s[..., rest]) and t[0, 0, :, 3].isnan().all() and p[2000:, 0, 3].isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_delta_rule_reads_slices_of_a_projection(dtype):
    """q, k, v and the gates as strided views, rows at odd addresses too, give the bits of contiguous ones."""
    torch, ops = torch_ops()
    lens, hk, hv, dk, dv = [0, 5, 150], 2, 4, 40, 24
    x = delta_inputs(5, sum(lens), 3, hk, hv, dk, dv, dtype, True)
    d = {n: a.cuda() for n, a in x.items()}
    kw = dict(normalize=True, a_scale=d["a_scale"], dt_bias=d["dt_bias"], seq_offsets=offsets(lens))
    want = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], **kw)
    for pad in (0, 1):
        parts = [d["q"].flatten(1), d["k"].flatten(1), d["v"].flatten(1), d["gate"], d["beta"]]
        wide = torch.cat([torch.zeros_like(parts[0][:, :pad])] + parts, dim=1)
        at, views = pad, []
        for p in parts:
            views.append(wide[:, at:at + p.shape[1]])
            at += p.shape[1]
        heads = [hk, hk, hv]
        views[:3] = [v.unflatten(1, (h, -1)) for v, h in zip(views, heads)]
        out = torch.zeros(sum(lens), 2 * hv, dv, dtype=d["v"].dtype, device="cuda")[:, ::2]
        got = ops.delta_rule(*views, d["state"], out=out, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dk,dv", [(64, 32), (128, 40), (37, 51)])
@pytest.mark.parametrize("which", ["q", "k", "v", "gate", "out"])
def test_delta_rule_tokens_far_apart(which, dk, dv):
    """More than 2^23 elements from token to token in one of the tensors: bf16 chunks in two launches."""
    torch, ops = torch_ops()
    lens, step = [70, 0, 20], (1 << 23) + 64
    n = sum(lens)
    x = delta_inputs(26, n, 3, 1, 2, dk, dv, "bf16", True)
    d = {name: a.cuda() for name, a in x.items()}
    d["out"] = torch.empty_like(d["v"])
    room = torch.empty(n * step, dtype=torch.bfloat16, device="cuda")
    far = room.as_strided(d[which].shape, (step,) + d[which].stride()[1:])
    far.copy_(d[which])
    d[which] = far
    o, s = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], seq_offsets=offsets(lens), out=d["out"], normalize=True,
                          a_scale=d["a_scale"], dt_bias=d["dt_bias"])
    c = numbers(x)
    want_o, want_s = ops_ref.delta_rule(c["q"], c["k"], c["v"], c["gate"], c["beta"], c["state"], spans_of(lens), dk ** -0.5, True, c["a_scale"],
                                        c["dt_bias"])
    assert o is d["out"]
    close(o, want_o, True)
    close(s, want_s)


def test_delta_rule_slots_and_states_in_place():
    torch, ops = torch_ops()
    lens = [3, 0, 70, 1, 20]
    x = delta_inputs(6, sum(lens), 9, 1, 2, 64, 32, "f32", False)
    d = {n: None if a is None else a.cuda() for n, a in x.items()}
    slots = [7, 2, 0, -1, 9]  # the last two have none: below zero, behind the last
    before = d["state"].clone()
    o, s = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], seq_offsets=offsets(lens),
                          slots=torch.tensor(slots, dtype=torch.int32).cuda())
    assert s is d["state"]
    c = numbers(x)
    start = np.stack([c["state"][i] if 0 <= i < 9 else np.zeros_like(c["state"][0]) for i in slots])
    want_o, want_s = ops_ref.delta_rule(c["q"], c["k"], c["v"], c["gate"], c["beta"], start, spans_of(lens), 64 ** -0.5)
    close(o, want_o)
    for i, slot in enumerate(slots[:3]):
        close(s[slot], want_s[i])
    rest = [i for i in range(9) if i not in slots]
    assert torch.equal(s[rest], before[rest]) and torch.equal(s[2], before[2])


def test_delta_rule_without_states_and_without_tokens():
    torch, ops = torch_ops()
    x = delta_inputs(7, 100, 1, 1, 1, 32, 32, "f32", False)
    d = {n: None if a is None else a.cuda() for n, a in x.items()}
    o, s = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"])
    c = numbers(x)
    want_o, want_s = ops_ref.delta_rule(c["q"], c["k"], c["v"], c["gate"], c["beta"], 0 * c["state"], [(0, 100)], 32 ** -0.5)
    close(o, want_o)
    close(s, want_s)
    o, t = ops.delta_rule(d["q"][:0], d["k"][:0], d["v"][:0], d["gate"][:0], d["beta"][:0], s)
    assert o.shape == (0, 1, 32) and torch.equal(t, s) and t is not s


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length", [1, 40])
def test_delta_rule_new_states_of_more_slots_than_sequences(length, dtype):
    """A new tensor of states has those of no sequence too: they stay as they were."""
    torch, ops = torch_ops()
    x = delta_inputs(21, 3 * length, 8, 1, 2, 64, 32, dtype, True)
    d = {n: a.cuda() for n, a in x.items()}
    before = d["state"].clone()
    for kw in (dict(n_seq=3), dict(seq_offsets=offsets([length] * 3))):
        junk = [torch.full_like(before, 7.0) for _ in range(4)]  # (what the new tensor may be made from)
        del junk
        o, s = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], normalize=True, a_scale=d["a_scale"],
                              dt_bias=d["dt_bias"], **kw)
        c = numbers(x)
        want_o, want_s = ops_ref.delta_rule(c["q"], c["k"], c["v"], c["gate"], c["beta"], c["state"][:3], spans_of([length] * 3), 64 ** -0.5,
                                            True, c["a_scale"], c["dt_bias"])
        close(o, want_o, dtype == "bf16")
        close(s[:3], want_s)
        assert s is not d["state"] and torch.equal(s[3:], before[3:]) and torch.equal(d["state"], before)


def test_delta_rule_n_seq_beside_offsets():
    torch, ops = torch_ops()
    x = delta_inputs(28, 6, 3, 1, 1, 16, 16, "f32", False)
    d = {n: None if a is None else a.cuda() for n, a in x.items()}
    call = lambda n_seq: ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], seq_offsets=offsets([1, 2, 3]), n_seq=n_seq)
    want = call(None)
    got = call(3)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for n_seq in (2, 6):
        with pytest.raises(ev.EvConvError) as e:
            call(n_seq)
        assert e.value.status == ev.ERR_SHAPE


def test_delta_rule_slots_need_states():
    """How many slots there are is known from `state` or `state_out` only."""
    torch, ops = torch_ops()
    x = delta_inputs(22, 2, 8, 1, 2, 64, 32, "f32", False)
    d = {n: None if a is None else a.cuda() for n, a in x.items()}
    slots = torch.tensor([5, 7], dtype=torch.int32).cuda()
    tokens = (d["q"], d["k"], d["v"], d["gate"], d["beta"])
    with pytest.raises(ev.EvConvError) as e:
        ops.delta_rule(*tokens, slots=slots)
    assert e.value.status == ev.ERR_INVALID_ARG
    out = torch.full_like(d["state"], 5.0)
    _, s = ops.delta_rule(*tokens, slots=slots, state_out=out)
    c = numbers(x)
    _, want = ops_ref.delta_rule(c["q"], c["k"], c["v"], c["gate"], c["beta"], 0 * c["state"][:2], [(0, 1), (1, 1)], 64 ** -0.5)
    close(s[[5, 7]], want)
    assert s is out and (s[[0, 1, 2, 3, 4, 6]] == 5.0).all()


@pytest.mark.parametrize("ragged", [False, True])
def test_delta_rule_without_tokens_hands_the_states_on(ragged):
    torch, ops = torch_ops()
    x = delta_inputs(20, 4, 3, 1, 2, 32, 16, "f32", True)
    d = {n: a.cuda() for n, a in x.items()}
    tokens = [d[n][:0] for n in ("q", "k", "v", "gate", "beta")]
    kw = dict(normalize=True, seq_offsets=offsets([0, 0, 0]) if ragged else None)
    o, s = ops.delta_rule(*tokens, d["state"], a_scale=d["a_scale"], dt_bias=d["dt_bias"], **kw)
    assert o.shape == (0, 2, 16) and s is not d["state"] and torch.equal(s, d["state"])
    for given in (dict(a_scale=d["a_scale"]), dict(dt_bias=d["dt_bias"])):
        with pytest.raises(ev.EvConvError) as e:
            ops.delta_rule(*tokens, d["state"], **given, **kw)
        assert e.value.status == ev.ERR_INVALID_ARG


def test_delta_rule_state_behind_32_bits():
    """A slot whose first value is at index 2^31 and more of the cache."""
    torch, ops = torch_ops()
    hv, dk, dv = 8, 128, 128
    n_slots = (1 << 31) // (hv * dk * dv) + 3
    cache = torch.empty(n_slots, hv, dk, dv, device="cuda")
    for lens in ([1, 2], [70, 40]):
        x = delta_inputs(8, sum(lens), 2, 4, hv, dk, dv, "bf16", True)
        slots = [n_slots - 1, n_slots - 2]
        for i, slot in enumerate(slots):
            cache[slot] = x["state"][i].cuda()
        x["state"], keep = cache, x["state"]
        d = {n: a.cuda() for n, a in x.items()}
        o, _ = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], cache, seq_offsets=offsets(lens), normalize=True,
                              slots=torch.tensor(slots, dtype=torch.int32).cuda(), a_scale=d["a_scale"], dt_bias=d["dt_bias"])
        c = numbers({n: a for n, a in x.items() if n != "state"})
        want_o, want_s = ops_ref.delta_rule(c["q"], c["k"], c["v"], c["gate"], c["beta"], keep.numpy(), spans_of(lens), dk ** -0.5,
                                            True, c["a_scale"], c["dt_bias"])
        close(o, want_o, True)
        for i, slot in enumerate(slots):
            close(cache[slot], want_s[i])


@pytest.mark.parametrize("length", [9, 200])
def test_delta_rule_decays(length):
    """No decay, strong decay, a decay that forgets everything (-inf), and tokens that do nothing."""
    x = delta_inputs(9, 2 * length, 2, 1, 2, 64, 16, "f32", False)
    x["gate"][::3] = 0.0
    x["gate"][4] = -np.inf
    x["gate"][5, 1] = -3e38
    x["gate"][7] = -90.0
    x["beta"][::4] = 0.0
    x["beta"][1::4] = 1.0
    o, s, want_o, want_s = run_delta(x, [length] * 2, ragged=False)
    close(o, want_o)
    close(s, want_s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_delta_rule_same_key_over_and_over(dtype):
    """Keys that are all alike, full strength, no decay: the worst conditioned chunk."""
    x = delta_inputs(10, 150, 1, 1, 1, 64, 16, dtype, False)
    key = x["k"][:1].float()
    x["k"] = (key / key.norm()).expand(150, 1, 64).to(x["k"].dtype).contiguous()
    x["gate"].zero_()
    x["beta"].fill_(1.0)
    o, s, want_o, want_s = run_delta(x, [150], ragged=False)
    close(o, want_o, dtype == "bf16")
    close(s, want_s)


@pytest.mark.parametrize("what", ["q", "k", "v", "gate", "beta", "state"])
@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("length,token", [(8, 3), (200, 70), (200, 64), (200, 127)])
def test_delta_rule_bad_values_reach_nothing_before_them(length, token, value, what):
    """A NaN or an infinity of one sequence leaves its other heads, its columns that it does not meet, the outputs before
    it, and the other sequences bit for bit."""
    torch, ops = torch_ops()
    x = delta_inputs(12, 2 * length, 2, 2, 2, 64, 32, "f32", False)
    d = {n: None if a is None else a.cuda() for n, a in x.items()}
    args = lambda: (d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"])
    o, s = ops.delta_rule(*args())
    at = {"q": (token, 1, 5), "k": (token, 1, 5), "v": (token, 1, 5), "gate": (token, 1), "beta": (token, 1), "state": (0, 1, 7, 5)}[what]
    d[what][at] = value
    p, t = ops.delta_rule(*args())
    assert torch.equal(p[:, 0], o[:, 0]) and torch.equal(t[:, 0], s[:, 0])
    assert torch.equal(p[length:], o[length:]) and torch.equal(t[1], s[1])
    if what in ("v", "state"):  # one column
        rest = [c for c in range(32) if c != 5]
        assert torch.equal(p[:, :, rest], o[:, :, rest]) and torch.equal(t[..., rest], s[..., rest])
    if what != "state":
        assert torch.equal(p[:token], o[:token])
    if what == "q":
        assert torch.equal(t, s) and torch.equal(p[token + 1:], o[token + 1:]) and not torch.isfinite(p[token, 1]).any()
    elif what != "gate" or np.isnan(value):
        assert not torch.isfinite(t[0, 1, :, 5]).all()


@pytest.mark.parametrize("what", ["q", "k", "v", "gate", "beta", "state"])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("dtype,dk,dv", [("bf16", 64, 32), ("bf16", 128, 72), ("bf16", 37, 51), ("bf16", 200, 20), ("f32", 96, 40), ("f32", 200, 20)])
def test_delta_rule_bad_values_in_chunks(dtype, dk, dv, value, what):
    """As above for every kernel of the chunks: vectors and single values, keys in halves; tokens in both halves of a chunk, on its
    ends, in a last chunk that is not whole, in a sequence that is one chunk; segments of a long sequence."""
    torch, ops = torch_ops()
    for length, tokens in ((200, [0, 31, 32, 63, 64, 150, 198]), (20, [13]), (3000, [1300])):
        x = delta_inputs(24, 2 * length, 2, 2, 2, dk, dv, dtype, False)
        d = {n: None if a is None else a.cuda() for n, a in x.items()}
        call = lambda: ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"])
        o, s = call()
        for token in tokens:
            at = {"q": (token, 1, 5), "k": (token, 1, 5), "v": (token, 1, 5), "gate": (token, 1), "beta": (token, 1), "state": (0, 1, 7, 5)}[what]
            keep = d[what][at].clone()
            d[what][at] = value
            p, t = call()
            d[what][at] = keep
            where = (length, token)
            assert torch.equal(p[:, 0], o[:, 0]) and torch.equal(t[:, 0], s[:, 0]), where
            assert torch.equal(p[length:], o[length:]) and torch.equal(t[1], s[1]), where
            if what in ("v", "state"):  # one column
                rest = [c for c in range(dv) if c != 5]
                assert torch.equal(p[:, :, rest], o[:, :, rest]) and torch.equal(t[..., rest], s[..., rest]), where
            if what != "state":
                assert torch.equal(p[:token], o[:token]), where
            if what == "q":
                assert torch.equal(t, s) and torch.equal(p[token + 1:], o[token + 1:]) and not torch.isfinite(p[token, 1]).any(), where
            elif what != "gate" or np.isnan(value):
                assert not torch.isfinite(t[0, 1, :, 5]).any() and not torch.isfinite(p[token if what != "state" else 0:length, 1, 5]).any(), where
            if what == "gate" and value == -np.inf:  # forgets what was
                assert torch.isfinite(p).all() and torch.isfinite(t).all(), where


@pytest.mark.parametrize("dtype,dk,dv", [("bf16", 64, 16), ("bf16", 128, 40), ("bf16", 37, 51), ("bf16", 144, 16), ("f32", 128, 72), ("f32", 37, 51)])
@pytest.mark.parametrize("length", [9, 200, 3000])
def test_delta_rule_decays_in_chunks(length, dtype, dk, dv):
    """No decay, strong decay, a decay that forgets everything and tokens that do nothing, in both halves of a chunk."""
    x = delta_inputs(25, 2 * length, 2, 1, 2, dk, dv, dtype, False)
    x["gate"][::3] = 0.0
    for first in range(4, 2 * length, 37):
        x["gate"][first] = -np.inf
        x["gate"][first + 1:first + 2, 1] = -3e38
        x["gate"][first + 3:first + 4] = -90.0
    x["beta"][::4] = 0.0
    x["beta"][1::4] = 1.0
    o, s, want_o, want_s = run_delta(x, [length] * 2, ragged=False)
    close(o, want_o, dtype == "bf16")
    close(s, want_s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", ["q", "k"])
@pytest.mark.parametrize("length,token", [(1, 0), (5, 3), (200, 0), (200, 70), (200, 199)])
def test_delta_rule_norms_beyond_fp32(length, token, what, dtype):
    """A query or a key whose sum of squares is beyond fp32 counts as infinite: NaN, not a vector of zeros."""
    torch, ops = torch_ops()
    x = delta_inputs(23, 2 * length, 2, 2, 2, 64, 32, dtype, True)
    d = {n: a.cuda() for n, a in x.items()}
    call = lambda: ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], normalize=True, a_scale=d["a_scale"], dt_bias=d["dt_bias"])
    o, s = call()
    d[what][token, 1, 5] = 3e19
    p, t = call()
    assert torch.equal(p[:, 0], o[:, 0]) and torch.equal(p[:token], o[:token]) and torch.equal(p[length:], o[length:])
    assert torch.equal(t[:, 0], s[:, 0]) and torch.equal(t[1], s[1])
    assert p[token, 1].isnan().all()
    if what == "q":
        assert torch.equal(t, s) and torch.equal(p[token + 1:], o[token + 1:])
    else:
        assert p[token:length, 1].isnan().all() and t[0, 1].isnan().all()


def test_delta_rule_offsets_out_of_order_stay_inside():
    """Offsets that are not ascending or not in range are empty sequences or cut off: nothing outside is read or
    written, and the sequences that are well formed keep their values."""
    torch, ops = torch_ops()
    x = delta_inputs(13, 300, 4, 1, 1, 64, 32, "f32", False)
    d = {n: None if a is None else a.cuda() for n, a in x.items()}
    bad = torch.tensor([0, 100, 50, 2000000000, -5], dtype=torch.int32).cuda()
    out = torch.full((300, 1, 32), 5.0, device="cuda")
    o, s = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], seq_offsets=bad, out=out)
    torch.cuda.synchronize()
    assert torch.equal(s[1], d["state"][1]) and torch.equal(s[3], d["state"][3])


@pytest.mark.parametrize("dtype,dk", [("f32", 64), ("bf16", 136)])
@pytest.mark.parametrize("kind", ["fives", "mixed", "random", "few", "fives and a long one"])
def test_delta_rule_chunks_of_many_sequences(kind, dtype, dk):
    """Sequences just long enough for a chunk of their own, packed as closely as they can be."""
    rng = np.random.default_rng(4)
    lens = {"fives": [5] * 70, "mixed": [5, 4, 5, 1, 64, 0, 65, 5, 5, 63, 4, 4, 4, 128, 5] * 3, "random": rng.integers(0, 14, 120).tolist(),
            "few": [5, 600, 5, 0, 700], "fives and a long one": [5] * 70 + [1200] + [5] * 20}[kind]
    x = delta_inputs(19, sum(lens), len(lens), 1, 2, dk, 24, dtype, True)
    o, s, want_o, want_s = run_delta(x, lens)
    close(o, want_o, dtype == "bf16")
    close(s, want_s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hk,hv,dk,dv", [(1, 2, 64, 32), (1, 1, 136, 20)])
@pytest.mark.parametrize("at", [[100, 230, 300], [64, 70, 400], [200] + list(range(200, 1000, 11)), [900, 50, 200, 203, 1000], [0, 70, 2000000000, 2000000000],
                                [-5, 70, 1000], [500, 500, 500, 100, 400, 900, 0]], ids=lambda at: f"{at[0]}-{at[1]}-{len(at) - 1}")
def test_delta_rule_offsets_that_start_anywhere(at, hk, hv, dk, dv, dtype):
    """Offsets of a part of the tokens (a slice of more offsets), a descending pair in front, values out of range: every sequence is
    right, and tokens of none keep what stands in the output."""
    torch, ops = torch_ops()
    n = 1000
    x = delta_inputs(18 + len(at), n, len(at) - 1, hk, hv, dk, dv, dtype, True)
    d = {name: a.cuda() for name, a in x.items()}
    out = torch.full((n, hv, dv), 5.0, dtype=d["v"].dtype, device="cuda")
    o, s = ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], seq_offsets=torch.tensor(at, dtype=torch.int32).cuda(), out=out,
                          normalize=True, a_scale=d["a_scale"], dt_bias=d["dt_bias"])
    inside = np.clip(at, 0, n)
    spans = [(int(a), max(int(b - a), 0)) for a, b in zip(inside, inside[1:])]
    c = numbers(x)
    want_o, want_s = ops_ref.delta_rule(c["q"], c["k"], c["v"], c["gate"], c["beta"], c["state"], spans, dk ** -0.5, True, c["a_scale"], c["dt_bias"])
    some = np.zeros(n, bool)
    for first, length in spans:
        some[first:first + length] = True
    close(o[torch.from_numpy(some)], want_o[some], dtype == "bf16")
    assert (o[torch.from_numpy(~some)] == 5.0).all()
    close(s, want_s)


@pytest.mark.parametrize("length", [1, 100])
def test_delta_rule_on_another_stream_and_in_a_graph(length):
    torch, ops = torch_ops()
    x = delta_inputs(14, 4 * length, 4, 2, 4, 64, 64, "bf16", True)
    d = {n: a.cuda() for n, a in x.items()}
    kw = dict(normalize=True, a_scale=d["a_scale"], dt_bias=d["dt_bias"])
    args = (d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"])
    want = ops.delta_rule(*args, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ops.delta_rule(*args, **kw)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = ops.delta_rule(*args, **kw)
    for turn in range(4):
        d["v"].copy_(x["v"].cuda() * (turn + 1))
        graph.replay()
        torch.cuda.synchronize()
        eager = ops.delta_rule(*args, **kw)
        torch.cuda.synchronize()
        assert torch.equal(captured[0], eager[0]) and torch.equal(captured[1], eager[1])


# ------------------------------------------------------------------- norms

def norm_case(seed, rows, dim, group, dtype, gate_act, without=()):
    import torch
    g = torch.Generator().manual_seed(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    normal = lambda *s: torch.randn(*s, generator=g)
    x = dict(x=(2 * normal(rows, dim)).to(t), branch=(normal(rows, dim) + 0.5).to(t), gate=normal(rows, dim).to(t) if gate_act != "none" else None,
             post_weight=1 + 0.1 * normal(group), post_bias=normal(group), res_scale=normal(dim), pre_weight=1 + 0.1 * normal(dim), pre_bias=normal(dim))
    return {n: None if n in without else a for n, a in x.items()}


def run_norm(x, **kw):
    torch, ops = torch_ops()
    d = {n: None if a is None else a.cuda() for n, a in x.items()}
    r = ops.block_norm(**d, **kw)
    torch.cuda.synchronize()
    ref = {n: a for n, a in kw.items() if n not in ("want", "x_out", "h_out")}
    return r, ops_ref.block_norm(**numbers(x), **ref)


def check_quantised(q, h, dim):
    """Rows of 8-bit integers against h in 64 bits: rounding may go the other way where 127 h / m is within 2^-10 of
    a half (the operator's h is right to about 2^-20 of the largest, 127 / m multiplies that)."""
    stored, scale = q.q.cpu().numpy(), q.scale.cpu().numpy().astype(np.float64)
    assert stored.shape[1] % 128 == 0 and (stored[:, dim:] == 0).all()
    m = np.abs(h).max(axis=1)
    np.testing.assert_allclose(scale, m / 127, rtol=2.0 ** -18, atol=1e-37)
    exact = h * np.where(m > 0, 127 / np.maximum(m, 1e-300), 0)[:, None]
    off = np.abs(stored[:, :dim] - exact)
    assert off.max() <= 0.5 + 2.0 ** -10
    assert np.abs(stored[:, :dim]).max(axis=1)[m > 0].min(initial=127) == 127


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("rows,dim,group,gate", [
    (1, 1, 1, "none"), (3, 8, 8, "silu"), (5, 513, 513, "sigmoid"), (2, 512, 64, "silu"), (7, 336, 112, "silu"), (4, 111, 37, "sigmoid"),
    (2050, 96, 32, "silu"), (3, 2048, 2048, "sigmoid"), (3, 2048, 128, "silu"), (2, 4100, 4100, "none"), (2, 4096, 256, "silu"),
    (2, 8192, 8192, "silu"), (2, 8192, 512, "none"), (2, 16384, 16384, "silu"), (2, 16384, 256, "sigmoid"), (3, 9001, 9001, "none")])
def test_block_norm(rows, dim, group, gate, kind, dtype):
    x = norm_case(rows + dim, rows, dim, group, dtype, gate)
    r, (want_x, want_h) = run_norm(x, gate_act=gate, group=group, kind=kind, pre_norm=True, want="xhq")
    close(r.x, want_x, dtype == "bf16")
    close(r.h, want_h, dtype == "bf16")
    check_quantised(r.q, want_h, dim)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_block_norm_every_operand_may_be_left_out(dtype):
    names = ["x", "branch", "gate", "post_weight", "post_bias", "res_scale", "pre_weight", "pre_bias"]
    of_branch = {"gate", "post_weight", "post_bias", "res_scale"}
    for name in names:
        gone = {name} | (of_branch if name == "branch" else set())
        gate = "none" if "gate" in gone else "silu"
        x = norm_case(3, 6, 200, 40 if name != "x" else 200, dtype, gate, gone)
        r, (want_x, want_h) = run_norm(x, gate_act=gate, group=40 if name not in ("x",) else 200, pre_norm=True, want="xhq")
        close(r.x, want_x, dtype == "bf16")
        close(r.h, want_h, dtype == "bf16")
        check_quantised(r.q, want_h, 200)
    x = norm_case(4, 6, 200, 200, dtype, "none", ("pre_weight", "pre_bias"))
    r, (want_x, _) = run_norm(x, want="x")
    close(r.x, want_x, dtype == "bf16")
    assert r.h is None and r.q is None


def test_block_norm_strides_and_in_place():
    torch, ops = torch_ops()
    for pad in (0, 3):
        x = norm_case(5, 20, 264, 264, "bf16", "sigmoid")
        d = {n: a.cuda() for n, a in x.items()}
        want = ops.block_norm(**d, gate_act="sigmoid", want="xh")
        wide = torch.cat([d["x"][:, :pad], d["x"], d["branch"], d["gate"]], dim=1)
        views = {n: wide[:, pad + i * 264:pad + (i + 1) * 264] for i, n in enumerate(("x", "branch", "gate"))}
        got = ops.block_norm(**{**d, **views}, gate_act="sigmoid", want="xh", x_out=views["x"])
        assert torch.equal(got.x, want.x) and torch.equal(got.h, want.h) and torch.equal(wide[:, pad:pad + 264], want.x)
        assert torch.equal(wide[:, pad + 264:pad + 528], d["branch"])


def test_block_norm_of_more_rows_than_one_launch_takes():
    """2^26 rows and some: with 64 threads to a row more than the 2^32 threads that a launch can have."""
    torch, ops = torch_ops()
    n, dim = (1 << 26) + 37, 8
    x = torch.randn(1 << 20, dim, device="cuda").bfloat16().repeat(65, 1)[:n]
    x[-37:] *= 3
    w = torch.rand(dim, device="cuda") + 0.5
    got = ops.block_norm(x, pre_norm=True, pre_weight=w, want="h").h
    part = ops.block_norm(x[:1 << 20].contiguous(), pre_norm=True, pre_weight=w, want="h").h
    for i in range(64):
        assert torch.equal(got[i << 20:(i + 1) << 20], part), i
    close(got[-37:], ops_ref.block_norm(x[-37:].float().cpu().numpy(), pre_norm=True, pre_weight=w.cpu().numpy())[1], True)


def test_block_norm_rows_of_zeros_and_bad_values():
    torch, ops = torch_ops()
    x = torch.randn(6, 300, generator=torch.Generator().manual_seed(1))
    x[1] = 0.0
    x[2, 7] = np.nan
    x[3, 8] = -np.inf
    x[4] *= 1e-42
    r = ops.block_norm(x.cuda(), pre_norm=True, want="hq")
    h, s, q = r.h.cpu(), r.q.scale.cpu(), r.q.q.cpu()
    assert (h[1] == 0).all() and s[1] == 0 and (q[1] == 0).all()
    assert h[2].isnan().all() and s[2].isnan() and s[3].isnan() and (q[2:4] == 0).all()
    assert torch.isfinite(h[[0, 1, 4, 5]]).all() and torch.isfinite(s[[0, 1, 4, 5]]).all()
    r = ops.quantize_rows(x.cuda())
    q, s = ops_ref.quantize_rows(x.numpy())
    assert np.array_equal(r.q.cpu().numpy()[:, :300], q) and np.array_equal(r.scale.cpu().numpy(), s, equal_nan=True)


# ------------------------------------------------------------------- products in 8 bits

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k,act,bias", [
    (1, 1, 1, "none", False), (1, 17, 128, "none", True), (2, 300, 129, "relu", True), (16, 1536, 512, "none", True), (15, 64, 4000, "tanh", True),
    (17, 777, 1000, "sigmoid", True), (33, 40, 64, "none", False), (64, 1024, 2048, "none", True), (100, 130, 300, "none", True), (257, 513, 640, "relu", False),
    (1000, 260, 128, "none", True), (511, 1024, 1100, "tanh", False), (600, 2049, 200, "none", True), (3, 8, 131072, "none", False),
    (300, 300, 20000, "none", False)])
def test_quant_matmul(m, n, k, act, bias, dtype):
    torch, ops = torch_ops()
    g = torch.Generator().manual_seed(m + n + k)
    x, w = torch.randn(m, k, generator=g), torch.randn(n, k, generator=g) / k ** 0.5
    b = torch.randn(n, generator=g) if bias else None
    want_a, want_b = ops_ref.quantize_rows(x.numpy()), ops_ref.quantize_rows(w.numpy())
    if k <= 16384:
        qa, qb = ops.quantize_rows(x.cuda()), ops.quantize_rows(w.cuda())
    else:  # (longer rows than the operator quantises)
        qa, qb = (ops.QuantRows(torch.nn.functional.pad(torch.from_numpy(q), (0, -k % 128)).cuda(), torch.from_numpy(s).cuda(), k)
                  for q, s in (want_a, want_b))
    assert np.array_equal(qa.q.cpu().numpy()[:, :k], want_a[0]) and np.array_equal(qb.q.cpu().numpy()[:, :k], want_b[0])
    assert np.array_equal(qa.scale.cpu().numpy(), want_a[1]) and np.array_equal(qb.scale.cpu().numpy(), want_b[1])
    y = ops.quant_matmul(qa, qb, bias=None if b is None else b.cuda(), act=act, out_dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    close(y, ops_ref.quant_matmul(*want_a, *want_b, None if b is None else b.numpy(), act), dtype == "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k,act,bias", [
    (2500, 2600, 200, "tanh", True), (2433, 2569, 129, "none", False), (2500, 2600, 1, "relu", True),  # 128 x 128
    (3500, 3600, 300, "none", True), (3329, 3585, 1153, "sigmoid", False),  # 256 x 256
    (50000, 33, 256, "relu", True), (40, 50000, 256, "none", True), (30000, 200, 128, "none", True)])  # narrow: 64 x 64, 128 x 128
def test_quant_matmul_in_large_tiles(m, n, k, act, bias, dtype):
    """From 384 tiles of 128 x 128 and 193 of 256 x 256 on; tiles that the ends cut, one row and column beyond a tile."""
    torch, ops = torch_ops()
    g = torch.Generator().manual_seed(m + n + k)
    x, w = torch.randn(m, k, generator=g), torch.randn(n, k, generator=g) / k ** 0.5
    b = torch.randn(n, generator=g) if bias else None
    want_a, want_b = ops_ref.quantize_rows(x.numpy()), ops_ref.quantize_rows(w.numpy())
    qa, qb = ops.quantize_rows(x.cuda()), ops.quantize_rows(w.cuda())
    out = torch.full((m, n + 8), 9.0, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    y = ops.quant_matmul(qa, qb, bias=None if b is None else b.cuda(), act=act, out=out[:, :n])
    close(y, ops_ref.quant_matmul(*want_a, *want_b, None if b is None else b.numpy(), act), dtype == "bf16")
    assert (out[:, n:] == 9.0).all()


@pytest.mark.parametrize("m", [2, 40, 300])
def test_quant_matmul_sums_are_exact(m):
    """The largest sums that 32 bits hold, and sums that cancel to 1."""
    torch, ops = torch_ops()
    k, n = 131072, 20
    a = torch.full((m, k), 127, dtype=torch.int8)
    b = torch.full((n, k), 127, dtype=torch.int8)
    b[1] = -127
    b[2, ::2] = -127
    b[2, 0] = -126
    one_m, one_n = torch.ones(m, device="cuda"), torch.ones(n, device="cuda")
    y = ops.quant_matmul(ops.QuantRows(a.cuda(), one_m, k), ops.QuantRows(b.cuda(), one_n, k))
    want = (a[:1].double() @ b.double().T)[0]
    assert torch.equal(y.cpu(), want.float().expand(m, n)) and want[2] == 127


def test_quant_matmul_strides_and_bad_scales():
    torch, ops = torch_ops()
    g = torch.Generator().manual_seed(2)
    x = torch.randn(40, 256, generator=g)
    x[3, 5] = np.nan
    w = ops.quantize_rows(torch.randn(70, 256, generator=g).cuda())
    qa = ops.quantize_rows(x.cuda())
    want = ops.quant_matmul(qa, w)
    assert want[3].isnan().all() and torch.isfinite(want[[i for i in range(40) if i != 3]]).all()
    wide = torch.full((40, 512), 99, dtype=torch.int8, device="cuda")
    wide[:, :256] = qa.q
    out = torch.full((40, 80), 7.0, device="cuda")
    got = ops.quant_matmul(ops.QuantRows(wide[:, :256], qa.scale, 256), w, out=out[:, 5:75])
    assert torch.equal(got.nan_to_num(), want.nan_to_num()) and (out[:, :5] == 7).all() and (out[:, 75:] == 7).all()


@pytest.mark.parametrize("m", [1, 16, 500])
def test_quant_matmul_in_a_graph(m):
    torch, ops = torch_ops()
    x = torch.randn(m, 3000, device="cuda")
    w = ops.quantize_rows(torch.randn(200, 3000, device="cuda"))
    ops.quant_matmul(ops.quantize_rows(x), w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ops.quant_matmul(ops.quantize_rows(x), w)
    for _ in range(4):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        want = ops.quant_matmul(ops.quantize_rows(x), w)
        torch.cuda.synchronize()
        assert torch.equal(y, want)


# ------------------------------------------------------------------- refusals

def test_refusals_leave_the_device_usable():
    torch, ops = torch_ops()
    x = delta_inputs(15, 8, 1, 1, 1, 16, 16, "f32", False)
    d = {n: None if a is None else a.cuda() for n, a in x.items()}
    good = (d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"])
    for i, bad, status in ((0, d["q"].bfloat16(), ev.ERR_INVALID_ARG), (1, d["k"][:4], ev.ERR_SHAPE), (2, d["v"].cpu(), ev.ERR_INVALID_ARG),
                           (3, d["gate"][:, :0], ev.ERR_SHAPE), (5, d["state"].double(), ev.ERR_INVALID_ARG),
                           (5, d["state"].transpose(2, 3)[..., ::2], ev.ERR_SHAPE), (0, d["q"].double(), ev.ERR_INVALID_ARG)):
        with pytest.raises(ev.EvConvError) as e:
            ops.delta_rule(*good[:i], bad, *good[i + 1:])
        assert e.value.status == status, (i, e.value)
    with pytest.raises(ev.EvConvError):
        ops.delta_rule(*good, n_seq=3)
    with pytest.raises(ev.EvConvError):
        ops.delta_rule(*good, a_scale=torch.ones(1, device="cuda"))
    with pytest.raises(ev.EvConvError):
        ops.block_norm(d["q"][:, 0], want="y")
    with pytest.raises(ev.EvConvError):
        ops.block_norm(d["q"][:, 0], d["q"][:, 0], group=5)
    with pytest.raises(ev.EvConvError):
        ops.quant_matmul(ops.QuantRows(torch.zeros(2, 100, dtype=torch.int8, device="cuda"), torch.ones(2, device="cuda"), 100),
                         ops.QuantRows(torch.zeros(2, 128, dtype=torch.int8, device="cuda"), torch.ones(2, device="cuda"), 100))
    o, _ = ops.delta_rule(*good)
    assert torch.isfinite(o).all()


def test_tensors_that_want_a_gradient_are_refused():
    """These operators have none, and their outputs would be detached without a word; under no_grad nothing is lost."""
    torch, ops = torch_ops()
    x = delta_inputs(27, 8, 1, 1, 1, 16, 16, "f32", True)
    d = {n: a.cuda() for n, a in x.items()}
    delta = lambda d: ops.delta_rule(d["q"], d["k"], d["v"], d["gate"], d["beta"], d["state"], normalize=True, a_scale=d["a_scale"], dt_bias=d["dt_bias"])[0]
    n = {i: a.cuda() for i, a in norm_case(6, 4, 32, 32, "f32", "silu").items()}
    norm = lambda n: ops.block_norm(**n).x
    w = ops.quantize_rows(torch.randn(8, 32, device="cuda"))
    product = lambda b: ops.quant_matmul(w, w, bias=b["bias"])
    rows = lambda x: ops.quantize_rows(x["x"]).scale
    for call, given in ((delta, d), (norm, n), (product, {"bias": torch.randn(8, device="cuda")}), (rows, {"x": n["x"]})):
        want = call(given)
        for name in given:
            some = {**given, name: given[name].clone().requires_grad_()}
            with pytest.raises(ev.EvConvError) as e:
                call(some)
            assert e.value.status == ev.ERR_INVALID_ARG and "gradient" in str(e.value), name
            with torch.no_grad():
                got = call(some)
            assert torch.equal(got, want) and not got.requires_grad
