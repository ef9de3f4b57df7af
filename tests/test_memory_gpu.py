"""The memory behind an incremental net (memory.py) on the GPU, against its formulas in 64 bits.

Tolerance, set beforehand: a value that is an ulp off can round to the next 8-bit integer, a step of about 0.03 of a row's rms,
and whatever a step moves makes others round differently further on; at worst every quantisation adds the noise of one more
rounding, 0.03 / sqrt(6) of the rms.  Seven in a row (two layers and the head) are 3 % of the norm; twice that, 2^-4, is
allowed for what the layers gain.  A wrong operand, order or state is off by the norm itself."""
import numpy as np
import pytest

import ops_ref

pytestmark = pytest.mark.gpu


def reference(memory, x, states, spans):
    """(outputs, states) of features x; spans: (first, windows) of every stream of `states`."""
    to, hk, hv, dk, dv = memory.columns, memory.heads_k, memory.heads_v, memory.d_k, memory.d_v
    product = lambda a, w, **kw: ops_ref.quant_matmul(*ops_ref.quantize_rows(a), *ops_ref.quantize_rows(w), **kw)
    n, states = len(x), [np.array(s, np.float64) for s in states]
    _, h = ops_ref.block_norm(x, pre_norm=True, pre_weight=memory.weights[0]["pre_norm"])
    for i, w in enumerate(memory.weights[:-1]):
        p = product(h, w["w_in"])
        q, k, v, z, a, b = (p[:, to[j]:to[j + 1]] for j in range(6))
        o, states[i] = ops_ref.delta_rule(q.reshape(n, hk, dk), k.reshape(n, hk, dk), v.reshape(n, hv, dv), a, b, states[i], spans,
                                          dk ** -0.5, normalize=True, a_scale=w["a_scale"], dt_bias=w["dt_bias"])
        _, g = ops_ref.block_norm(None, o.reshape(n, -1), z, post_weight=w["head_norm"], gate_act="silu", group=dv)
        following = memory.weights[i + 1]
        x, h = ops_ref.block_norm(x, product(g, w["w_out"]), post_weight=w["post_norm"], res_scale=w["res_scale"], pre_norm=True,
                                  pre_weight=following["pre_norm"] if "pre_norm" in following else following["norm"])
    return product(h, memory.weights[-1]["head"], bias=memory.weights[-1]["bias"]), states


def near(got, want):
    got = got.detach().double().cpu().numpy()
    assert got.shape == np.shape(want) and np.isfinite(got).all()
    assert np.linalg.norm(got - want) <= 2.0 ** -4 * np.linalg.norm(want), np.linalg.norm(got - want) / np.linalg.norm(want)


def bf16():
    import torch
    return torch.bfloat16


def make(**kw):
    import torch
    from paper_2303_04670_amd.memory import Memory
    torch.manual_seed(1)
    return torch, Memory(**{**dict(dim=96, n_streams=5, n_out=11, dtype=torch.float32, seed=3), **kw})


@pytest.mark.parametrize("sizes", [{}, dict(dim=128, heads_k=1, heads_v=3, d_k=40, d_v=24), dict(dim=101, layers=1, heads_v=2, d_k=160, d_v=16)])
def test_windows_one_by_one_and_at_once(sizes):
    torch, memory = make(**sizes)
    _, other = make(**sizes)
    windows, dim = 12, memory.dim
    x = torch.randn(5, windows, dim, device="cuda")
    one = torch.stack([memory(x[:, i].contiguous()) for i in range(windows)], dim=1)
    offsets = torch.arange(6, dtype=torch.int32, device="cuda") * windows
    everything = other(x.view(-1, dim), seq_offsets=offsets)
    zeros = [np.zeros(s.shape) for s in memory.states]
    want, states = reference(memory, x.cpu().numpy().reshape(-1, dim), zeros, [(i * windows, windows) for i in range(5)])
    near(one.view(-1, 11), want)
    near(everything, want)
    for got, also, s in zip(memory.states, other.states, states):
        near(got, s)
        near(also, s)


def test_ragged_windows_in_bf16_continue_their_streams():
    torch, memory = make(dtype=bf16())
    lens, slots = [30, 0, 1, 75], [4, 2, 0, 1]
    n = sum(lens)
    x = torch.randn(n, 96, device="cuda").bfloat16()
    for s in memory.states:
        s.normal_()
    before = [s.clone() for s in memory.states]
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    got = memory(x, slots=torch.tensor(slots, dtype=torch.int32, device="cuda"), seq_offsets=offsets)
    first = np.concatenate([[0], np.cumsum(lens)])
    want, states = reference(memory, x.float().cpu().numpy(), [s.cpu().numpy()[slots] for s in before],
                             [(int(first[i]), lens[i]) for i in range(4)])
    near(got, want)
    for s, b, w in zip(memory.states, before, states):
        near(s[slots], w)
        assert torch.equal(s[3], b[3]) and torch.equal(s[2], b[2])  # a stream that is not named, one without windows


def test_streams_are_independent():
    torch, memory = make()
    _, other = make()
    order = torch.tensor([3, 0, 4], dtype=torch.int32, device="cuda")
    for _ in range(3):
        x = torch.randn(5, 96, device="cuda")
        whole = memory(x)
        assert torch.equal(other(x[order.long()], slots=order), whole[order.long()])
    for a, b in zip(memory.states, other.states):
        assert torch.equal(a[order.long()], b[order.long()]) and not b[[1, 2]].any()
    memory.forget([3])
    assert not memory.states[0][3].any() and memory.states[0][4].any()


@pytest.mark.parametrize("how", ["type", "width", "dimensions", "slots"])
def test_a_refused_window_leaves_the_states(how):
    torch, memory = make()
    from paper_2303_04670_amd import evconv as ev
    x = torch.randn(5, 96, device="cuda")
    memory(x)
    before = [s.clone() for s in memory.states]
    bad, slots = {"type": (x.bfloat16(), None), "width": (x[:, :95], None), "dimensions": (x[0], None),
                  "slots": (x, torch.arange(4, dtype=torch.int32, device="cuda"))}[how]
    with pytest.raises(ev.EvConvError):
        memory(bad, slots=slots)
    for s, b in zip(memory.states, before):
        assert torch.equal(s, b)


@pytest.mark.parametrize("on", ["cuda", "cpu", "list"])
def test_forgetting_takes_slots_as_a_window_does(on):
    """Negative ones are no stream's."""
    torch, memory = make()
    memory(torch.randn(5, 96, device="cuda"))
    before = [s.clone() for s in memory.states]
    slots = [3, -1, 0]
    memory.forget(slots if on == "list" else torch.tensor(slots, dtype=torch.int32, device=on))
    for s, b in zip(memory.states, before):
        assert not s[[0, 3]].any() and torch.equal(s[[1, 2, 4]], b[[1, 2, 4]]) and b.flatten(1).any(dim=1).all()
    memory.forget()
    assert not any(s.any() for s in memory.states)


def test_a_window_in_a_graph():
    torch, memory = make()
    _, other = make()
    x = torch.randn(5, 96, device="cuda")
    memory(x)
    other(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = memory(x)
    for _ in range(4):
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, other(x))
        torch.cuda.synchronize()


def test_behind_a_net():
    torch, memory = make(dim=32, n_streams=2)
    from paper_2303_04670_amd import evconv as ev
    from paper_2303_04670_amd import workloads as wl
    net = ev.EvConvNet(wl.net_resnet18(h=64, w=64, width=16, n_classes=32), n_streams=2)
    frames = [np.stack(f) for f in zip(*(list(wl.stream_histogram(7 + s, 64, 64, 4)) for s in range(2)))]
    seen, answers = [], []
    for i, frame in enumerate(frames):
        frame = torch.from_numpy(frame).cuda()
        net.reset(frame) if i == 0 else net.step_frame(frame)
        features = torch.stack([net.outputs(s)[0]["y"].reshape(-1) for s in range(2)])
        answers.append(memory(features))
        seen.append(features.cpu().numpy())
    torch.cuda.synchronize()
    net.destroy()
    n = len(frames)
    want, _ = reference(memory, np.stack(seen, axis=1).reshape(-1, 32), [np.zeros(s.shape) for s in memory.states], [(0, n), (n, n)])
    near(torch.stack(answers, dim=1).view(-1, 11), want)
