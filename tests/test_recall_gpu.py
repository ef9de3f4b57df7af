"""Layers of the memory that look back into a paged cache (memory.py), against their formulas in 64 bits.

Tolerance: that of test_memory_gpu.py, 2^-4 of the norm, whose reasons hold here too: 8-bit rows that round differently are what there is
to be off by, and a value of 4 bits that rounds to its other neighbour counts as one of them."""
import numpy as np
import pytest

import ops_ref

pytestmark = pytest.mark.gpu


def make(**kw):
    import torch
    from paper_2303_04670_amd.memory import Memory
    torch.manual_seed(1)
    return torch, Memory(**{**dict(dim=96, n_streams=4, n_out=11, dtype=torch.float32, seed=3, recall=(0, 1), recall_windows=200, longest=300), **kw})


def held(x, kind):
    import torch
    if kind == "bf16":
        return torch.from_numpy(np.asarray(x, np.float32)).bfloat16().double().numpy()
    return ops_ref.fp4_values(*ops_ref.fp4_rows(x))


def reference(memory, x, spans, kind="fp4", pages=None):
    """Outputs of whole streams' features; spans: (first, windows)."""
    hk, hv, d = memory.heads_k, memory.heads_v, memory.d_v
    product = lambda a, w, **kw: ops_ref.quant_matmul(*ops_ref.quantize_rows(a), *ops_ref.quantize_rows(w), **kw)
    _, h = ops_ref.block_norm(x, pre_norm=True, pre_weight=memory.weights[0]["pre_norm"])
    freqs = memory.freqs.cpu().numpy()
    for i, w in enumerate(memory.weights[:-1]):
        p = product(h, w["w_in"])
        n, o = len(p), np.zeros((len(p), hv, d))
        cut = np.cumsum([0, hv * d, hk * d, hk * d, hv * d])
        q, k, v, z = (p[:, a:b] for a, b in zip(cut, cut[1:]))
        for first, count in spans:
            at, t = slice(first, first + count), np.arange(count)
            turn = lambda y, heads, norm: ops_ref.head_rows(y[at].reshape(count, heads, d), w[norm], 1e-6, freqs, "halves", t)
            qs, raw = turn(q, hv, "q_norm"), turn(k, hk, "k_norm")
            ks, vs = held(raw, kind), held(v[at].reshape(count, hk, d), kind)
            for head in range(hv):
                g = head // (hv // hk)
                seen = (t <= t[:, None]) & (t > t[:, None] - memory.recall_windows)
                if pages:
                    seen = np.zeros((count, count), bool)
                    low = held(raw, "bf16")[:, g]
                    for j in range(count):
                        score = []
                        for page in range(j // 64 + 1):
                            mine = low[page * 64:min(page * 64 + 64, count)]
                            each = qs[j, g * (hv // hk):(g + 1) * (hv // hk)]
                            score.append(np.maximum(each * mine.min(0), each * mine.max(0)).sum(-1).max())
                        for page in ops_ref.choose(np.float32(score), pages, 1, 1):
                            if page >= 0:
                                seen[j, page * 64:min(page * 64 + 64, j + 1)] = True
                o[at, head], _ = ops_ref.attend(qs[:, head], ks[:, g], vs[:, g], d ** -0.5, seen)
        _, g = ops_ref.block_norm(None, o.reshape(n, -1), z, post_weight=w["head_norm"], gate_act="silu", group=d)
        following = memory.weights[i + 1]
        x, h = ops_ref.block_norm(x, product(g, w["w_out"]), post_weight=w["post_norm"], res_scale=w["res_scale"], pre_norm=True,
                                  pre_weight=following["pre_norm"] if "pre_norm" in following else following["norm"])
    return product(h, memory.weights[-1]["head"], bias=memory.weights[-1]["bias"])


def near(got, want):
    got = got.detach().double().cpu().numpy()
    assert got.shape == np.shape(want) and np.isfinite(got).all()
    assert np.linalg.norm(got - want) <= 2.0 ** -4 * np.linalg.norm(want), np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("sizes", [{}, dict(recall_kind="bf16", d_v=40, heads_v=3, heads_k=1), dict(recall_windows=30), dict(recall_windows=256, recall_pages=3)])
def test_windows_one_by_one_and_at_once(sizes):
    torch, memory = make(**sizes)
    _, other = make(**sizes)
    lens = [230, 0, 1, 65]
    first = np.concatenate([[0], np.cumsum(lens)])
    x = torch.randn(sum(lens), 96, device="cuda")
    want = reference(memory, x.cpu().numpy(), [(int(a), n) for a, n in zip(first, lens)], sizes.get("recall_kind", "fp4"), sizes.get("recall_pages"))
    near(memory(x, seq_offsets=torch.tensor(first, dtype=torch.int32, device="cuda")), want)
    assert memory.past.tolist() == lens
    if sizes.get("recall_pages"):
        return  # (which pages are taken may hang on an 8-bit rounding)
    one = torch.zeros(sum(lens), 11, device="cuda")
    for i in range(max(lens)):
        live = [s for s in range(4) if lens[s] > i]
        rows = torch.tensor([int(first[s]) + i for s in live], device="cuda")
        one[rows] = other(x[rows], slots=torch.tensor(live, dtype=torch.int32, device="cuda"))
    near(one, want)
    assert other.past.tolist() == lens


def test_pages_go_round():
    """A stream that is longer than all its pages sees its last windows only."""
    torch, memory = make(recall_windows=64, longest=100, n_streams=2)
    assert memory.n_pages == 2 * 4
    x = torch.randn(2 * 500, 96, device="cuda")
    want = reference(memory, x.cpu().numpy(), [(0, 500), (500, 500)])
    got = []
    for at in range(0, 500, 50):
        rows = torch.cat([x[at:at + 50], x[500 + at:550 + at]])
        got.append(memory(rows, seq_offsets=torch.tensor([0, 50, 100], dtype=torch.int32, device="cuda")).view(2, 50, 11))
    near(torch.cat(got, dim=1).reshape(1000, 11), want)


def test_layers_of_both_kinds_forget_and_mind_their_streams():
    torch, memory = make(recall=(1,), layers=3)
    _, other = make(recall=(1,), layers=3)
    for i in range(5):
        x = torch.randn(4, 96, device="cuda")
        a, b = memory(x), other(x)
        assert torch.equal(a, b)
    memory.forget([2, -1])
    assert memory.past.tolist() == [5, 5, 0, 5]
    x = torch.randn(4, 96, device="cuda")
    a = memory(x)
    assert torch.equal(a[[0, 1, 3]], other(x)[[0, 1, 3]])
    _, fresh = make(recall=(1,), layers=3)
    near(a[2:3], fresh(x[2:3], slots=torch.tensor([2], dtype=torch.int32, device="cuda")).double().cpu().numpy())
    before = memory.past.tolist()
    memory(x[:1], slots=torch.tensor([-1], dtype=torch.int32, device="cuda"))
    assert memory.past.tolist() == before


def test_a_refused_window_leaves_everything():
    torch, memory = make()
    from paper_2303_04670_amd import evconv as ev
    x = torch.randn(4, 96, device="cuda")
    memory(x)
    state = [t.clone() for layer in memory.layers for t in layer.cache[:5] if t is not None] + [memory.past.clone()]
    offsets = torch.tensor([0, 301], dtype=torch.int32, device="cuda")
    for call in (lambda: memory(x.bfloat16()), lambda: memory(x[:, :95]), lambda: memory(x[:3]), lambda: memory(torch.zeros(301, 96, device="cuda"), seq_offsets=offsets),
                 lambda: memory(x, slots=torch.arange(3, dtype=torch.int32, device="cuda")), lambda: make(recall=(2,))):
        with pytest.raises(ev.EvConvError):
            call()
    for a, b in zip(state, [t for layer in memory.layers for t in layer.cache[:5] if t is not None] + [memory.past]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_a_window_in_a_graph():
    torch, memory = make(recall=(0,), dtype=__import__("torch").bfloat16)
    _, other = make(recall=(0,), dtype=torch.bfloat16)
    x = torch.randn(4, 96, device="cuda").bfloat16()
    memory(x)
    other(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = memory(x)
    for _ in range(70):
        x.normal_()
        graph.replay()
        assert torch.equal(y, other(x))
    torch.cuda.synchronize()
    assert memory.past.tolist() == other.past.tolist() == [71] * 4


@pytest.mark.parametrize("kind", ["fp4", "bf16"])
@pytest.mark.parametrize("how", ["pieces", "slots"])
def test_a_stream_that_goes_round_many_times(how, kind):
    """Pages go round every 256 windows here, again and again; what is seen stays the last 64 windows."""
    torch, memory = make(recall_windows=64, longest=100, n_streams=3, recall_kind=kind, lifetime=320)
    n, x = 1400, torch.randn(2 * 1400, 96, device="cuda")
    want = reference(memory, x.cpu().numpy(), [(0, n), (n, n)], kind)
    slots = torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    got, at = torch.empty(2, n, 11, device="cuda"), 0
    for step in [50, 1, 37, 1] * 100:  # (no step brings the round's end to the same place)
        step = min(step, n - at)
        if not step:
            break
        rows = torch.cat([x[at:at + step], x[n + at:n + at + step]])
        if how == "slots" and step == 1:
            got[:, at] = memory(rows, slots=slots)
        else:
            got[:, at:at + step] = memory(rows, slots=slots, seq_offsets=torch.tensor([0, step, 2 * step], dtype=torch.int32, device="cuda")).view(2, step, 11)
        at += step
    near(got.view(2 * n, 11), want)
    assert memory.windows.tolist() == [n, 0, n] and memory.past[1] == 0 and 64 <= int(memory.past.max()) < memory.round + 64
    assert 64 * memory.table.shape[1] == 2 * memory.round


def test_angles_far_on(monkeypatch):
    """A stream whose windows are numbered from 2^33 on."""
    torch, memory = make(recall_windows=64, longest=100, n_streams=1)
    memory.windows += 1 << 33
    x, rows = torch.randn(300, 96, device="cuda"), ops_ref.head_rows
    monkeypatch.setattr(ops_ref, "head_rows", lambda y, weight, eps, freqs, pairs, at: rows(y, weight, eps, freqs, pairs, at + (1 << 33)))
    want = reference(memory, x.cpu().numpy(), [(0, 300)])
    offsets = torch.tensor([0, 100], dtype=torch.int32, device="cuda")
    near(torch.cat([memory(x[at:at + 100], seq_offsets=offsets) for at in (0, 100, 200)]), want)


def test_pages_that_are_kept_are_the_first_ones():
    """Windows behind them look at what is kept, however far behind."""
    torch, memory = make(recall_windows=128, recall_pages=2, n_streams=2)
    x = torch.randn(2, 96, device="cuda")
    for i in range(150):
        memory(torch.randn(2, 96, device="cuda"))
    assert memory.past.tolist() == [128, 128] and memory.windows.tolist() == [150, 150]
    kept = [t.clone() for layer in memory.layers for t in layer.cache[:5]]
    a = memory(x)
    memory.past[:], memory.windows[:] = 100000, 150
    assert torch.equal(memory(x), a) and torch.isfinite(a).all()
    for t, u in zip(kept, (t for layer in memory.layers for t in layer.cache[:5])):
        assert torch.equal(t.view(torch.uint8), u.view(torch.uint8))


def test_rounds_in_a_graph():
    torch, memory = make(recall=(0,), recall_windows=64, longest=64, n_streams=2)
    _, other = make(recall=(0,), recall_windows=64, longest=64, n_streams=2)
    x = torch.randn(2, 96, device="cuda")
    memory(x)
    other(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = memory(x)
    for _ in range(600):
        x.normal_()
        graph.replay()
        assert torch.equal(y, other(x))
    torch.cuda.synchronize()
    assert memory.past.tolist() == other.past.tolist() and memory.windows.tolist() == [601, 601] and int(memory.past[0]) < 601


@pytest.mark.parametrize("offsets,good", [([0, 2, 9], [0, 2, 3]), ([-4, 2, 3], [0, 2, 3]), ([0, 3, 1], [0, 3, 3]), ([7, 9, 8], [3, 3, 3])])
def test_offsets_out_of_range_are_cut_off(offsets, good):
    """What is behind the windows of a call is nobody's: streams move on by the windows that they had."""
    torch, memory = make()
    _, other = make()
    x, slots = torch.randn(3, 96, device="cuda"), torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    first = torch.randn(4, 96, device="cuda")
    y = [m(x, slots=slots, seq_offsets=torch.tensor(o, dtype=torch.int32, device="cuda")) for m, o in ((memory, offsets), (other, good)) if m(first) is not None]
    if good[0] == 0 and good[2] == 3:
        assert torch.equal(*y)
    assert memory.past.tolist() == other.past.tolist() == [1, 1 + good[2] - good[1], 1, 1 + good[1] - good[0]] and torch.equal(memory.windows, other.windows)
    for _ in range(3):
        x = torch.randn(4, 96, device="cuda")
        a, b = memory(x), other(x)
        assert torch.equal(a, b) and torch.isfinite(a).all()


@pytest.mark.parametrize("bad", [dict(d_v=4), dict(d_v=300), dict(recall=(1,), d_k=300), dict(dtype="float16"), dict(recall_kind="int4"), dict(dim=20000)])
def test_sizes_that_a_call_would_refuse_are_refused_when_the_memory_is_made(bad):
    import torch
    from paper_2303_04670_amd import evconv as ev
    with pytest.raises(ev.EvConvError):
        make(**{k: getattr(torch, v) if k == "dtype" else v for k, v in bad.items()})
    torch.cuda.synchronize()


@pytest.mark.parametrize("recall", [(0,), (1,), (0, 1)])
def test_slots_and_offsets_are_refused_before_anything_is_rewritten(recall):
    torch, memory = make(recall=recall)
    from paper_2303_04670_amd import evconv as ev
    x = torch.randn(4, 96, device="cuda")
    memory(x)
    everything = lambda: [t for layer in memory.layers if layer.cache for t in layer.cache[:5] if t is not None] + [s for s in memory.states if s is not None] + [memory.past, memory.windows]
    before = [t.clone() for t in everything()]
    slots, offsets = torch.arange(4, dtype=torch.int32, device="cuda"), torch.arange(5, dtype=torch.int32, device="cuda")
    for call in (lambda: memory(x, slots=slots.long()), lambda: memory(x, slots=slots.cpu()), lambda: memory(x, slots=slots[:, None]), lambda: memory(x, slots=slots.float()),
                 lambda: memory(x, seq_offsets=offsets.long()), lambda: memory(x, seq_offsets=offsets.cpu()), lambda: memory(x, slots=slots, seq_offsets=offsets[:4]),
                 lambda: memory(x, slots=torch.stack([slots, slots], 1)[:, 0]), lambda: memory(x[0], seq_offsets=offsets), lambda: memory(x[0, 0], seq_offsets=offsets)):
        with pytest.raises(ev.EvConvError):
            call()
        for a, b in zip(before, everything()):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_every_stream_brings_up_to_the_longest():
    """The limit is each stream's; one above it is left as it was, the others are not concerned."""
    torch, memory = make()
    lens = [250, 300, 290, 1]
    first = np.concatenate([[0], np.cumsum(lens)])
    x = torch.randn(sum(lens), 96, device="cuda")
    near(memory(x, seq_offsets=torch.tensor(first, dtype=torch.int32, device="cuda")), reference(memory, x.cpu().numpy(), [(int(a), n) for a, n in zip(first, lens)]))
    assert memory.past.tolist() == memory.windows.tolist() == lens


@pytest.mark.parametrize("named", [False, True])
def test_a_stream_that_brings_too_many_windows_is_left_as_it_was(named):
    torch, memory = make(recall=(1,), layers=3)
    _, other = make(recall=(1,), layers=3)
    start, slots = torch.randn(4, 96, device="cuda"), torch.tensor([2, 0, 3], dtype=torch.int32, device="cuda")
    order = [2, 0, 3] if named else [0, 1, 2]
    for m in (memory, other):
        m(start)
    many, few = torch.randn(20 + 310 + 290, 96, device="cuda"), [20, 310, 290]
    bounds = torch.tensor([0, 20, 330, 620], dtype=torch.int32, device="cuda")
    y = memory(many, seq_offsets=bounds, slots=slots if named else None)
    # the same without the stream of 310
    rest = torch.cat([many[:20], many[330:]])
    z = other(rest, seq_offsets=torch.tensor([0, 20, 20, 310], dtype=torch.int32, device="cuda"), slots=slots if named else None)
    assert y[20:330].isnan().all() and torch.isfinite(z).all()
    near(torch.cat([y[:20], y[330:]]), z.double().cpu().numpy())  # (sums may be cut otherwise)
    want = [1, 1, 1, 1]
    want[order[0]] += 20
    want[order[2]] += 290
    assert memory.past.tolist() == memory.windows.tolist() == want
    x = torch.randn(4, 96, device="cuda")
    a, b = memory(x), other(x)
    near(a, b.double().cpu().numpy())
    assert torch.equal(a[order[1]], b[order[1]])


@pytest.mark.parametrize("sizes", [dict(recall=(0,)), dict(recall=(0, 1), recall_windows=128, recall_pages=2), dict(recall=(1,), longest=30)])
def test_ragged_windows_in_a_graph(sizes):
    """Recorded once, replayed with other offsets, slots and windows; in the last case a stream brings too many of them now and then."""
    torch, memory = make(**sizes)
    _, other = make(**sizes)
    x, offsets, slots = torch.randn(80, 96, device="cuda"), torch.tensor([0, 20, 50, 80], dtype=torch.int32, device="cuda"), torch.tensor([3, 0, 1], dtype=torch.int32, device="cuda")
    memory(x, slots=slots, seq_offsets=offsets)
    other(x, slots=slots, seq_offsets=offsets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = memory(x, slots=slots, seq_offsets=offsets)
    for bounds, named in (([0, 20, 50, 80], [3, 0, 1]), ([0, 0, 60, 80], [2, -1, 1]), ([0, 33, 33, 80], [0, 1, 2]), ([0, 30, 55, 80], [1, 2, 3]), ([0, 1, 2, 80], [3, 2, 0])):
        x.normal_()
        offsets.copy_(torch.tensor(bounds))
        slots.copy_(torch.tensor(named))
        graph.replay()
        want = other(x, slots=slots, seq_offsets=offsets)
        assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.nan_to_num(), want.nan_to_num())
        assert torch.isfinite(y).all() or "longest" in sizes
        torch.cuda.synchronize()
        assert torch.equal(memory.past, other.past) and torch.equal(memory.windows, other.windows)
    memory.forget([3])
    assert memory.past[3] == 0 and memory.windows[3] == 0 and torch.equal(memory.windows[:3], other.windows[:3])
