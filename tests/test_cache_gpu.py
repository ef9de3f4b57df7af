"""The paged cache on the GPU, through the C ABI's binding, against its formulas in 64 bits.

Tolerances, set beforehand.  Rows that are normed and rotated: fp32 2^-20 of the largest value (some ten roundings of 2^-24 and a
cosine of 2^-24), bf16 half a step, 2^-8 of the value, plus that.  Attention in fp32: as the other sequence operators, 2^-18 of the norm
and 2^-15 of the largest value.  Attention in bf16: half a step of the result, 2^-8 of it, and half a step of each weight, 2^-8 of the
weights' sum over |v|, and 2^-16 of that for all that is fp32."""
import numpy as np
import pytest

import ops_ref
from paper_2303_04670_amd import evconv as ev

pytestmark = pytest.mark.gpu


def torch_ops():
    import torch
    from paper_2303_04670_amd import ops
    return torch, ops


def to_bf16(x):
    import torch
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)


class Streams:
    """Streams with `past` tokens each in a cache whose other places hold what nobody may see."""

    def __init__(self, seed, past, news, heads, d, kind, page, spare=3, poison=True):
        torch, ops = torch_ops()
        self.rng = rng = np.random.default_rng(seed)
        self.past, self.news, self.heads, self.d, self.kind, self.page = list(past), list(news), heads, d, kind, page
        held = [max(-(-(p + n) // page), 0) for p, n in zip(past, news)]
        self.n_pages, self.width = sum(held) + spare, max(held) + 2
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(past), self.width), -1, np.int32)
        at = 0
        for s, h in enumerate(held):
            self.table[s, :h] = order[at:at + h]
            at += h
        self.cache = ops.cache_new(self.n_pages, heads, d, page=page, kind=kind, device="cuda")
        self.dp = self.cache.bounds.shape[-1]
        # every value that is not written is a NaN, or (codes) has a scale that is one
        for t in self.cache[:5]:
            if t is not None:
                t.fill_(0xff if t.dtype == torch.uint8 else float("nan") if poison else 0)
        self.k = [rng.standard_normal((max(p, 0), heads, d)) for p in past]
        self.v = [rng.standard_normal((max(p, 0), heads, d)) for p in past]

    def offsets(self):
        torch, _ = torch_ops()
        return torch.tensor(np.concatenate([[0], np.cumsum(self.news)]), dtype=torch.int32, device="cuda")

    def args(self, equal=False):
        torch, _ = torch_ops()
        return dict(table=torch.from_numpy(self.table).cuda(), past=torch.tensor(self.past, dtype=torch.int32, device="cuda"),
                    seq_offsets=None if equal else self.offsets())

    def held(self, x):
        """What the cache makes of rows, as 64-bit values."""
        if self.kind == "bf16":
            return to_bf16(x).float().numpy().astype(np.float64)
        return ops_ref.fp4_values(*ops_ref.fp4_rows(x))

    def place(self, s, t):
        return int(self.table[s, t // self.page]), t % self.page

    def fill(self):
        """The past's tokens into the cache, written by their layout.  (Keys and values then are what the cache holds.)"""
        import torch
        c, numbers = self.cache, [t if t is None else t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy() for t in self.cache[:5]]
        k_to, v_to, k_scale, v_scale, bounds = numbers
        for s in range(len(self.past)):
            self.k[s], self.v[s] = self.k[s].astype(np.float32), self.v[s].astype(np.float32)
            low = to_bf16(self.k[s]).float().numpy()
            for t in range(len(self.k[s])):
                page, slot = self.place(s, t)
                if slot == 0:
                    bounds[page] = 0
                    bounds[page, :, :, :self.d] = low[t][:, None]
                bounds[page, :, 0, :self.d] = np.minimum(bounds[page, :, 0, :self.d], low[t])
                bounds[page, :, 1, :self.d] = np.maximum(bounds[page, :, 1, :self.d], low[t])
                if self.kind == "bf16":
                    k_to[page, :, slot], v_to[page, :, :, slot] = 0, 0
                    k_to[page, :, slot, :self.d], v_to[page, :, :self.d, slot] = low[t], to_bf16(self.v[s][t]).float().numpy()
                else:
                    (kc, ks), (vc, vs) = ops_ref.fp4_rows(self.k[s][t]), ops_ref.fp4_rows(self.v[s][t])
                    kc, vc = (np.pad(x, ((0, 0), (0, self.dp - self.d))) for x in (kc, vc))
                    k_to[page, :, slot] = kc[:, ::2] | kc[:, 1::2] << 4
                    byte, shift = slot // 2, 4 * (slot % 2)
                    v_to[page, :, :, byte] = (v_to[page, :, :, byte] & (0xf0 >> shift)) | vc << shift
                    k_scale[page, :, slot], v_scale[page, :, slot] = ks, vs
            self.k[s], self.v[s] = self.held(self.k[s]), self.held(self.v[s])
        for t, x in zip(c[:5], numbers):
            if t is not None:
                t.copy_(torch.from_numpy(x).to(t.dtype))
        return self


def freqs_of(rot):
    import torch
    return torch.tensor(1000.0 ** (-np.arange(0, rot, 2) / max(rot, 1)), dtype=torch.float32, device="cuda") if rot else None


def close_rows(got, want, bf16):
    got = got.detach().float().cpu().numpy().astype(np.float64)
    assert got.shape == want.shape
    slack = (2.0 ** -8 if bf16 else 0) * np.abs(want) + 2.0 ** -20 * np.abs(want).max(initial=1e-30)
    assert (np.abs(got - want) <= slack).all(), (np.abs(got - want) - slack).max()


LENGTHS = [([0, 5, 31, 32, 200, 63], [1, 1, 1, 1, 1, 1]), ([0, 3, 70, 0, 64, 33], [100, 0, 1, 33, 64, 130]), ([7, 0], [300, 2])]


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", range(3))
@pytest.mark.parametrize("hq,hk,d,page,rot,pairs,norm", [
    (4, 2, 64, 64, 64, "halves", True), (3, 3, 80, 32, 48, "neighbours", True), (6, 1, 37, 128, 20, "halves", True), (2, 2, 128, 64, 48, "halves", False),
    (0, 2, 17, 32, 6, "neighbours", False), (5, 5, 250, 256, 250, "halves", True), (1, 1, 1, 32, 0, "halves", True), (16, 4, 192, 32, 0, "halves", True)])
def test_append(hq, hk, d, page, rot, pairs, norm, lengths, dtype, kind):
    torch, ops = torch_ops()
    past, news = LENGTHS[lengths]
    st = Streams(lengths, past, news, hk, d, kind, page).fill()
    t, n, g = torch.float32 if dtype == "f32" else torch.bfloat16, sum(news), torch.Generator().manual_seed(d)
    q, k, v = (torch.randn(n, h, d, generator=g).to(t) for h in (hq, hk, hk))
    weights = [1 + 0.2 * torch.randn(d, generator=g) if norm else None for _ in range(2)]
    freqs = freqs_of(rot)
    untouched = [None if x is None else x.clone() for x in st.cache[:5]]
    got = ops.cache_append(st.cache, k.cuda(), v.cuda(), q=q.cuda() if hq else None, q_norm=None if not norm else weights[0].cuda(),
                           k_norm=None if not norm else weights[1].cuda(), freqs=freqs, pairs=pairs, **st.args())
    position = np.concatenate([p + np.arange(m) for p, m in zip(past, news)])
    stream = np.concatenate([[s] * m for s, m in enumerate(news)]).astype(int)
    rows = lambda x, w: ops_ref.head_rows(x.float().numpy(), None if w is None else w.numpy(), 1e-6, None if freqs is None else freqs.cpu().numpy(), pairs, position)
    if hq:
        close_rows(got, rows(q, weights[0]), dtype == "bf16")
    else:
        assert got is None
    k_want, v_want = rows(k, weights[1]), v.float().numpy().astype(np.float64)
    back_k, back_v = ops.cache_read(st.cache, n=n, **st.args())
    if kind == "bf16":
        close_rows(back_k, k_want, True)
        assert np.array_equal(back_v.cpu().numpy(), to_bf16(v_want).float().numpy())
    else:  # half of the widest gap between two codes that the value lies between, for a value of fp32 a little beside it
        for back, want in ((back_k, k_want), (back_v, v_want)):
            m = np.abs(want).max(-1, keepdims=True)
            got_rows = back.cpu().numpy().astype(np.float64)
            y = 6 * np.abs(want) / m
            gap = np.where(y < 2, 0.25, np.where(y < 4, 0.5, 1.0))
            assert (np.abs(got_rows - want) <= (gap + 2.0 ** -19) * m / 6).all()
        code, scale = ops_ref.fp4_rows(v_want)
        assert np.array_equal(back_v.cpu().numpy(), ops_ref.fp4_values(code, scale).astype(np.float32))
    # bounds: of every page that was written to; all else as it was
    k_low = to_bf16(k_want).float().numpy()
    bounds, before = st.cache.bounds.float().cpu().numpy(), untouched[4].float().cpu().numpy()
    expect = before.copy()
    touched = np.zeros((st.n_pages, page), bool)
    for i in range(n):
        p, slot = st.place(stream[i], position[i])
        touched[p, slot] = True
        if slot == 0:
            expect[p] = 0
            expect[p, :, :, :d] = k_low[i][:, None]
        expect[p, :, 0, :d], expect[p, :, 1, :d] = np.minimum(expect[p, :, 0, :d], k_low[i]), np.maximum(expect[p, :, 1, :d], k_low[i])
    fine = np.isfinite(expect)
    assert np.array_equal(fine, np.isfinite(bounds))
    assert (np.abs(bounds - expect)[fine] <= 2.0 ** -7 * np.abs(expect[fine]) + 2.0 ** -20).all()  # (a step of bf16, where a key lies between two)
    keep = torch.from_numpy(~touched).cuda()
    same = lambda a, b: torch.equal(a.view(torch.uint8) if a.dtype != torch.uint8 else a, b.view(torch.uint8) if b.dtype != torch.uint8 else b)
    pages = keep.nonzero()
    assert same(st.cache.k[pages[:, 0], :, pages[:, 1]].contiguous(), untouched[0][pages[:, 0], :, pages[:, 1]].contiguous())
    if kind == "bf16":
        assert same(st.cache.v[pages[:, 0], :, :, pages[:, 1]].contiguous(), untouched[1][pages[:, 0], :, :, pages[:, 1]].contiguous())
    else:
        pick = lambda v: v[pages[:, 0], :, :, pages[:, 1] // 2] >> (4 * (pages[:, 1] % 2))[:, None, None] & 15
        assert torch.equal(pick(st.cache.v), pick(untouched[1]))
        for i in (2, 3):
            assert same(st.cache[i].transpose(1, 2)[keep].contiguous(), untouched[i].transpose(1, 2)[keep].contiguous())


def test_fp4_codes_are_the_nearest_with_ties_to_even():
    """Every quotient of 6 x / m over a fine grid, the middles among them, on both sides."""
    torch, ops = torch_ops()
    y = np.concatenate([np.linspace(-6, 6, 12 * 64 + 1), np.nextafter(np.float32([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]), np.float32(9)),
                        np.nextafter(np.float32([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]), np.float32(0))]).astype(np.float32)
    for m in (1.0, 0.75, 2.0 ** -100, 3e38, 2.0 ** -126):
        d = 64
        n = -(-len(y) // (d - 1))
        x = np.zeros((n, 1, d), np.float32)
        x[:, 0, 0] = 6
        flat = np.resize(y, n * (d - 1)).reshape(n, d - 1)
        x[:, 0, 1:] = flat
        x = (x.astype(np.float64) * (m / 6)).astype(np.float32)
        st = Streams(1, [0], [n], 1, d, "fp4", 32)
        k = torch.from_numpy(x).cuda()
        ops.cache_append(st.cache, k, k, **st.args())
        back_k, back_v = ops.cache_read(st.cache, n=n, **st.args())
        if m < 3e38:  # (there the reference's own 6 x is infinite)
            code, scale = ops_ref.fp4_rows(x)
        else:
            code, _ = ops_ref.fp4_rows((x.astype(np.float64) * 2.0 ** -20).astype(np.float32))
            scale = np.abs(x).max(-1) / np.float32(6)
        want = ops_ref.fp4_values(code, scale).astype(np.float32)
        assert np.array_equal(back_k.cpu().numpy(), want) and np.array_equal(back_v.cpu().numpy(), want), m


def attend_case(st, hq, dtype, equal=False, causal=True, window=None, scale=None, selected=None, q=None, **kw):
    """The call and its reference over streams whose cache holds past + news tokens."""
    torch, ops = torch_ops()
    t, n, d = torch.float32 if dtype == "f32" else torch.bfloat16, sum(st.news), st.d
    if q is None:
        q = torch.from_numpy(1.5 * st.rng.standard_normal((n, hq, d))).to(t)
    args = st.args(equal)
    if selected is not None:
        kw["selected"] = torch.from_numpy(selected).cuda()
    got = ops.cache_attend(q.cuda(), st.cache, causal=causal, window=window, scale=scale, **args, **kw)
    want, spread = np.zeros((2, n, hq, d))
    share, at, x = hq // st.heads, 0, q.float().numpy().astype(np.float64)
    for s, (past, new) in enumerate(zip(st.past, st.news)):
        k, v = st.k[s], st.v[s]
        token = np.arange(len(k))
        position = past + np.arange(new)
        seen = token <= position[:, None] if causal else np.broadcast_to(token < past, (new, len(k)))
        if window:
            seen = seen & (token > position[:, None] - window)
        for h in range(hq):
            mine = seen
            if selected is not None:
                mine = seen & np.array([[t // st.page in selected[at + i, h // share] for t in token] for i in range(new)], bool).reshape(seen.shape)
            want[at:at + new, h], spread[at:at + new, h] = ops_ref.attend(x[at:at + new, h], k[:, h // share], v[:, h // share], d ** -0.5 if scale is None else scale, mine)
        at += new
    return got, want, spread


def check_attention(got, want, spread, dtype):
    got = got.detach().float().cpu().numpy().astype(np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), "values that are not finite, elsewhere"
    if not fine.any():
        return
    diff, w = np.abs(got - want)[fine], np.abs(want)[fine]
    if dtype == "f32":
        assert np.linalg.norm(diff) <= 2.0 ** -18 * np.linalg.norm(w), np.linalg.norm(diff) / np.linalg.norm(w)
        assert diff.max() <= 2.0 ** -15 * w.max(), diff.max() / w.max()
    else:
        slack = 2.0 ** -8 * w + (2.0 ** -8 + 2.0 ** -16) * spread[fine]
        assert (diff <= slack).all(), (diff / np.maximum(slack, 1e-30)).max()
    assert not got[want == 0].any()  # (rows that see nothing)


def whole(past, news, *args, **kw):
    """Streams that hold the new tokens too."""
    st = Streams(args[0], [max(p + n, 0) for p, n in zip(past, news)], [0] * len(news), *args[1:], **kw).fill()
    st.past, st.news = list(past), list(news)
    return st


SHAPES = [(4, 2, 64, 64), (6, 3, 80, 32), (8, 8, 32, 128), (5, 1, 37, 32), (16, 1, 128, 64), (3, 1, 250, 256), (40, 2, 100, 64), (2, 2, 160, 32), (1, 1, 1, 64)]


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk,d,page", SHAPES)
def test_attend_single_tokens(hq, hk, d, page, dtype, kind):
    past = [0, 1, 30, 31, 32, 33, 63, 64, 127, 128, 129, 255, 700]
    st = whole(past, [1] * len(past), d, hk, d, kind, page)
    check_attention(*attend_case(st, hq, dtype, equal=True), dtype)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk,d,page", SHAPES)
def test_attend_pieces(hq, hk, d, page, dtype, kind):
    past, news = [0, 3, 70, 0, 64, 33, 500, 0], [100, 0, 1, 33, 64, 130, 3, 1]
    st = whole(past, news, d, hk, d, kind, page)
    check_attention(*attend_case(st, hq, dtype), dtype)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 100, 5000])
def test_attend_window(window, dtype, kind):
    past, news = [0, 3, 300, 0, 64, 500], [100, 0, 1, 33, 200, 3]
    st = whole(past, news, 5, 2, 96, kind, 32)
    check_attention(*attend_case(st, 4, dtype, window=window), dtype)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("news", [[1] * 5, [40, 1, 7, 0, 150]])
def test_attend_without_causal(news, dtype, kind):
    """Queries that look at what is cached, nothing too."""
    st = Streams(3, [0, 1, 130, 32, 600], news, 2, 64, kind, 64).fill()
    check_attention(*attend_case(st, 6, dtype, causal=False, scale=0.3), dtype)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("past,new,hq,hk", [([5000], 1, 4, 2), ([9000, 100, 3000], 1, 2, 1), ([6000], 5, 16, 2), ([4000, 1, 2500], 70, 4, 1)])
def test_attend_long(past, new, hq, hk, dtype, kind):
    """Rows whose tokens several workgroups share."""
    st = whole(past, [new] * len(past), 7, hk, 64, kind, 64)
    check_attention(*attend_case(st, hq, dtype, equal=True), dtype)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk,count,page", [(4, 2, 5, 32), (6, 1, 3, 64), (40, 2, 9, 128), (2, 2, 60, 32)])
def test_attend_chosen_pages(hq, hk, count, page, dtype, kind):
    past, news = [0, 3, 300, 0, 64, 900], [10, 0, 1, 33, 40, 3]
    st = whole(past, news, 9, hk, 64, kind, page)
    n, rng = sum(news), np.random.default_rng(3)
    selected = np.full((n, hk, count), -1, np.int32)
    for i in range(n):
        for h in range(hk):
            pages = rng.permutation(st.width)[:rng.integers(0, count + 1)]  # pages behind the query and of no tokens among them
            selected[i, h, rng.permutation(count)[:len(pages)]] = pages
    selected[0, 0, :] = -5
    check_attention(*attend_case(st, hq, dtype, selected=selected), dtype)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk,d,page,count", [(4, 2, 64, 32, 4), (3, 3, 37, 64, 2), (16, 1, 128, 32, 9), (20, 1, 200, 32, 3), (2, 1, 20, 128, 70), (8, 2, 96, 32, 1)])
def test_select(hq, hk, d, page, count, dtype, kind):
    torch, ops = torch_ops()
    past, news = [0, 3, 300, 0, 64, 2000], [10, 0, 1, 33, 40, 3]
    st = whole(past, news, d, hk, d, kind, page)
    t, n = torch.float32 if dtype == "f32" else torch.bfloat16, sum(news)
    q = torch.from_numpy(st.rng.standard_normal((n, hq, d))).to(t)
    for first, last in ((1, 1), (0, 2), (3, 1), (0, 1)):
        if first + last > count:
            continue
        got = ops.cache_select(q.cuda(), st.cache, count=count, first=first, last=last, **st.args()).cpu().numpy()
        bounds, x, i = st.cache.bounds.float().cpu().numpy().astype(np.float64), q.float().numpy().astype(np.float64), 0
        for s, (p, m) in enumerate(zip(past, news)):
            for j in range(m):
                pages = st.table[s, :(p + j) // page + 1]
                for h in range(hk):
                    mine = x[i, h * (hq // hk):(h + 1) * (hq // hk), None]
                    score = np.maximum(mine * bounds[pages, h, 0, :d], mine * bounds[pages, h, 1, :d]).sum(-1).max(0).astype(np.float32)
                    assert got[i, h].tolist() == ops_ref.choose(score, count, first, last), (i, h, first, last)
                i += 1


def test_select_of_equal_pages_takes_the_lower_ones():
    torch, ops = torch_ops()
    st = whole([3199], [1], 1, 2, 64, "bf16", 32)
    st.cache.bounds[:] = 1.0
    q = torch.zeros(1, 4, 64, device="cuda")
    for value in (0.0, 1.0, -1.0):
        got = ops.cache_select(q + value, st.cache, count=7, first=0, **st.args()).cpu().tolist()
        assert got == [[[0, 1, 2, 3, 4, 5, 99]] * 2]
    st.cache.bounds[int(st.table[0, 50]), 1, 0, 5] = float("nan")
    got = ops.cache_select(q + 1, st.cache, count=3, first=0, **st.args()).cpu().tolist()
    assert got == [[[0, 1, 99], [0, 50, 99]]]
    st.table[0, 1] = -1  # a page that is not there
    got = ops.cache_select(q + 1, st.cache, count=4, first=2, **st.args()).cpu().tolist()
    assert got == [[[0, 2, 3, 99], [0, 2, 50, 99]]]


@pytest.mark.parametrize("n_pages", [5, 1500, 5000])
def test_select_of_many_pages(n_pages):
    """Scores that repeat, and a choice among thousands."""
    torch, ops = torch_ops()
    rng = np.random.default_rng(n_pages)
    cache = ops.cache_new(n_pages, 1, 32, page=32, device="cuda")
    values = rng.integers(-20, 20, n_pages)
    cache.bounds[:, 0] = torch.from_numpy(values).float().cuda()[:, None, None].expand(-1, 2, 32).to(torch.bfloat16)
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda")[None]
    past = torch.tensor([32 * n_pages - 1], dtype=torch.int32, device="cuda")
    q = torch.ones(1, 1, 32, device="cuda")
    for count in (1, 2, 3, 64, 1000, 4999, 6000):
        got = ops.cache_select(q, cache, table, past, count, first=min(count - 1, 1)).cpu().tolist()[0][0]
        assert got == ops_ref.choose(32 * values, count, min(count - 1, 1), 1), count
