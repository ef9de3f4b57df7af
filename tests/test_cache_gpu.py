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


@pytest.mark.parametrize("close", [1, 2, 255, 256, 257, 400])
def test_select_among_close_scores(close):
    """The last page chosen is one of some that lie close together, most of them equal to others, between few that lie far above and below."""
    torch, ops = torch_ops()
    rng = np.random.default_rng(close)
    values = np.concatenate([1 + rng.integers(0, 4, close) / 128, 2.0 ** rng.integers(8, 30, 40), -2.0 ** rng.integers(8, 30, 200)])  # exact in bf16
    rng.shuffle(values)
    values = np.append(values, 0)  # the newest page, always chosen
    n_pages = len(values)
    cache = ops.cache_new(n_pages, 1, 32, page=32, device="cuda")
    cache.bounds[:, 0] = torch.from_numpy(values).float().cuda()[:, None, None].expand(-1, 2, 32).to(torch.bfloat16)
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda")[None]
    past = torch.tensor([32 * n_pages - 1], dtype=torch.int32, device="cuda")
    q = torch.ones(1, 1, 32, device="cuda")
    for count in sorted({41, 42, 41 + close // 2, 40 + close, 41 + close, 42 + close}):
        got = ops.cache_select(q, cache, table, past, count, first=0).cpu().tolist()[0][0]
        assert got == ops_ref.choose(32 * values, count, 0, 1), count


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


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("news", [[1, 1, 1], [40, 3, 150]])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_bad_values_reach_those_who_look_at_them(value, where, news, dtype, kind):
    """One token of one head: its stream's queries of that head from its position on are NaN, all others as without it."""
    torch, ops = torch_ops()
    past = [70, 0, 33]
    st = whole(past, news, 2, 2, 64, kind, 32)
    t, n = torch.float32 if dtype == "f32" else torch.bfloat16, sum(news)
    q = torch.from_numpy(st.rng.standard_normal((n, 4, 64))).to(t).cuda()
    clean = ops.cache_attend(q, st.cache, **st.args())
    # the stream's last tokens again, one of them with a bad value
    s, again = 0, 40 if news[0] > 1 else 1
    at = past[0] + news[0] - again
    rows = {i: torch.from_numpy(getattr(st, i)[s][at:at + again]).float() for i in ("k", "v")}
    bad = again // 2
    rows[where][bad, 1, 17] = value
    args = st.args()
    ops.cache_append(st.cache, rows["k"].cuda(), rows["v"].cuda(), args["table"][:1], torch.tensor([at], dtype=torch.int32, device="cuda"))
    got = ops.cache_attend(q, st.cache, **st.args())
    hit = torch.zeros(n, 4, dtype=torch.bool)
    hit[max(at + bad - past[0], 0):news[0], 2:] = True
    assert got[hit.cuda()].isnan().all()
    if kind == "bf16":  # (rows of 4 bits are rounded once more by being appended again)
        assert torch.equal(got[~hit.cuda()], clean[~hit.cuda()])
    else:
        assert torch.isfinite(got[~hit.cuda()]).all()
    # and a page that holds such a key is always worth a look
    if where == "k" or kind == "bf16":
        last = past[0] + news[0] - 1
        chosen = ops.cache_select(q[news[0] - 1:news[0]].contiguous(), st.cache, args["table"][:1], torch.tensor([last], dtype=torch.int32, device="cuda"), 3)
        assert (at + bad) // 32 in chosen[0, 1].tolist()


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("news", [[1, 1], [50, 3]])
def test_rows_anywhere(news, dtype, kind):
    """Slices of one projection at odd places, results between others', queries in place, angles by positions of their own."""
    torch, ops = torch_ops()
    t, n, d, g = torch.float32 if dtype == "f32" else torch.bfloat16, sum(news), 24, torch.Generator().manual_seed(3)
    wide = torch.randn(n, 3 + 6 * d + 5, generator=g).to(t).cuda()
    parts = [wide[:, 3 + a * d:3 + b * d].unflatten(1, (-1, d)) for a, b in ((0, 2), (2, 4), (4, 6))]
    positions = torch.randint(0, 1 << 40, (n,), generator=g).cuda()
    one, two = Streams(4, [40, 0], news, 2, d, kind, 32).fill(), Streams(4, [40, 0], news, 2, d, kind, 32).fill()
    kw = dict(freqs=freqs_of(24) * 1e-6, positions=positions, q_norm=torch.ones(d, device="cuda"))
    plain = [p.contiguous() for p in parts]
    before = wide.clone()
    q = ops.cache_append(one.cache, plain[1], plain[2], q=plain[0], **kw, **one.args())
    assert torch.equal(wide, before)
    same = ops.cache_append(two.cache, parts[1], parts[2], q=parts[0], q_out=parts[0], **kw, **two.args())
    assert same is parts[0] and torch.equal(same, q) and torch.equal(wide[:, :3], before[:, :3]) and torch.equal(wide[:, 3 + 2 * d:], before[:, 3 + 2 * d:])
    for a, b in zip(ops.cache_read(one.cache, n=n, **one.args()), ops.cache_read(two.cache, n=n, **two.args())):
        assert torch.equal(a, b)
    close_rows(q, ops_ref.head_rows(before[:, 3:3 + 2 * d].unflatten(1, (-1, d)).float().cpu().numpy(), np.ones(d), 1e-6, kw["freqs"].cpu().numpy(), "halves",
                                    positions.cpu().numpy()), dtype == "bf16")
    want = ops.cache_attend(q, one.cache, **one.args())
    room = torch.full((n, 4, d + 3), 7.0, dtype=t, device="cuda")
    out = ops.cache_attend(parts[0], two.cache, out=room[:, 1:3, 2:2 + d], **two.args())
    assert torch.equal(out, want) and room[:, 0].eq(7).all() and room[:, 3].eq(7).all() and room[:, :, :2].eq(7).all() and room[:, :, -1].eq(7).all()
    a, b = (ops.cache_select(x, st.cache, count=4, **st.args()) for x, st in ((q, one), (parts[0], two)))
    assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("news", [[1] * 6, [30, 1, 70, 2, 90, 5]])
def test_tokens_that_have_no_place(news, kind):
    """Table entries and positions out of range hold nothing, and nothing is written for them."""
    torch, ops = torch_ops()
    past = [100, 100, 100, -3, 60, 2 ** 31 - 1]
    st = Streams(5, [100, 100, 100, 0, 60, 0], news, 1, 32, kind, 32).fill()
    st.past = past
    st.table[0, 1], st.table[1, 3], st.table[2, 0] = -1, st.n_pages, -2 ** 31
    st.table[5] = -1  # (its past is said to be long, but was never written)
    args = st.args()
    args["table"] = args["table"][:, :5]  # streams 2 and 4 run out of it
    n, g = sum(news), torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(n, 1, 32, generator=g).cuda() for _ in range(3))
    before = [x if x is None else x.clone() for x in st.cache[:5]]
    ops.cache_append(st.cache, k, v, q=q, **args)
    back_k, back_v = (x.cpu().numpy() for x in ops.cache_read(st.cache, n=n, **args))
    got = ops.cache_attend(q, st.cache, **args).cpu().numpy()
    chosen = ops.cache_select(q, st.cache, count=6, **args).cpu().numpy()
    looked = ops.cache_attend(q, st.cache, selected=torch.from_numpy(chosen).cuda(), **args).cpu().numpy()
    pages, i, written = st.table[:, :5], 0, set()
    there = lambda s, t: 0 <= t < 5 * 32 and 0 <= pages[s, t // 32] < st.n_pages
    for s, new in enumerate(news):
        held = {t: (st.k[s][t], st.v[s][t]) for t in range(max(min(past[s], 160), 0)) if t < len(st.k[s]) and there(s, t)}
        for j in range(new):
            t = past[s] + j
            if there(s, t):
                held[t] = (st.held(k[i].cpu().numpy()), st.held(v[i].cpu().numpy()))
                written.add(int(pages[s, t // 32]))
                assert np.allclose(back_k[i], held[t][0], atol=1e-6) and np.allclose(back_v[i], held[t][1], atol=1e-6)
            else:
                assert not back_k[i].any() and not back_v[i].any()
            seen = [x for u, x in held.items() if u <= t]
            want = np.zeros((1, 32))
            if seen:
                kk, vv = np.stack([x[0] for x in seen])[:, 0], np.stack([x[1] for x in seen])[:, 0]
                want, _ = ops_ref.attend(q[i].cpu().numpy().astype(np.float64), kk, vv, 32 ** -0.5, np.ones((1, len(kk)), bool))
            assert np.allclose(got[i], want, atol=2e-5) and np.allclose(looked[i], want, atol=2e-5), (s, j)
            assert [c for c in chosen[i, 0] if c >= 0] == [c for c in range(min(max(t, -1) // 32, 4) + 1) if 0 <= pages[s, c] < st.n_pages]
            i += 1
    for page in set(range(st.n_pages)) - written:
        for x, y in zip(before, st.cache[:5]):
            assert x is None or torch.equal(x[page].view(torch.uint8), y[page].view(torch.uint8))


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
def test_offsets_out_of_order_stay_inside(kind):
    torch, ops = torch_ops()
    st = whole([100] * 4, [20] * 4, 1, 2, 64, kind, 32)
    args, q = st.args(), torch.randn(80, 4, 64, device="cuda")
    for bad in ([0, 50, 20, 70, 80], [-5, 20, 200, 60, 80], [80, 60, 40, 20, 0], [0, 0, 0, 0, 0], [30, 31, 32, 33, 34], [2 ** 31 - 1, -2 ** 31, 5, 90, 7]):
        args["seq_offsets"] = torch.tensor(bad, dtype=torch.int32, device="cuda")
        k = torch.randn(80, 2, 64, device="cuda")
        ops.cache_append(st.cache, k, k, q=q, **args)
        ops.cache_read(st.cache, n=80, **args)
        chosen = ops.cache_select(q, st.cache, count=3, out=torch.full((80, 2, 3), 99, dtype=torch.int32, device="cuda"), **args)
        ops.cache_attend(q, st.cache, **args)
        ops.cache_attend(q, st.cache, selected=chosen, **args)
    torch.cuda.synchronize()
    # rows of no sequence are left as they were
    args["seq_offsets"] = torch.tensor([10, 20, 20, 50, 60], dtype=torch.int32, device="cuda")
    out = torch.full((80, 4, 64), 3.0, device="cuda")
    ops.cache_attend(q, st.cache, out=out, **args)
    rotated = ops.cache_append(st.cache, k, k, q=q, q_out=torch.full_like(q, 3.0), freqs=freqs_of(64), **args)
    for x in (out, rotated):
        assert x[:10].eq(3).all() and x[60:].eq(3).all() and not x[10:60].eq(3).any()


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
def test_cache_behind_32_bits(kind):
    """Pages whose values begin behind 2^32 bytes."""
    torch, ops = torch_ops()
    d, page, pages = 128, 256, 70000 if kind == "bf16" else 280000
    cache = ops.cache_new(pages, 1, d, page=page, kind=kind)
    table = torch.arange(pages - 1, pages - 5, -1, dtype=torch.int32, device="cuda").view(2, 2).contiguous()
    past, n = torch.zeros(2, dtype=torch.int32, device="cuda"), 600
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(n, h, d, generator=g).cuda() for h in (2, 1, 1))
    ops.cache_append(cache, k, v, table, past, q)
    small = ops.cache_new(4, 1, d, page=page, kind=kind)
    near = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    ops.cache_append(small, k, v, near, past, q)
    for a, b in zip(ops.cache_read(cache, table, past, n), ops.cache_read(small, near, past, n)):
        assert torch.equal(a, b)
    last = torch.full((2,), 299, dtype=torch.int32, device="cuda")
    for rows, at in ((q, past), (q[:2].contiguous(), last)):
        assert torch.equal(ops.cache_attend(rows, cache, table, at), ops.cache_attend(rows, small, near, at))
        one, two = (ops.cache_select(rows, c, t, at, 2) for c, t in ((cache, table), (small, near)))
        assert torch.equal(one, two)
        assert torch.equal(ops.cache_attend(rows, cache, table, at, selected=one), ops.cache_attend(rows, small, near, at, selected=two))


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hk,past,new", [(4, 2, 3000, 1), (4, 2, 200, 1), (40, 1, 2500, 2), (4, 4, 900, 70)])
def test_steps_in_a_graph_and_on_another_stream(hq, hk, past, new, kind):
    """The calls of a step recorded once and replayed with other tokens, beside the same calls made one by one; two such graphs, whose
    workspaces are their own, by turns."""
    torch, ops = torch_ops()

    def setting(seed):
        st = whole([past, past // 3, 0], [new] * 3, seed, hk, 64, kind, 64)
        room = st.args(equal=True)
        wide = torch.cat([room["table"], torch.arange(8, dtype=torch.int32, device="cuda").expand(3, 8) % st.n_pages], dim=1).contiguous()
        torch.manual_seed(seed)
        x = [torch.randn(3 * new, h, 64, device="cuda") for h in (hq, hk, hk)]
        return st.cache, wide, room["past"], x

    def step(cache, table, at, x):
        q = ops.cache_append(cache, x[1], x[2], table, at, x[0], freqs=freqs)
        pages = ops.cache_select(q, cache, table, at, 5)
        o = ops.cache_attend(q, cache, table, at), ops.cache_attend(q, cache, table, at, selected=pages)
        at.add_(0)
        return q, pages, *o
    freqs = freqs_of(64)
    both = []
    for seed in (1, 2):
        a, b = setting(seed), setting(seed)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            first = step(*a)
            second = step(*b)
        side.synchronize()
        for u, w in zip(first, second):
            assert torch.equal(u, w)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step(*a)
        both.append((graph, a, b, got))
    for turn in range(4):
        for graph, a, b, _ in both:
            for u, w in zip(a[3], b[3]):
                u.normal_()
                w.copy_(u)
            graph.replay()
        for graph, a, b, got in both:
            for u, w in zip(got, step(*b)):
                assert torch.equal(u, w), turn
        torch.cuda.synchronize()


def test_refusals_leave_the_device_usable_and_gradients_are_refused():
    torch, ops = torch_ops()
    st = whole([40, 9], [1, 1], 1, 2, 64, "bf16", 32)
    args = st.args(equal=True)
    q, k = torch.randn(2, 4, 64, device="cuda"), torch.randn(2, 2, 64, device="cuda")
    want = ops.cache_attend(q, st.cache, **args)
    wrong = dict(args, past=args["past"].long())
    for call in (lambda: ops.cache_attend(q[:, :3], st.cache, **args), lambda: ops.cache_attend(q, st.cache, **wrong), lambda: ops.cache_attend(q.half(), st.cache, **args),
                 lambda: ops.cache_attend(q[..., :63], st.cache, **args), lambda: ops.cache_attend(q, st.cache, window=0, **args),
                 lambda: ops.cache_attend(q, st.cache, max_len=0, **args), lambda: ops.cache_attend(q, st.cache, scale=float("nan"), **args),
                 lambda: ops.cache_attend(q, st.cache, selected=torch.zeros(2, 2, 0, dtype=torch.int32, device="cuda"), **args),
                 lambda: ops.cache_attend(q, st.cache, selected=torch.zeros(2, 4, 3, dtype=torch.int32, device="cuda"), **args),
                 lambda: ops.cache_attend(q, st.cache, causal=False, window=3, **args), lambda: ops.cache_attend(q.cpu(), st.cache, **args),
                 lambda: ops.cache_attend(q, st.cache._replace(k=st.cache.k.float()), **args), lambda: ops.cache_attend(q, st.cache._replace(d=32), **args),
                 lambda: ops.cache_append(st.cache, k, k[:, :1], **args), lambda: ops.cache_append(st.cache, k, k, pairs="thirds", **args),
                 lambda: ops.cache_append(st.cache, k, k, freqs=torch.ones(33, device="cuda"), **args), lambda: ops.cache_append(st.cache, k.bfloat16(), k, **args),
                 lambda: ops.cache_append(st.cache, k, k, k_norm=torch.ones(63, device="cuda"), **args), lambda: ops.cache_read(st.cache, n=3, **args),
                 lambda: ops.cache_select(q, st.cache, count=1, **args), lambda: ops.cache_select(q, st.cache._replace(bounds=None), count=3, **args),
                 lambda: ops.cache_attend(q.clone().requires_grad_(), st.cache, **args), lambda: ops.cache_append(st.cache, k.clone().requires_grad_(), k, **args),
                 lambda: ops.cache_append(st.cache, k, k, k_norm=torch.ones(64, device="cuda", requires_grad=True), **args)):
        with pytest.raises(ev.EvConvError):
            call()
    with torch.no_grad():
        assert torch.equal(ops.cache_attend(q.clone().requires_grad_(), st.cache, **args), want)
    none = dict(table=args["table"], past=args["past"])
    assert ops.cache_attend(q[:0], st.cache, **none).shape == (0, 4, 64) and ops.cache_select(q[:0], st.cache, count=3, **none).shape == (0, 2, 3)
    assert ops.cache_append(st.cache, k[:0], k[:0], q=q[:0], **none).shape == (0, 4, 64) and ops.cache_read(st.cache, n=0, **none)[0].shape == (0, 2, 64)
    assert torch.equal(ops.cache_attend(q, st.cache, **args), want)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_far_apart(dtype, kind):
    """Weights from 1 down to nothing, maxima that rise and fall along the tokens; and all alike."""
    torch, ops = torch_ops()
    for hq, news in ((4, [1, 1]), (4, [90, 40])):
        st = whole([900, 300], news, 6, 2, 64, kind, 64)
        t, n = torch.float32 if dtype == "f32" else torch.bfloat16, sum(news)
        q = torch.from_numpy(20 * st.rng.standard_normal((n, hq, 64))).to(t)
        got, want, spread = attend_case(st, hq, dtype, q=q)
        if dtype == "f32":  # a score of s = 160 is off by up to 2^-24 * s * 8 (three parts, 64 terms), and so is the weight's exponent
            diff = np.abs(got.float().cpu().numpy() - want)
            assert (diff <= 2.0 ** -13 * spread + 1e-6).all(), (diff / spread).max()
        else:
            diff = np.abs(got.float().cpu().numpy() - want)
            assert (diff <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -13) * spread).all()
        check_attention(*attend_case(st, hq, dtype, q=q * 0), dtype)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("n_seq", [63, 65, 4097, 20000])
def test_many_sequences_with_offsets(n_seq, kind):
    """Whose a workgroup's tokens are, among up to 64 sequences and more, empty ones too: against the same calls without offsets."""
    torch, ops = torch_ops()
    rng = np.random.default_rng(n_seq)
    news = torch.from_numpy(rng.integers(0, 2, n_seq))
    live = news.nonzero()[:, 0].cuda()
    n = len(live)
    past = torch.from_numpy(rng.integers(0, 40, n_seq)).int().cuda()
    table = torch.arange(2 * n_seq, dtype=torch.int32, device="cuda").view(n_seq, 2)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), news.cumsum(0)]).int().cuda()
    q, k, v, old = (torch.randn(n, h, 16, device="cuda") for h in (2, 1, 1, 1))
    results = []
    for ragged in (False, True):
        cache = ops.cache_new(2 * n_seq, 1, 16, page=32, kind=kind)
        torch.manual_seed(1)
        start = torch.randn(40 * n_seq, 1, 16, device="cuda")
        ops.cache_append(cache, start, start.roll(1, 0).contiguous(), table, torch.zeros_like(past))
        args = dict(table=table, past=past, seq_offsets=offsets) if ragged else dict(table=table[live], past=past[live])
        turned = ops.cache_append(cache, k, v, q=q, freqs=freqs_of(16), **args)
        pages = ops.cache_select(turned, cache, count=2, **args)
        results.append([turned, pages, ops.cache_attend(turned, cache, **args), ops.cache_attend(turned, cache, window=7, **args),
                        ops.cache_attend(turned, cache, selected=pages, **args), *ops.cache_read(cache, n=n, **args), cache.bounds.view(torch.int16)])
    for a, b in zip(*results):
        if a.dtype == torch.float32:
            assert torch.allclose(a, b, rtol=0, atol=2e-6)  # (sums may be cut otherwise)
        else:
            assert torch.equal(a, b)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("news", [[1, 1, 1], [60, 1, 9]])
def test_tokens_behind_max_len_are_not_seen(news, kind):
    torch, ops = torch_ops()
    past = [300, 10, 129]
    st = whole(past, news, 2, 1, 64, kind, 32)
    q = torch.from_numpy(st.rng.standard_normal((sum(news), 2, 64))).float()
    got = ops.cache_attend(q.cuda(), st.cache, max_len=130, **st.args())
    x, at = q.numpy().astype(np.float64), 0
    for s, (p, n) in enumerate(zip(past, news)):
        token = np.arange(len(st.k[s]))
        seen = (token <= (p + np.arange(n))[:, None]) & (token < 130)
        for h in range(2):
            want, _ = ops_ref.attend(x[at:at + n, h], st.k[s][:, 0], st.v[s][:, 0], 1 / 8, seen)
            assert np.allclose(got[at:at + n, h].cpu().numpy(), want, atol=2e-5)
        at += n
    chosen = ops.cache_select(q.cuda(), st.cache, count=9, max_len=130, **st.args()).cpu().numpy()
    position = np.concatenate([p + np.arange(n) for p, n in zip(past, news)])
    for row, p in zip(chosen[:, 0], position):
        assert [c for c in row if c >= 0] == list(range(min(p, 129) // 32 + 1))


@pytest.mark.parametrize("n_pages,count,first,last", [(40, 3, 1, 1), (2000, 64, 1, 1), (2000, 600, 0, 3), (5000, 128, 2, 2), (20000, 128, 1, 1)])
def test_select_among_pages_that_score_no_number(n_pages, count, first, last):
    """0, need - 1, need, need + 1 and all pages NaN, of one head these and of the other those: whole rows, and nothing written behind them."""
    torch, ops = torch_ops()
    rng, need = np.random.default_rng(n_pages + count), count - first - last
    cache = ops.cache_new(n_pages, 2, 32, page=32, device="cuda")
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda")[None]
    past = torch.tensor([32 * n_pages - 3], dtype=torch.int32, device="cuda")
    q = torch.ones(3, 4, 32, device="cuda")
    numbers = sorted({0, need - 1, need, need + 1, n_pages})
    for bads in zip(numbers, numbers[1:] + numbers[:1]):
        for values in (rng.standard_normal(n_pages), -2.0 ** rng.integers(8, 100, n_pages)):
            scores = np.tile(to_bf16(values).float().numpy(), (2, 1))
            for head, bad in enumerate(bads):
                scores[head, first + rng.permutation(n_pages - first - last)[:bad] if bad < n_pages else slice(None)] = np.nan
            cache.bounds[:] = torch.from_numpy(scores.T.copy()).cuda().to(torch.bfloat16)[:, :, None, None].expand(-1, -1, 2, 32)
            room = torch.full((1 << 16,), 7, dtype=torch.int32, device="cuda")
            out = room[1 << 12:][:3 * 2 * count].view(3, 2, count)
            got = ops.cache_select(q, cache, table, past, count, first=first, last=last, out=out).cpu().numpy()
            assert room[:1 << 12].eq(7).all() and room[(1 << 12) + out.numel():].eq(7).all(), bads
            for head in range(2):
                want = ops_ref.choose(32 * scores[head], count, first, last)
                for token in range(3):
                    assert got[token, head].tolist() == want, (bads, head, token)


@pytest.mark.parametrize("ragged", [False, True])
def test_rows_behind_31_bits(ragged):
    """A sequence of more than 2^31 tokens x query heads of a key head: every token sees the same 32 tokens of one page."""
    torch, ops = torch_ops()
    n, heads = (1 << 21) + 3, 1024
    st = Streams(8, [32], [0], 1, 1, "bf16", 32).fill()
    q = torch.linspace(-3, 3, heads).to(torch.bfloat16).view(1, heads, 1)
    table, past = torch.from_numpy(st.table[:, :1].copy()).cuda(), torch.tensor([31], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, n], dtype=torch.int32, device="cuda") if ragged else None
    got = ops.cache_attend(q.cuda().expand(n, -1, -1), st.cache, table, past, seq_offsets=offsets)
    x = q.float().numpy().astype(np.float64)[0]
    want, spread = ops_ref.attend(x, st.k[0][:, 0], st.v[0][:, 0], 1.0, np.ones((heads, 32), bool))
    check_attention(got[:1], want[None], spread[None], "bf16")
    for at in range(0, n, 1 << 18):
        assert got[at:at + (1 << 18)].eq(got[:1]).all(), at


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [1000, 1500, 1999])
@pytest.mark.parametrize("past,news,hq,hk,page", [
    ([3100, 4999, 700], [1, 1, 1], 4, 2, 64), ([4200, 900, 3333], [5, 5, 5], 6, 2, 32), ([3000, 4000, 990], [200, 200, 200], 4, 2, 64), ([3333], [70], 5, 1, 128),
    ([3300, 0, 4100, 1200, 5, 2999, 3001, 4500], [1, 1, 100, 1, 0, 1, 130, 3], 2, 1, 64)])
def test_windows_whose_tokens_several_workgroups_share(past, news, hq, hk, page, window, dtype, kind, monkeypatch):
    """Stretches begin where the first of a workgroup's rows begins to see; the join has to find the same places, of sequences of few rows
    and of many, also in one call."""
    torch, ops = torch_ops()
    sizes, enqueue = [], ops._enqueue

    def spy(call, args, gpu, workspace_of=None):
        n = ops.ctypes.c_size_t(0)
        assert workspace_of(args, ops.ctypes.byref(n)) == ev.OK
        sizes.append(n.value)
        return enqueue(call, args, gpu, workspace_of)
    monkeypatch.setattr(ops, "_enqueue", spy)
    st = whole(past, news, 11, hk, 64, kind, page)
    check_attention(*attend_case(st, hq, dtype, equal=len(set(news)) == 1, window=window), dtype)
    assert sizes[0] > 0, "nothing is joined"


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
@pytest.mark.parametrize("how", ["step", "ragged", "chosen"])
@pytest.mark.parametrize("hq,hk,d", [(4, 2, 64), (8, 1, 128), (3, 3, 37)])
def test_few_rows_of_bf16_hold_their_weights_in_16_bits(hq, hk, d, how, kind):
    """Single tokens, short sequences beside each other, chosen pages: half a step of the result, and 2^-15 of the weights' sum over |v|.
    (Two bf16 parts leave 2^-16 of a weight; scores of a few are off by 2^-19, the exponential of fp32 by 2^-20.)"""
    past, news = ([5, 700, 2500], [1, 1, 1]) if how == "step" else ([5, 700, 2500, 40], [1, 2, 0, 1])
    st = whole(past, news, 13, hk, d, kind, 64)
    selected = None
    if how == "chosen":
        selected = np.full((sum(news), hk, 5), -1, np.int32)
        for i in range(len(selected)):
            for h in range(hk):
                selected[i, h] = st.rng.permutation(st.width)[:5]
        selected[:, :, 0] = [0]
        selected[:, :, 1:][selected[:, :, 1:] == 0] = -1
    got, want, spread = attend_case(st, hq, "bf16", equal=how == "step", selected=selected)
    diff, slack = np.abs(got.float().cpu().numpy() - want), 2.0 ** -8 * np.abs(want) + 2.0 ** -15 * spread
    assert (diff <= slack).all(), (diff / slack).max()


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
def test_what_the_bounds_hold_for(kind):
    """Keys in bf16 lie inside; keys in 4 bits may lie outside, by their own rounding: half the widest gap of two codes, a sixth of the row's
    largest value, and half a step of bf16."""
    torch, ops = torch_ops()
    d, page = 48, 64
    k = torch.randn(3 * page + 1, 2, d, generator=torch.Generator().manual_seed(5))
    k[-1, 0, :] = 0.3
    k[-1, 0, 0] = 6  # (0.3 becomes 0.5, alone on the last page)
    cache = ops.cache_new(4, 2, d, page=page, kind=kind)
    table, past = torch.arange(4, dtype=torch.int32, device="cuda")[None], torch.zeros(1, dtype=torch.int32, device="cuda")
    ops.cache_append(cache, k.cuda(), k.cuda(), table, past)
    for rows, place in ((k[:3 * page], np.arange(3 * page) // page), (k[-1:], np.array([3]))):
        at = torch.tensor([int(place[0]) * page], dtype=torch.int32, device="cuda")
        held, _ = ops.cache_read(cache, table, at, len(rows))
        held, bounds = held.cpu().numpy(), cache.bounds.float().cpu().numpy()[place]
        lo, hi = bounds[:, :, 0, :d], bounds[:, :, 1, :d]
        over = np.maximum(held - hi, lo - held)
        if kind == "bf16":
            assert (over <= 0).all()
        else:
            m = rows.abs().amax(-1, keepdim=True).numpy()
            assert (over <= m * (1 / 6 + 2.0 ** -8)).all()
            assert len(rows) > 1 or (held[0, 0, 1:] == 0.5).all() and (over[0, 0, 1:] > 0.19).all()
