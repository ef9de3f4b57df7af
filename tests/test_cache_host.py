"""Host-side checks of the paged cache's C ABI that need no GPU: refusals (all made before any GPU work), workspace sizes, the
structures' layout, and the 64-bit references against other forms of their formulas."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import ops_ref
from paper_2303_04670_amd import evconv as ev
from paper_2303_04670_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20  # an address that no refused call reads


def make(kind, cache=None, tokens=None, **kw):
    c = dict(kind=0, n_pages=50, heads=2, page=64, d=64, k=FAKE, v=FAKE, bounds=FAKE)
    c.update(cache or {})
    t = dict(n_seq=2, width=10, n_tokens=20, table=FAKE, table_stride=10, past=FAKE)
    t.update(tokens or {})
    rows = ops.Heads(FAKE, 4 * 64, 64)
    a = dict(abi_version=ops.ABI_VERSION, dtype=0, cache=ops.CacheArgs(**c), tokens=ops.TokenArgs(**t))
    if kind is ops.AppendArgs:
        a.update(heads_q=4, q=rows, k=rows, v=rows, q_out=FAKE, eps=1e-6)
    elif kind is ops.ReadArgs:
        a.update(k=FAKE, v=FAKE)
    elif kind is ops.AttendArgs:
        a.update(heads_q=4, causal=1, scale=0.1, q=rows, o=FAKE, o_token_stride=256, o_head_stride=64)
    else:
        a.update(heads_q=4, count=4, first=1, last=1, q=rows, selected=FAKE)
    a.update(kw)
    return kind(**a)


CACHE = [
    (dict(cache=dict(kind=2)), ev.ERR_INVALID_ARG), (dict(cache=dict(kind=1)), ev.ERR_INVALID_ARG), (dict(cache=dict(page=48)), ev.ERR_UNSUPPORTED),
    (dict(cache=dict(page=16)), ev.ERR_UNSUPPORTED), (dict(cache=dict(d=0)), ev.ERR_SHAPE), (dict(cache=dict(d=257)), ev.ERR_UNSUPPORTED),
    (dict(cache=dict(n_pages=0)), ev.ERR_SHAPE), (dict(cache=dict(k=None)), ev.ERR_INVALID_ARG), (dict(cache=dict(v=FAKE + 4)), ev.ERR_INVALID_ARG),
    (dict(cache=dict(bounds=FAKE + 8)), ev.ERR_INVALID_ARG), (dict(cache=dict(heads=0)), ev.ERR_SHAPE), (dict(cache=dict(heads=1025), heads_q=1025), ev.ERR_UNSUPPORTED),
    (dict(tokens=dict(n_seq=0)), ev.ERR_SHAPE), (dict(tokens=dict(n_seq=70000)), ev.ERR_UNSUPPORTED), (dict(tokens=dict(n_tokens=21)), ev.ERR_SHAPE),
    (dict(tokens=dict(n_tokens=-2)), ev.ERR_SHAPE), (dict(tokens=dict(n_tokens=1 << 31)), ev.ERR_UNSUPPORTED), (dict(tokens=dict(width=0)), ev.ERR_SHAPE),
    (dict(tokens=dict(width=1 << 24)), ev.ERR_UNSUPPORTED), (dict(tokens=dict(table=None)), ev.ERR_INVALID_ARG), (dict(tokens=dict(past=None)), ev.ERR_INVALID_ARG),
    (dict(abi_version=7), ev.ERR_BAD_DESC), (dict(dtype=2), ev.ERR_INVALID_ARG)]
APPEND = [
    (dict(heads_q=-1), ev.ERR_SHAPE), (dict(heads_q=2000), ev.ERR_UNSUPPORTED), (dict(rot=3, freqs=FAKE), ev.ERR_SHAPE), (dict(rot=66, freqs=FAKE), ev.ERR_SHAPE),
    (dict(rot=64), ev.ERR_INVALID_ARG), (dict(pairs=2), ev.ERR_INVALID_ARG), (dict(eps=-1.0), ev.ERR_INVALID_ARG), (dict(eps=float("nan")), ev.ERR_INVALID_ARG),
    (dict(k=ops.Heads(None, 64, 64)), ev.ERR_INVALID_ARG), (dict(q_out=None), ev.ERR_INVALID_ARG)]
ATTEND = [
    (dict(heads_q=3), ev.ERR_SHAPE), (dict(heads_q=0), ev.ERR_SHAPE), (dict(heads_q=1026), ev.ERR_UNSUPPORTED), (dict(causal=2), ev.ERR_INVALID_ARG),
    (dict(window=-1), ev.ERR_INVALID_ARG), (dict(window=5, causal=0), ev.ERR_INVALID_ARG), (dict(window=5, selected=FAKE, count=3), ev.ERR_INVALID_ARG),
    (dict(selected=FAKE), ev.ERR_SHAPE), (dict(selected=FAKE, count=70000), ev.ERR_UNSUPPORTED), (dict(max_len=-1), ev.ERR_INVALID_ARG),
    (dict(scale=0.0), ev.ERR_INVALID_ARG), (dict(scale=-1.0), ev.ERR_INVALID_ARG), (dict(scale=float("nan")), ev.ERR_INVALID_ARG),
    (dict(scale=float("inf")), ev.ERR_INVALID_ARG), (dict(o=None), ev.ERR_INVALID_ARG)]
SELECT = [
    (dict(heads_q=3), ev.ERR_SHAPE), (dict(count=0), ev.ERR_SHAPE), (dict(count=65537), ev.ERR_UNSUPPORTED), (dict(first=-1), ev.ERR_INVALID_ARG),
    (dict(last=0), ev.ERR_INVALID_ARG), (dict(first=3, last=2), ev.ERR_INVALID_ARG), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), ev.ERR_INVALID_ARG),
    (dict(cache=dict(bounds=None)), ev.ERR_INVALID_ARG), (dict(selected=None), ev.ERR_INVALID_ARG), (dict(max_len=-5), ev.ERR_INVALID_ARG)]


@pytest.mark.parametrize("kind,change,status", [(k, *c) for k, more in ((ops.AppendArgs, APPEND), (ops.ReadArgs, []), (ops.AttendArgs, ATTEND), (ops.SelectArgs, SELECT))
                                                for c in CACHE + more if not (k is ops.ReadArgs and "heads_q" in c[0])])
def test_refusals(kind, change, status):
    L, a, n = ops._calls(), make(kind, **change), ctypes.c_size_t(77)
    if kind is ops.AppendArgs:
        assert L.evconv_cache_append(ctypes.byref(a), None) == status
    elif kind is ops.ReadArgs:
        assert L.evconv_cache_read(ctypes.byref(a), None) == status
    else:
        size, call = (L.evconv_cache_attend_workspace, L.evconv_cache_attend) if kind is ops.AttendArgs else (L.evconv_cache_select_workspace, L.evconv_cache_select)
        assert size(ctypes.byref(a), ctypes.byref(n)) == status and n.value == 77
        assert call(ctypes.byref(a), FAKE, 1 << 40, None) == status
        assert size(ctypes.byref(a), None) == ev.ERR_INVALID_ARG and size(None, ctypes.byref(n)) == ev.ERR_INVALID_ARG
    assert ev.lib().evconv_last_error(None).decode().startswith("cache ")


def test_calls_without_tokens_do_nothing():
    L, n, none = ops._calls(), ctypes.c_size_t(5), dict(n_tokens=0, table=None, past=None)
    empty = dict(cache=dict(k=None, v=None, bounds=None), tokens=none)
    assert L.evconv_cache_append(ctypes.byref(make(ops.AppendArgs, **empty)), None) == ev.OK
    assert L.evconv_cache_read(ctypes.byref(make(ops.ReadArgs, **empty)), None) == ev.OK
    for kind, size, call in ((ops.AttendArgs, L.evconv_cache_attend_workspace, L.evconv_cache_attend), (ops.SelectArgs, L.evconv_cache_select_workspace, L.evconv_cache_select)):
        a = make(kind, **empty)
        assert size(ctypes.byref(a), ctypes.byref(n)) == ev.OK and n.value == 0
        assert call(ctypes.byref(a), None, 0, None) == ev.OK


def test_workspace_is_asked_for():
    L, n = ops._calls(), ctypes.c_size_t(0)

    def attend(**kw):
        a = make(ops.AttendArgs, **kw)
        assert L.evconv_cache_attend_workspace(ctypes.byref(a), ctypes.byref(n)) == ev.OK
        if n.value:
            for ws, size in ((None, 0), (FAKE, n.value - 1), (FAKE + 16, n.value)):
                assert L.evconv_cache_attend(ctypes.byref(a), ws, size, None) == ev.ERR_WORKSPACE
        return n.value
    step, long = dict(n_tokens=2), dict(n_tokens=2, width=100000)
    assert attend(tokens=step, max_len=200) == 0                    # one workgroup has all of a row's tokens
    assert attend(tokens=long) > 0                                  # several
    assert attend(tokens=long, max_len=300) == 0                    # none of them is that long
    assert attend(tokens=long, window=100) == 0
    assert attend(tokens=long, selected=FAKE, count=2) == 0
    a = make(ops.SelectArgs)
    assert L.evconv_cache_select_workspace(ctypes.byref(a), ctypes.byref(n)) == ev.OK and n.value == 20 * 2 * 12 * 4
    assert L.evconv_cache_select(ctypes.byref(a), FAKE, n.value - 1, None) == ev.ERR_WORKSPACE


def test_structures_have_the_header_s_layout(tmp_path):
    names = {"AppendArgs": "evconv_append_args", "ReadArgs": "evconv_read_args", "AttendArgs": "evconv_attend_args", "SelectArgs": "evconv_select_args",
             "CacheArgs": "evconv_cache", "TokenArgs": "evconv_tokens"}
    lines = []
    for py, c in names.items():
        lines.append(f'printf("%zu ", sizeof({c}));')
        lines += [f'printf("%zu ", offsetof({c}, {field}));' for field, _ in getattr(ops, py)._fields_]
    source = tmp_path / "layout.c"
    source.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "evconv_ops.h"\nint main(void) {' + "\n".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "layout"), str(source)], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for py in names:
        of = getattr(ops, py)
        want += [ctypes.sizeof(of)] + [getattr(of, field).offset for field, _ in of._fields_]
    assert got == want


def test_binding_refuses_before_the_library():
    torch = pytest.importorskip("torch")
    cache = ops.cache_new(4, 2, 40, device="cpu")
    assert cache.k.shape == (4, 2, 64, 64) and cache.v.shape == (4, 2, 64, 64) and cache.bounds.shape == (4, 2, 2, 64)
    four = ops.cache_new(4, 2, 100, page=32, kind="fp4", bounds=False, device="cpu")
    assert four.k.shape == (4, 2, 32, 64) and four.v.shape == (4, 2, 128, 16) and four.k_scale.shape == (4, 2, 32) and four.bounds is None
    x, table, past = torch.zeros(2, 2, 40), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: ops.cache_append(cache, x, x, table, past), lambda: ops.cache_read(cache, table, past, 2),
                 lambda: ops.cache_attend(x, cache, table, past), lambda: ops.cache_select(x, cache, table, past, 3),
                 lambda: ops.cache_new(4, 2, 300, device="cpu"), lambda: ops.cache_new(4, 2, 40, kind="int4", device="cpu")):
        with pytest.raises(ev.EvConvError):
            call()


# ---- the references

def test_numbers_out_of_range_are_refused_by_the_binding():
    """What would fail in an allocation or does not fit its field is refused like any other argument."""
    torch = pytest.importorskip("torch")
    q, cache = torch.zeros(1, 4, 64), ops.Cache(*[torch.zeros(1)] * 5, 64)
    table, past = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for count, status in ((-1, ev.ERR_SHAPE), (0, ev.ERR_SHAPE), (65537, ev.ERR_UNSUPPORTED), (1 << 40, ev.ERR_UNSUPPORTED)):
        with pytest.raises(ev.EvConvError) as e:
            ops.cache_select(q, cache, table, past, count)
        assert e.value.status == status and "count" in str(e.value)
    with pytest.raises(ev.EvConvError) as e:
        ops.cache_read(cache, table, past, -1)
    assert e.value.status == ev.ERR_SHAPE
    fields = [0] * len(ops._flat(ops.AttendArgs)._fields_)
    window = [name for name, _ in ops._flat(ops.AttendArgs)._fields_].index("window")
    assert len(ops._attend_args(*fields)) == ctypes.sizeof(ops.AttendArgs)
    fields[window] = 1 << 31
    with pytest.raises(ev.EvConvError) as e:
        ops._attend_args(*fields)
    assert e.value.status == ev.ERR_INVALID_ARG


def test_fp4_reference_against_a_search():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal((50, 32)), np.zeros((1, 32)), rng.integers(-24, 25, (50, 32)) / 4]).astype(np.float32)
    code, scale = ops_ref.fp4_rows(x)
    value = ops_ref.fp4_values(code, scale)
    every = np.concatenate([ops_ref.LEVELS, -ops_ref.LEVELS]) * scale.astype(np.float64)[:, None]
    best = np.abs(x.astype(np.float64)[..., None] - every[:, None]).min(-1)
    assert (np.abs(value - x) <= best + 1e-6 * np.abs(x).max()).all()
    assert (value[50] == 0).all() and np.isnan(ops_ref.fp4_rows(np.float32([[1, np.inf]]))[1]).all()


def test_head_rows_reference_keeps_products_of_equal_distance():
    """A rotated query times a rotated key depends on how far they are apart."""
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((2, 1, 1, 10))
    freqs = [1.0, 0.3, 0.01]
    for pairs in ("halves", "neighbours"):
        got = [(ops_ref.head_rows(q, None, 0, freqs, pairs, [a + 7]) * ops_ref.head_rows(k, None, 0, freqs, pairs, [a])).sum() for a in (0, 5, 1e6)]
        assert np.allclose(got, got[0], atol=1e-8)


def test_attend_reference_against_a_loop():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 4, 5))
    seen = np.tril(np.ones((4, 4), bool), -1)
    got, _ = ops_ref.attend(q, k, v, 0.5, seen)
    for i in range(4):
        w = np.array([np.exp(0.5 * q[i] @ k[t]) for t in range(i)])
        assert np.allclose(got[i], (w[:, None] * v[:i]).sum(0) / w.sum() if i else 0)


def test_a_place_for_queries_needs_queries():
    """q_out without q would come back unwritten."""
    torch = pytest.importorskip("torch")
    x, cache = torch.zeros(1, 2, 40), ops.Cache(*[torch.zeros(1)] * 5, 40)
    table, past = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ev.EvConvError) as e:
        ops.cache_append(cache, x, x, table, past, q_out=torch.zeros_like(x))
    assert e.value.status == ev.ERR_INVALID_ARG and "q_out" in str(e.value)
