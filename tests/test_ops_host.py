"""Host-side checks of the sequence operators' C ABI that need no GPU: exported symbols, refusals (all
made before any GPU work), workspace sizes, and the 64-bit references against other forms of their formulas."""
import ctypes
import os
import re

import numpy as np
import pytest

import ops_ref
from paper_2303_04670_amd import evconv as ev
from paper_2303_04670_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20  # an address that no refused call reads


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "evconv_ops.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert set(re.findall(r"\b(evconv_[a-z_]+)\s*\(", text)) == set(ops.EXPORTS)
    for name in ops.EXPORTS:
        assert hasattr(ev.lib(), name), name


def delta_args(**kw):
    a = ops.DeltaArgs(abi_version=ops.ABI_VERSION, dtype=0, gate_dtype=0, heads_k=2, heads_v=4, d_k=64, d_v=64, n_seq=2, n_slots=2,
                      n_tokens=200, scale=1.0, o=FAKE, o_token_stride=256, o_head_stride=64, state_in=FAKE, state_out=FAKE)
    for h, heads in (("q", 2), ("k", 2), ("v", 4)):
        setattr(a, h, ops.Heads(FAKE, heads * 64, 64))
    a.gate = a.beta = ops.Heads(FAKE, 4, 1)
    for name, value in kw.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(abi_version=7), ev.ERR_BAD_DESC), (dict(dtype=2), ev.ERR_INVALID_ARG), (dict(gate_dtype=5), ev.ERR_INVALID_ARG),
    (dict(flags=8), ev.ERR_INVALID_ARG), (dict(heads_v=3), ev.ERR_SHAPE), (dict(heads_k=0), ev.ERR_SHAPE), (dict(d_k=0), ev.ERR_SHAPE),
    (dict(d_k=257), ev.ERR_UNSUPPORTED), (dict(d_v=300), ev.ERR_UNSUPPORTED), (dict(heads_v=2048), ev.ERR_UNSUPPORTED),
    (dict(n_seq=0), ev.ERR_SHAPE), (dict(n_seq=70000, n_slots=70000), ev.ERR_UNSUPPORTED), (dict(n_seq=3, n_slots=3), ev.ERR_SHAPE),
    (dict(n_tokens=-2), ev.ERR_SHAPE), (dict(n_tokens=1 << 31), ev.ERR_UNSUPPORTED), (dict(n_slots=1), ev.ERR_SHAPE),
    (dict(q=ops.Heads(None, 128, 64)), ev.ERR_INVALID_ARG), (dict(o=None), ev.ERR_INVALID_ARG),
    (dict(flags=ops.DELTA_RAW_GATES), ev.ERR_INVALID_ARG),
    (dict(n_tokens=(1 << 31) - 100, heads_k=1, heads_v=1024), ev.ERR_UNSUPPORTED)])
def test_delta_rule_refusals(change, status):
    n = ctypes.c_size_t(77)
    a = delta_args(**change)
    assert ops._calls().evconv_delta_rule_workspace(ctypes.byref(a), ctypes.byref(n)) == status
    assert n.value == 77
    assert ops._calls().evconv_delta_rule(ctypes.byref(a), FAKE, 1 << 40, None) == status
    assert ev.lib().evconv_last_error(None).decode().startswith("delta rule")


def test_delta_rule_workspace():
    L, n = ops._calls(), ctypes.c_size_t(0)

    def need(**kw):
        assert L.evconv_delta_rule_workspace(ctypes.byref(delta_args(**kw)), ctypes.byref(n)) == ev.OK
        return n.value

    assert need(n_tokens=2) == 0 and need(n_tokens=0) == 0 and need(n_tokens=2, state_in=None, state_out=None) == 0
    small, large = need(n_tokens=256), need(n_tokens=256 * 64)
    assert 0 < small < large < 128 * small
    a = delta_args(n_tokens=256)
    for ws, size in ((None, small), (FAKE, small - 1), (FAKE + 8, small)):
        assert L.evconv_delta_rule(ctypes.byref(a), ws, size, None) == ev.ERR_WORKSPACE
    assert str(small) in ev.lib().evconv_last_error(None).decode()
    assert L.evconv_delta_rule_workspace(None, ctypes.byref(n)) == ev.ERR_INVALID_ARG
    assert L.evconv_delta_rule_workspace(ctypes.byref(a), None) == ev.ERR_INVALID_ARG
    assert L.evconv_delta_rule(None, None, 0, None) == ev.ERR_INVALID_ARG


@pytest.mark.parametrize("n", [256, 4096, 65535])
@pytest.mark.parametrize("dtype", [0, 1])
def test_delta_rule_workspace_of_single_tokens_with_offsets(n, dtype):
    """Room for the chunks that so many tokens can have: sequences of up to four go token by token, so at most a fifth of the tokens begin one."""
    kw = dict(dtype=dtype, heads_k=8, heads_v=16, d_k=192, d_v=128)  # (keys of which both types need a workspace)
    one, some = ctypes.c_size_t(0), ctypes.c_size_t(0)
    L = ops._calls()
    assert L.evconv_delta_rule_workspace(ctypes.byref(delta_args(n_tokens=64, n_seq=1, n_slots=1, **kw)), ctypes.byref(one)) == ev.OK
    assert L.evconv_delta_rule_workspace(ctypes.byref(delta_args(n_tokens=n, n_seq=n, n_slots=n, seq_offsets=FAKE, **kw)), ctypes.byref(some)) == ev.OK
    assert 0 < some.value <= (n // 64 + n // 5 + 1) * (one.value + 512)
    assert L.evconv_delta_rule_workspace(ctypes.byref(delta_args(n_tokens=n * 64, n_seq=1, n_slots=1, seq_offsets=FAKE, **kw)), ctypes.byref(some)) == ev.OK
    assert some.value <= (n + 1) * (one.value + 512)  # (one long sequence: its chunks)


@pytest.mark.parametrize("given", [dict(), dict(a_scale=FAKE), dict(dt_bias=FAKE)])
@pytest.mark.parametrize("n", [0, 200])
def test_delta_rule_raw_gates_need_their_parameters(n, given):
    """Without tokens too: the states are handed on by the kernel that goes token by token, which reads them first."""
    size = ctypes.c_size_t(77)
    a = delta_args(n_tokens=n, flags=ops.DELTA_RAW_GATES, **given)
    assert ops._calls().evconv_delta_rule_workspace(ctypes.byref(a), ctypes.byref(size)) == ev.ERR_INVALID_ARG and size.value == 77
    assert ops._calls().evconv_delta_rule(ctypes.byref(a), FAKE, 1 << 40, None) == ev.ERR_INVALID_ARG
    a.a_scale = a.dt_bias = FAKE
    assert ops._calls().evconv_delta_rule_workspace(ctypes.byref(a), ctypes.byref(size)) == ev.OK


@pytest.mark.parametrize("kw,few,many", [
    # single tokens: 64 threads to a sequence, head and 32 columns
    (dict(n_tokens=65535, d_v=64), 512, 1024),
    # with offsets the chunks' launch stands behind it: eight waves to each, which end at once
    (dict(n_tokens=65535, d_v=64, seq_offsets=FAKE), 64, 1024),
    # chunks: eight (twelve) waves to a sequence and head of one launch
    (dict(n_tokens=7 * 65535, dtype=1), 128, 256), (dict(n_tokens=7 * 65535, dtype=1, seq_offsets=FAKE), 128, 256), (dict(n_tokens=7 * 65535, dtype=1, d_v=65), 64, 128),
    (dict(n_tokens=13 * 65535), 128, 256), (dict(n_tokens=13 * 65535, d_k=200, d_v=200), 64, 128)])
def test_delta_rule_refuses_more_than_a_launch_takes(kw, few, many):
    """HIP counts a launch's threads in 32 bits; nothing has been enqueued when a call is refused for it."""
    n, kw = ctypes.c_size_t(77), dict(n_seq=65535, n_slots=65535, **kw)
    L = ops._calls()
    assert L.evconv_delta_rule_workspace(ctypes.byref(delta_args(heads_k=few, heads_v=few, **kw)), ctypes.byref(n)) == ev.OK
    for heads in (many, 1024):
        a = delta_args(heads_k=heads, heads_v=heads, **kw)
        assert L.evconv_delta_rule_workspace(ctypes.byref(a), ctypes.byref(n)) == ev.ERR_UNSUPPORTED
        assert L.evconv_delta_rule(ctypes.byref(a), FAKE, 1 << 50, None) == ev.ERR_UNSUPPORTED


def norm_args(**kw):
    a = ops.NormArgs(abi_version=ops.ABI_VERSION, dim=512, group=512, rows=4, eps=1e-6, x=FAKE, branch=FAKE, x_out=FAKE,
                     x_stride=512, branch_stride=512, x_out_stride=512)
    for name, value in kw.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(abi_version=0), ev.ERR_BAD_DESC), (dict(dtype=2), ev.ERR_INVALID_ARG), (dict(norm=2), ev.ERR_INVALID_ARG),
    (dict(gate_act=3, gate=FAKE), ev.ERR_INVALID_ARG), (dict(gate_act=1), ev.ERR_INVALID_ARG), (dict(gate=FAKE), ev.ERR_INVALID_ARG),
    (dict(dim=0), ev.ERR_SHAPE), (dict(group=100), ev.ERR_SHAPE), (dict(rows=-1), ev.ERR_SHAPE), (dict(rows=1 << 31), ev.ERR_UNSUPPORTED),
    (dict(dim=16392, group=16392), ev.ERR_UNSUPPORTED), (dict(dim=2048, group=1024), ev.ERR_UNSUPPORTED),
    (dict(group=4), ev.ERR_UNSUPPORTED), (dict(eps=-1.0), ev.ERR_INVALID_ARG), (dict(eps=float("nan")), ev.ERR_INVALID_ARG),
    (dict(x=None, branch=None), ev.ERR_INVALID_ARG), (dict(x_out=None), ev.ERR_INVALID_ARG),
    (dict(branch=None, res_scale=FAKE), ev.ERR_INVALID_ARG), (dict(pre_weight=FAKE), ev.ERR_INVALID_ARG),
    (dict(q=FAKE, q_stride=512), ev.ERR_INVALID_ARG), (dict(q=FAKE, q_scale=FAKE, q_stride=500), ev.ERR_SHAPE),
    (dict(q=FAKE, q_scale=FAKE, q_stride=640), ev.ERR_SHAPE), (dict(q=FAKE + 4, q_scale=FAKE, q_stride=512), ev.ERR_SHAPE)])
def test_block_norm_refusals(change, status):
    assert ops._calls().evconv_block_norm(ctypes.byref(norm_args(**change)), None) == status
    assert ev.lib().evconv_last_error(None).decode().startswith("block norm")


def quant_args(**kw):
    a = ops.QuantArgs(abi_version=ops.ABI_VERSION, n=8, k=100, m=4, a=FAKE, b=FAKE, a_stride=128, b_stride=128, a_scale=FAKE,
                      b_scale=FAKE, y=FAKE, y_stride=8)
    for name, value in kw.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change,status", [
    (dict(abi_version=2), ev.ERR_BAD_DESC), (dict(dtype=2), ev.ERR_INVALID_ARG), (dict(act=4), ev.ERR_INVALID_ARG),
    (dict(act=-1), ev.ERR_INVALID_ARG), (dict(n=0), ev.ERR_SHAPE), (dict(k=0), ev.ERR_SHAPE), (dict(m=-1), ev.ERR_SHAPE),
    (dict(k=131073, a_stride=131200, b_stride=131200), ev.ERR_UNSUPPORTED), (dict(m=1 << 31), ev.ERR_UNSUPPORTED),
    (dict(a=None), ev.ERR_INVALID_ARG), (dict(b_scale=None), ev.ERR_INVALID_ARG), (dict(a_stride=100), ev.ERR_SHAPE),
    (dict(k=129), ev.ERR_SHAPE), (dict(b=FAKE + 8), ev.ERR_SHAPE), (dict(y_stride=7), ev.ERR_SHAPE)])
def test_quant_matmul_refusals(change, status):
    assert ops._calls().evconv_quant_matmul(ctypes.byref(quant_args(**change)), None) == status
    assert ev.lib().evconv_last_error(None).decode().startswith("quantised product")


@pytest.mark.parametrize("m,n", [((1 << 31) - 1, 1), (1 << 23, 1 << 16), (1, (1 << 24) + 1)])
def test_quant_matmul_refuses_more_than_a_launch_takes(m, n):
    """Tiles of 256 x 256 with 512 threads each, fewer than 2^32 together; at most 2^24 columns."""
    a = quant_args(m=m, n=n, y_stride=n)
    assert ops._calls().evconv_quant_matmul(ctypes.byref(a), None) == ev.ERR_UNSUPPORTED


def test_nothing_to_do_is_ok():
    assert ops._calls().evconv_block_norm(ctypes.byref(norm_args(rows=0, x=None, branch=None)), None) == ev.OK
    assert ops._calls().evconv_quant_matmul(ctypes.byref(quant_args(m=0, a=None, y=None)), None) == ev.OK


def test_binding_refuses_tensors_on_the_host():
    import torch
    x = torch.zeros(2, 8)
    with pytest.raises(ev.EvConvError):
        ops.block_norm(x, want="q")
    with pytest.raises(ev.EvConvError):
        ops.delta_rule(x[:, None], x[:, None], x[:, None], x[:, :1], x[:, :1])
    with pytest.raises(ev.EvConvError) as e:
        ops.quant_matmul(ops.QuantRows(torch.zeros(2, 128, dtype=torch.int8), torch.zeros(2), 100),
                         ops.QuantRows(torch.zeros(2, 128, dtype=torch.int8), torch.zeros(2), 99))
    assert e.value.status == ev.ERR_SHAPE


def test_reference_delta_rule_solves_a_linear_system():
    """A token's state against the definition as a least-squares step, and a chunk against its matrix form."""
    rng = np.random.default_rng(3)
    n, dk, dv = 12, 5, 4
    q, k, v = rng.standard_normal((n, 1, dk)), rng.standard_normal((n, 1, dk)), rng.standard_normal((n, 1, dv))
    g, b, s0 = -rng.random((n, 1)), rng.random((n, 1)), rng.standard_normal((1, 1, dk, dv))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    o, s = ops_ref.delta_rule(q, k, v, g, b, s0, [(0, n)], 0.5)
    sums = np.cumsum(g[:, 0])
    decay = np.tril(np.exp(sums[:, None] - sums))
    a = np.tril(k[:, 0] @ k[:, 0].T, -1) * decay * b
    d = np.linalg.solve(np.eye(n) + a, b * (v[:, 0] - np.exp(sums)[:, None] * (k[:, 0] @ s0[0, 0])))
    want = np.exp(sums[-1]) * s0[0, 0] + (k[:, 0] * np.exp(sums[-1] - sums)[:, None]).T @ d
    np.testing.assert_allclose(s[0, 0], want, rtol=1e-11, atol=1e-12)
    p = (q[:, 0] @ k[:, 0].T) * decay
    np.testing.assert_allclose(o[:, 0], 0.5 * (np.exp(sums)[:, None] * (q[:, 0] @ s0[0, 0]) + p @ d), rtol=1e-10, atol=1e-11)
    # beta 1 and no decay: the state maps the last key to its value
    _, s = ops_ref.delta_rule(q, k, v, 0 * g, 0 * b + 1, s0, [(0, n)], 1.0)
    np.testing.assert_allclose(s[0, 0].T @ k[-1, 0], v[-1, 0], rtol=1e-12, atol=1e-12)


def test_reference_quantisation():
    x = np.array([[0, 0, 0], [1, -2, 0.5], [np.inf, 1, 2], [np.nan, 1, 2], [127, -63.5, 0.5]], np.float32)
    q, s = ops_ref.quantize_rows(x)
    assert q.tolist() == [[0, 0, 0], [64, -127, 32], [0, 0, 0], [0, 0, 0], [127, -64, 0]]
    assert s[0] == 0 and np.isnan(s[2:4]).all() and s[4] == 1
