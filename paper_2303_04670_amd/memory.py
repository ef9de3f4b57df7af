"""A memory over the windows of event streams, of the sequence operators (ops.py).

An incremental net answers every window of a stream by itself.  `Memory` is a stack of layers behind it that
remembers: each layer keeps one matrix per head and stream (the state of the gated delta rule), reads and rewrites
it with every window's features, and costs the same after the millionth window as after the first.  Of a layer:

    p  = W_in  rows8(norm(x))                 q, k, v, gate z, decays and strengths in one product of 8-bit integers
    o  = delta_rule(p, state)                 states of the streams named by `slots`, rewritten in place
    y  = W_out rows8(norm(o per head) * silu(z))
    x += res_scale * norm(y)                  in one kernel with the next layer's norm and its 8-bit rows

    python -m paper_2303_04670_amd.memory     a classifier's streams with a memory behind them, timed

Weights are seeded random numbers (as the nets of workloads.py); nothing here is trained.
"""
from __future__ import annotations

from typing import NamedTuple

import numpy as np
import torch

from . import ops
from .evconv import ERR_INVALID_ARG, EvConvError


class Layer(NamedTuple):
    w_in: ops.QuantRows  # q, k, v, z, decays, strengths (and rows of zeros up to a multiple of eight)
    w_out: ops.QuantRows
    pre_norm: torch.Tensor  # of x
    head_norm: torch.Tensor  # of a head's o
    post_norm: torch.Tensor  # of y
    res_scale: torch.Tensor
    a_scale: torch.Tensor  # decay of a window: exp(-a_scale * softplus(projection + dt_bias))
    dt_bias: torch.Tensor


class Memory:
    """`layers` layers over features of `dim` values, then a linear head of `n_out` values.  One state per stream
    and layer: fp32 [n_streams, heads_v, d_k, d_v], zero at first."""

    def __init__(self, dim, n_streams, n_out, layers=2, heads_k=2, heads_v=4, d_k=64, d_v=64, dtype=torch.bfloat16, device="cuda:0",
                 seed=0):
        self.dim, self.n_streams, self.dtype, self.device = dim, n_streams, dtype, torch.device(device)
        self.heads_k, self.heads_v, self.d_k, self.d_v = heads_k, heads_v, d_k, d_v
        rng = np.random.default_rng(seed)
        wide_k, wide_v = heads_k * d_k, heads_v * d_v
        self.columns = np.cumsum([0, wide_k, wide_k, wide_v, wide_v, heads_v, heads_v]).tolist()
        padded = -(-self.columns[-1] // 8) * 8  # (rows of p whose slices can be read in vectors)
        self.weights = []  # of every layer in fp32 on the host, by name: what the quantised ones were made from
        self.layers = []
        for _ in range(layers):
            w = {"w_in": rng.standard_normal((padded, dim)) / np.sqrt(dim), "w_out": rng.standard_normal((dim, wide_v)) / np.sqrt(wide_v),
                 "pre_norm": rng.uniform(0.5, 1.5, dim), "head_norm": rng.uniform(0.5, 1.5, d_v), "post_norm": rng.uniform(0.5, 1.5, dim),
                 "res_scale": np.full(dim, 0.5), "a_scale": rng.uniform(0.02, 0.2, heads_v), "dt_bias": rng.uniform(-2, 0, heads_v)}
            w["w_in"][self.columns[-1]:] = 0
            self.weights.append({n: a.astype(np.float32) for n, a in w.items()})
            self.layers.append(Layer(**{n: self._rows(a) if n.startswith("w_") else self._of(a) for n, a in self.weights[-1].items()}))
        self.weights.append({n: a.astype(np.float32) for n, a in (
            ("norm", rng.uniform(0.5, 1.5, dim)), ("head", rng.standard_normal((n_out, dim)) / np.sqrt(dim)), ("bias", np.zeros(n_out)))})
        self.norm, self.bias = self._of(self.weights[-1]["norm"]), self._of(self.weights[-1]["bias"])
        self.head = self._rows(self.weights[-1]["head"])
        self.states = [torch.zeros(n_streams, heads_v, d_k, d_v, device=self.device) for _ in range(layers)]

    def _of(self, a):
        return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(self.device)

    def _rows(self, a):
        return ops.quantize_rows(self._of(a))

    def forget(self, slots=None):
        """Streams (all of them) begin anew.  slots: as in a window's call, or whatever else indexes the streams."""
        if slots is None or isinstance(slots, slice) or torch.is_tensor(slots) and slots.dtype == torch.bool:
            for state in self.states:
                state[slots if slots is not None else slice(None)] = 0
            return
        # (on the GPU alone: which streams are meant is not waited for, and a slot that is none is not an index from the end)
        slots, n = torch.as_tensor(slots, device=self.device).reshape(-1).long(), self.n_streams
        meant = torch.zeros(n + 1, dtype=torch.bool, device=self.device)
        meant.index_fill_(0, torch.where((slots >= 0) & (slots < n), slots, n), True)
        rows = slots.clamp(0, n - 1)
        for state in self.states:
            state[rows] = torch.where(meant[rows][:, None, None, None], torch.zeros((), device=self.device), state[rows])

    def __call__(self, x, slots=None, seq_offsets=None):
        """Features [windows, dim] -> [windows, n_out].  By default one window of every stream, in their order; with
        slots (int32 [n], a stream at most once; negative: nothing is remembered) one window of each of those; with
        seq_offsets (int32 [n + 1]) windows seq_offsets[i] .. seq_offsets[i + 1] are the next ones of stream slots[i]."""
        if x.dtype != self.dtype:  # (found by the last call of a layer only, behind the one that rewrites its states)
            raise EvConvError(ERR_INVALID_ARG, f"features are {x.dtype}, the memory's {self.dtype}")
        to = self.columns
        n_seq = None if slots is not None or seq_offsets is not None else self.n_streams
        rows = ops.block_norm(x, pre_norm=True, pre_weight=self.layers[0].pre_norm, want="q").q
        for i, layer in enumerate(self.layers):
            p = ops.quant_matmul(rows, layer.w_in, out_dtype=self.dtype)
            q, k, v, z, a, b = (p[:, to[j]:to[j + 1]] for j in range(6))
            o, _ = ops.delta_rule(q.unflatten(1, (self.heads_k, self.d_k)), k.unflatten(1, (self.heads_k, self.d_k)),
                                  v.unflatten(1, (self.heads_v, self.d_v)), a, b, self.states[i], state_out=self.states[i],
                                  seq_offsets=seq_offsets, slots=slots, n_seq=n_seq, normalize=True,
                                  a_scale=layer.a_scale, dt_bias=layer.dt_bias)
            rows = ops.block_norm(None, o.flatten(1), z, post_weight=layer.head_norm, group=self.d_v, want="q").q
            y = ops.quant_matmul(rows, layer.w_out, out_dtype=self.dtype)
            following = self.layers[i + 1].pre_norm if i + 1 < len(self.layers) else self.norm
            x, _, rows = ops.block_norm(x, y, post_weight=layer.post_norm, res_scale=layer.res_scale, pre_norm=True,
                                        pre_weight=following, want="xq")
        return ops.quant_matmul(rows, self.head, bias=self.bias)


def main():
    import argparse
    import time

    from . import evconv as ev
    from . import workloads as wl
    cli = argparse.ArgumentParser(prog="python -m paper_2303_04670_amd.memory", description=__doc__.split("\n")[0])
    cli.add_argument("--streams", type=int, default=4)
    cli.add_argument("--windows", type=int, default=20)
    cli.add_argument("--features", type=int, default=128, help="outputs of the classifier, the memory's inputs")
    cli.add_argument("--classes", type=int, default=101)
    cli.add_argument("--layers", type=int, default=2)
    cli.add_argument("--heads", type=int, default=4)
    cli.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    arg = cli.parse_args()
    net = ev.EvConvNet(wl.net_resnet18(h=64, w=64, width=16, n_classes=arg.features), n_streams=arg.streams)
    memory = Memory(arg.features, arg.streams, arg.classes, arg.layers, max(arg.heads // 2, 1), arg.heads,
                    dtype=torch.bfloat16 if arg.dtype == "bf16" else torch.float32)
    streams = [list(wl.stream_histogram(1004 + s, 64, 64, arg.windows)) for s in range(arg.streams)]
    frames = [torch.from_numpy(np.stack(f) if arg.streams > 1 else f[0]).cuda() for f in zip(*streams)]
    features = torch.empty(arg.streams, arg.features, device="cuda", dtype=memory.dtype)
    times = []
    for i, frame in enumerate(frames):
        start = time.perf_counter()
        net.reset(frame) if i == 0 else net.step_frame(frame)
        for s in range(arg.streams):
            features[s] = net.outputs(s)[0]["y"].view(-1)
        torch.cuda.synchronize()
        seen = time.perf_counter()
        if i == 0:  # a window's calls, five a layer and two more, are recorded once
            classes = memory(features)
            torch.cuda.synchronize()
            window = torch.cuda.CUDAGraph()
            with torch.cuda.graph(window):
                classes = memory(features)
            continue
        window.replay()
        torch.cuda.synchronize()
        times.append((seen - start, time.perf_counter() - seen))
    of_net, of_memory = np.median(np.array(times), axis=0) * 1e6
    print(f"{arg.streams} streams, {len(frames)} windows: net {of_net:.0f} us, memory of {arg.layers} layers {of_memory:.0f} us a window; "
          f"classes {classes.argmax(dim=1).tolist()}")
    net.destroy()


if __name__ == "__main__":
    main()
