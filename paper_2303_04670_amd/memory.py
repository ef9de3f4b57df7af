"""A memory over the windows of event streams, of the sequence operators (ops.py).

An incremental net answers every window of a stream by itself.  `Memory` is a stack of layers behind it that
remembers: each layer keeps one matrix per head and stream (the state of the gated delta rule), reads and rewrites
it with every window's features, and costs the same after the millionth window as after the first.  Of a layer:

    p  = W_in  rows8(norm(x))                 q, k, v, gate z, decays and strengths in one product of 8-bit integers
    o  = delta_rule(p, state)                 states of the streams named by `slots`, rewritten in place
    y  = W_out rows8(norm(o per head) * silu(z))
    x += res_scale * norm(y)                  in one kernel with the next layer's norm and its 8-bit rows

A layer may look back instead (`recall`): its windows' keys and values stay in a paged cache, in 4 bits or bf16, and
o is attention over the stream's last `recall_windows` ones, whose pages go round, or over the best `recall_pages` pages of
all that fit:

    q  = cache_append(cache, norm, turn by the window's number, of p)
    o  = cache_attend(q, cache, the last windows or cache_select(q, cache))

    python -m paper_2303_04670_amd.memory     a classifier's streams with a memory behind them, timed

Weights are seeded random numbers (as the nets of workloads.py); nothing here is trained.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import numpy as np
import torch

from . import ops
from .evconv import ERR_INVALID_ARG, ERR_SHAPE, EvConvError


class Layer(NamedTuple):
    """Of a layer that looks back the decays and strengths, their scale and bias are absent; it has a cache, and norms of its heads."""
    w_in: ops.QuantRows  # q, k, v, z, decays, strengths (and rows of zeros up to a multiple of eight)
    w_out: ops.QuantRows
    pre_norm: torch.Tensor  # of x
    head_norm: torch.Tensor  # of a head's o
    post_norm: torch.Tensor  # of y
    res_scale: torch.Tensor
    a_scale: Optional[torch.Tensor]  # decay of a window: exp(-a_scale * softplus(projection + dt_bias))
    dt_bias: Optional[torch.Tensor]
    cache: Optional[ops.Cache] = None
    q_norm: Optional[torch.Tensor] = None
    k_norm: Optional[torch.Tensor] = None


class Windows(NamedTuple):
    """Whose the windows of a call are, for the layers that look back."""
    table: torch.Tensor  # of every sequence; one that is no stream's has no pages
    past: torch.Tensor
    seq_offsets: Optional[torch.Tensor]
    slots: Optional[torch.Tensor]
    number: torch.Tensor  # of every window, since its stream began
    new: object  # windows of every sequence, or 1
    left_out: Optional[torch.Tensor]  # windows of streams that bring too many


class Memory:
    """`layers` layers over features of `dim` values, then a linear head of `n_out` values.  One state per stream
    and layer: fp32 [n_streams, heads_v, d_k, d_v], zero at first.

    recall: numbers of the layers that look back, heads_v query heads on heads_k key heads of d_v channels, into a cache of kind
    recall_kind.  They see the last recall_windows windows of a stream, however long it is; or, with recall_pages,
    that many pages of 64 windows among the first recall_windows ones, which are all that is kept.  A stream brings `longest` windows at
    most in a call (what the pages that go round have room for beside the windows that are seen).  lifetime: of no effect."""

    PAGE = 64

    def __init__(self, dim, n_streams, n_out, layers=2, heads_k=2, heads_v=4, d_k=64, d_v=64, dtype=torch.bfloat16, device="cuda:0",
                 seed=0, recall=(), recall_kind="fp4", recall_windows=1024, recall_pages=None, longest=1024, lifetime=None):
        self.recall, self.recall_windows, self.recall_pages, self.longest = frozenset(recall), recall_windows, recall_pages, longest
        if self.recall:  # (nothing of a window may be refused behind the layers that have rewritten their states and caches)
            self._check_recall(layers, heads_k, heads_v)
        self.dim, self.n_streams, self.dtype, self.device = dim, n_streams, dtype, torch.device(device)
        self.heads_k, self.heads_v, self.d_k, self.d_v = heads_k, heads_v, d_k, d_v
        rng = np.random.default_rng(seed)
        wide_k, wide_v = heads_k * d_k, heads_v * d_v
        self.columns = np.cumsum([0, wide_k, wide_k, wide_v, wide_v, heads_v, heads_v]).tolist()
        padded = -(-self.columns[-1] // 8) * 8  # (rows of p whose slices can be read in vectors)
        self.weights = []  # of every layer in fp32 on the host, by name: what the quantised ones were made from
        self.layers, self.states = [], []
        if self.recall:
            self._make_pages()
        for i in range(layers):
            if i in self.recall:
                self._recall_layer(rng, recall_kind)
                continue
            w = {"w_in": rng.standard_normal((padded, dim)) / np.sqrt(dim), "w_out": rng.standard_normal((dim, wide_v)) / np.sqrt(wide_v),
                 "pre_norm": rng.uniform(0.5, 1.5, dim), "head_norm": rng.uniform(0.5, 1.5, d_v), "post_norm": rng.uniform(0.5, 1.5, dim),
                 "res_scale": np.full(dim, 0.5), "a_scale": rng.uniform(0.02, 0.2, heads_v), "dt_bias": rng.uniform(-2, 0, heads_v)}
            w["w_in"][self.columns[-1]:] = 0
            self.weights.append({n: a.astype(np.float32) for n, a in w.items()})
            self.layers.append(Layer(**{n: self._rows(a) if n.startswith("w_") else self._of(a) for n, a in self.weights[-1].items()}))
            self.states.append(torch.zeros(n_streams, heads_v, d_k, d_v, device=self.device))
        self.weights.append({n: a.astype(np.float32) for n, a in (
            ("norm", rng.uniform(0.5, 1.5, dim)), ("head", rng.standard_normal((n_out, dim)) / np.sqrt(dim)), ("bias", np.zeros(n_out)))})
        self.norm, self.bias = self._of(self.weights[-1]["norm"]), self._of(self.weights[-1]["bias"])
        self.head = self._rows(self.weights[-1]["head"])
        if self.recall:  # what the calls themselves refuse: a call of no windows
            self(torch.empty(0, dim, dtype=dtype, device=self.device), seq_offsets=torch.zeros(n_streams + 1, dtype=torch.int32, device=self.device))

    def _check_recall(self, layers, heads_k, heads_v):
        if self.recall - set(range(layers)):
            raise EvConvError(ERR_INVALID_ARG, f"layers {sorted(self.recall)} of {layers} look back")
        if self.recall_windows < 1 or self.longest < 1:
            raise EvConvError(ERR_INVALID_ARG, f"recall_windows {self.recall_windows}, longest {self.longest}: at least 1")
        if self.recall_pages is not None and not 2 <= self.recall_pages <= 65536:  # (the first and the newest are always among them)
            raise EvConvError(ERR_INVALID_ARG, f"recall_pages {self.recall_pages}: 2 to 65536, None for the last windows")
        if heads_k < 1 or heads_v < 1 or heads_v % heads_k:
            raise EvConvError(ERR_SHAPE, f"{heads_v} heads on {heads_k} key heads")
        if self._entries() * self.PAGE >= 1 << 30:
            raise EvConvError(ERR_SHAPE, f"recall_windows {self.recall_windows}, longest {self.longest}: a stream's pages have room for less than 2^30")

    def _own_pages(self):
        return -(-self.recall_windows // self.PAGE) if self.recall_pages is not None else -(-(self.recall_windows + self.longest) // self.PAGE) + 1

    def _entries(self):
        return self._own_pages() * (1 if self.recall_pages is not None else 2)

    def _make_pages(self):
        """Every stream's own pages: the last windows' in turns, or those of the first ones.  Pages that go round stand in the table twice: once
        a stream's place is so far on that its windows fill a round and what is seen, it goes back by a round, to the same pages, with as
        much behind it as is seen.  `windows` goes on, for the angles."""
        n, own = self.n_streams, self._own_pages()
        self.round = own * self.PAGE
        entry = torch.arange(self._entries(), dtype=torch.int32, device=self.device) % own
        self.n_pages = n * own
        self.table = (torch.arange(n, dtype=torch.int32, device=self.device)[:, None] * own + entry).contiguous()
        self.past = torch.zeros(n, dtype=torch.int32, device=self.device)  # tokens in the table's places
        self.windows = torch.zeros(n, dtype=torch.int64, device=self.device)  # since each stream began
        self.freqs = self._of(10000.0 ** (-np.arange(0, self.d_v // 2 * 2, 2) / max(self.d_v, 1)))

    def _recall_layer(self, rng, kind):
        dim, hk, hv, d = self.dim, self.heads_k, self.heads_v, self.d_v
        rows = 2 * hv * d + 2 * hk * d  # q, k, v, z
        padded = -(-rows // 8) * 8
        w = {"w_in": rng.standard_normal((padded, dim)) / np.sqrt(dim), "w_out": rng.standard_normal((dim, hv * d)) / np.sqrt(hv * d),
             "pre_norm": rng.uniform(0.5, 1.5, dim), "head_norm": rng.uniform(0.5, 1.5, d), "post_norm": rng.uniform(0.5, 1.5, dim),
             "res_scale": np.full(dim, 0.5), "q_norm": rng.uniform(0.5, 1.5, d), "k_norm": rng.uniform(0.5, 1.5, d)}
        w["w_in"][rows:] = 0
        self.weights.append({n: a.astype(np.float32) for n, a in w.items()})
        self.layers.append(Layer(**{n: self._rows(a) if n.startswith("w_") else self._of(a) for n, a in self.weights[-1].items()},
                                 a_scale=None, dt_bias=None, cache=ops.cache_new(self.n_pages, hk, d, page=self.PAGE, kind=kind,
                                                                                 bounds=self.recall_pages is not None, device=self.device)))
        self.states.append(None)

    def _of(self, a):
        return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(self.device)

    def _rows(self, a):
        return ops.quantize_rows(self._of(a))

    def forget(self, slots=None):
        """Streams (all of them) begin anew.  slots: as in a window's call, or whatever else indexes the streams."""
        states = [s for s in self.states if s is not None] + ([self.past, self.windows] if self.recall else [])
        if slots is None or isinstance(slots, slice) or torch.is_tensor(slots) and slots.dtype == torch.bool:
            for state in states:
                state[slots if slots is not None else slice(None)] = 0
            return
        # (on the GPU alone: which streams are meant is not waited for, and a slot that is none is not an index from the end)
        slots, n = torch.as_tensor(slots, device=self.device).reshape(-1).long(), self.n_streams
        meant = torch.zeros(n + 1, dtype=torch.bool, device=self.device)
        meant.index_fill_(0, torch.where((slots >= 0) & (slots < n), slots, n), True)
        rows = slots.clamp(0, n - 1)
        for state in states:
            state[rows] = torch.where(meant[rows].view(-1, *[1] * (state.dim() - 1)), torch.zeros((), dtype=state.dtype, device=self.device), state[rows])

    def __call__(self, x, slots=None, seq_offsets=None):
        """Features [windows, dim] -> [windows, n_out].  By default one window of every stream, in their order; with
        slots (int32 [n], a stream at most once; negative: nothing is remembered) one window of each of those; with
        seq_offsets (int32 [n + 1]) windows seq_offsets[i] .. seq_offsets[i + 1] are the next ones of stream slots[i].  (With layers that look
        back a stream that brings more than `longest` of them is left as it was and its windows answered by NaN; more than n times `longest` are refused.)"""
        if x.dtype != self.dtype:  # (found by the last call of a layer only, behind the one that rewrites its states)
            raise EvConvError(ERR_INVALID_ARG, f"features are {x.dtype}, the memory's {self.dtype}")
        to = self.columns
        if self.recall:
            whose = self._whose(x, slots, seq_offsets)
            seq_offsets, slots = whose.seq_offsets, whose.slots
        n_seq = None if slots is not None or seq_offsets is not None else self.n_streams
        rows = ops.block_norm(x, pre_norm=True, pre_weight=self.layers[0].pre_norm, want="q").q
        for i, layer in enumerate(self.layers):
            p = ops.quant_matmul(rows, layer.w_in, out_dtype=self.dtype)
            if layer.cache is not None:
                o, z = self._look_back(layer, p, whose)
                x, rows = self._behind(i, x, o, z)
                continue
            q, k, v, z, a, b = (p[:, to[j]:to[j + 1]] for j in range(6))
            o, _ = ops.delta_rule(q.unflatten(1, (self.heads_k, self.d_k)), k.unflatten(1, (self.heads_k, self.d_k)),
                                  v.unflatten(1, (self.heads_v, self.d_v)), a, b, self.states[i], state_out=self.states[i],
                                  seq_offsets=seq_offsets, slots=slots, n_seq=n_seq, normalize=True,
                                  a_scale=layer.a_scale, dt_bias=layer.dt_bias)
            x, rows = self._behind(i, x, o, z)
        y = ops.quant_matmul(rows, self.head, bias=self.bias)
        if self.recall:
            self._move_on(whose.new, slots)
            if whose.left_out is not None:
                y.masked_fill_(whose.left_out[:, None], float("nan"))
        return y

    def _behind(self, i, x, o, z):
        """What of a layer comes behind its heads: (x', 8-bit rows of the next layer's norm)."""
        layer = self.layers[i]
        rows = ops.block_norm(None, o.flatten(1), z, post_weight=layer.head_norm, group=self.d_v, want="q").q
        y = ops.quant_matmul(rows, layer.w_out, out_dtype=self.dtype)
        following = self.layers[i + 1].pre_norm if i + 1 < len(self.layers) else self.norm
        x, _, rows = ops.block_norm(x, y, post_weight=layer.post_norm, res_scale=layer.res_scale, pre_norm=True,
                                    pre_weight=following, want="xq")
        return x, rows

    def _whose(self, x, slots, seq_offsets):
        n = slots.numel() if slots is not None else seq_offsets.numel() - 1 if seq_offsets is not None else self.n_streams
        if n > self.n_streams or x.dim() != 2 or (seq_offsets is None and x.shape[0] != n) or (seq_offsets is not None and seq_offsets.numel() != n + 1):
            raise EvConvError(ERR_SHAPE, f"{tuple(x.shape)} windows of {n} sequences, {self.n_streams} streams")
        for t, name, size in ((slots, "slots", n), (seq_offsets, "seq_offsets", n + 1)):
            ops._packed(t, name, x.get_device(), torch.int32, (size,))
        new, left_out = 1, None
        if seq_offsets is not None:
            if x.shape[0] > n * self.longest:
                raise EvConvError(ERR_SHAPE, f"{x.shape[0]} windows of {n} sequences in a call: at most {self.longest} of each")
            # (what is out of range is cut off there, a pair that descends is an empty sequence: all layers have the same windows, and as many are past)
            seq_offsets = seq_offsets.clamp(0, x.shape[0]).cummax(0).values
            new = seq_offsets[1:] - seq_offsets[:-1]
            window = torch.arange(x.shape[0], dtype=torch.int32, device=self.device)
            whose = torch.searchsorted(seq_offsets[1:], window, right=True).clamp_(max=n - 1)
            if x.shape[0] > self.longest:  # (one of them may bring too many, which only the GPU knows)
                many = new > self.longest
                slots = torch.where(many, -1, torch.arange(n, dtype=torch.int32, device=self.device) if slots is None else slots)
                left_out = many[whose]
        table, past, number = self.table[:n], self.past[:n], self.windows[:n]
        if slots is not None:
            inside = (slots >= 0) & (slots < self.n_streams)
            at = slots.clamp(0, self.n_streams - 1).long()
            table, past, number = torch.where(inside[:, None], self.table[at], -1), torch.where(inside, self.past[at], 0), torch.where(inside, self.windows[at], 0)
        if seq_offsets is not None:
            number = number[whose] + (window - seq_offsets[whose])
        return Windows(table, past, seq_offsets, slots, number, new, left_out)

    def _look_back(self, layer, p, whose):
        """(o, z) of a layer over a cache."""
        table, past, seq_offsets, number = whose.table, whose.past, whose.seq_offsets, whose.number
        wide, narrow = self.heads_v * self.d_v, self.heads_k * self.d_v
        q, k, v, z = (p[:, a:b] for a, b in ((0, wide), (wide, wide + narrow), (wide + narrow, wide + 2 * narrow), (wide + 2 * narrow, 2 * (wide + narrow))))
        q, k, v = (t.unflatten(1, (-1, self.d_v)) for t in (q, k, v))
        q = ops.cache_append(layer.cache, k, v, table, past, q, seq_offsets=seq_offsets, q_norm=layer.q_norm, k_norm=layer.k_norm, freqs=self.freqs,
                             positions=number)
        if self.recall_pages is not None:
            pages = ops.cache_select(q, layer.cache, table, past, self.recall_pages, seq_offsets=seq_offsets)
            return ops.cache_attend(q, layer.cache, table, past, seq_offsets=seq_offsets, selected=pages), z
        return ops.cache_attend(q, layer.cache, table, past, seq_offsets=seq_offsets, window=self.recall_windows), z

    def _move_on(self, new, slots):
        """The call's windows are past."""
        if slots is not None:
            inside, at = (slots >= 0) & (slots < self.n_streams), slots.clamp(0, self.n_streams - 1).long()
            new = torch.where(inside, new, 0)
        for count in (self.past, self.windows):
            if slots is not None:
                count.index_add_(0, at, new.to(count.dtype))
            else:
                count[:len(new) if torch.is_tensor(new) else None] += new
        if self.recall_pages is not None:
            self.past.clamp_(max=self.round)  # (all that is kept)
        else:
            self.past.add_(self.past >= self.round + self.recall_windows, alpha=-self.round)


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
    cli.add_argument("--recall", type=int, nargs="*", default=[], metavar="LAYER", help="layers that look back into a cache of 4 bits")
    cli.add_argument("--recall-windows", type=int, default=1024, help="over so many windows")
    arg = cli.parse_args()
    net = ev.EvConvNet(wl.net_resnet18(h=64, w=64, width=16, n_classes=arg.features), n_streams=arg.streams)
    memory = Memory(arg.features, arg.streams, arg.classes, arg.layers, max(arg.heads // 2, 1), arg.heads,
                    dtype=torch.bfloat16 if arg.dtype == "bf16" else torch.float32, recall=arg.recall, recall_windows=arg.recall_windows)
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
