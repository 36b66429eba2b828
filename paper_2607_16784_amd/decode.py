"""A served model's decode step on the library's kernels, and its kernel trace
as the predictor takes it.

    model = DecodeModel(layers=4, width=1024, heads=8, kv_heads=2, head_dim=128,
                        hidden=2816)
    state = model.new_state(sequences=16, most_tokens=2048)
    y = model.step(x, state, new=1)                # x [tokens, width]
    library = trace_library([(model, state)])      # the shape of workloads.make_library

Weights are random: this is a workload, with the launches, bytes and arithmetic
of a model of that shape, not a trained one.
"""
from __future__ import annotations

import numpy as np
import torch

from . import api


def rotary_frequencies(rot, base=10000.0, scaling="none", factor=1.0, trained=4096):
    """(inv_freq float32 [rot / 2], rot_scale) of rm_rotary_append.

    The angles are those of Su et al. 2021.  scaling "linear" divides positions by
    `factor` (Chen et al. 2023); "ntk" raises the base so that the slowest pair
    turns `factor` times slower and the fastest as before; "parts" (Peng et al.
    2023) divides the pairs that turn fewer than once over `trained` positions,
    keeps those that turn more than 32 times and goes linearly between, with
    queries and keys scaled up by 0.1 ln(factor) + 1 each."""
    i = np.arange(0, rot, 2, dtype=np.float64) / rot
    scale = 1.0
    if scaling == "ntk" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    freq = base ** -i
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "parts":
        turns = trained * freq / (2 * np.pi)
        keep = np.clip((turns - 1.0) / 31.0, 0.0, 1.0)
        freq = freq / factor * (1 - keep) + freq * keep
        scale = 0.1 * np.log(factor) + 1.0 if factor > 1 else 1.0
    elif scaling not in ("none", "ntk"):
        raise ValueError(f"scaling: expected none, linear, ntk or parts, got {scaling!r}")
    return torch.tensor(freq, dtype=torch.float32), float(scale)


class DecodeModel:
    """`layers` layers: norm, projection, rotary append, attention, projection,
    gated residual between two norms, gated projection, projection."""

    def __init__(self, layers, width, heads, kv_heads, head_dim, hidden, group=128,
                 dtype=torch.bfloat16, codes=torch.int8, page_tokens=64, seed=0, device="cuda"):
        self.width, self.heads, self.kv_heads, self.head_dim = width, heads, kv_heads, head_dim
        self.group, self.dtype, self.codes, self.page_tokens = group, dtype, codes, page_tokens
        self.device = torch.device(device)
        gen = torch.Generator(device=device).manual_seed(seed)

        def projection(n, k):
            groups = -(-k // group)
            return {"codes": torch.randint(0, 256, (n, (k + 1) // 2), generator=gen, device=device,
                                           dtype=torch.uint8),
                    # codes are uniform over 16 steps around the zero 8: deviation 4.6
                    "scales": torch.full((n, groups), 1 / (4.6 * k ** 0.5), dtype=dtype,
                                         device=device)}

        def gain(n):
            return (1 + torch.randn(n, generator=gen, device=device) / 16).to(dtype)

        self.layers = [{
            "pre": gain(width), "qkv": projection((heads + 2 * kv_heads) * head_dim, width),
            "out": projection(width, heads * head_dim), "post": gain(width),
            "gate": torch.full((width,), 0.5, dtype=dtype, device=device),
            "mid": gain(width), "up": projection(2 * hidden, width),
            "down": projection(width, hidden)} for _ in range(layers)]
        self.last = gain(width)
        inv, self.rot_scale = rotary_frequencies(head_dim)
        self.inv_freq = inv.to(device)

    def new_state(self, sequences, most_tokens):
        """Empty caches, a table of pages for every sequence and lengths 0."""
        pages = -(-most_tokens // self.page_tokens)
        table = torch.arange(sequences * pages, dtype=torch.int32, device=self.device)
        return {"caches": [api.new_cache(sequences * pages, self.kv_heads, self.page_tokens,
                                         self.head_dim, self.codes, self.device)
                           for _ in self.layers],
                "table": table.reshape(sequences, pages),
                "lengths": torch.zeros(sequences, dtype=torch.int32, device=self.device),
                "status": api.new_status(self.device)}

    def calls(self, x, state, new=1):
        """The step's calls in order, each a (name, function of no argument).  x
        [sequences * new, width]: `new` tokens of every sequence, counted in
        state["lengths"] already."""
        n = state["table"].shape[0]
        offsets = None
        if new != 1:
            offsets = torch.arange(0, n * new + 1, new, dtype=torch.int32, device=self.device)
        seqs = dict(token_offsets=offsets, max_tokens=new, status=state["status"])
        h, kv, d = self.heads, self.kv_heads, self.head_dim
        now = {"x": x, "y": None}

        def linear(w, source, to, act="none"):
            def run():
                now[to] = api.rm_w4_linear(now[source], w["codes"], w["scales"], self.group,
                                           act=act)
            return run

        def norm(weight, gate=None, post=None):
            y = now["y"] is not None

            def run():
                now["x"], now["h"] = api.rm_norm_residual(
                    now["x0"], now["y"] if y else None, gate=gate, post_weight=post,
                    pre_weight=weight)
            return run

        def keep():
            now["x0"] = now["x"]

        def append(cache):
            def run():
                qkv = now["qkv"].view(n * new, h + 2 * kv, d)
                now["q"] = api.rm_rotary_append(
                    qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:], self.inv_freq, cache,
                    state["table"], state["lengths"], rot_scale=self.rot_scale, **seqs)
            return run

        def attend(cache):
            def run():
                now["a"] = api.rm_cache_attention(now["q"], cache, state["table"],
                                                  state["lengths"], **seqs).view(n * new, h * d)
            return run

        # a call may be run again: what it reads is set by the calls before it
        for layer, cache in zip(self.layers, state["caches"]):
            keep()
            yield "norm", norm(layer["pre"])
            yield "qkv", linear(layer["qkv"], "h", "qkv")
            yield "append", append(cache)
            yield "attend", attend(cache)
            yield "out", linear(layer["out"], "a", "y")
            keep()
            yield "norm", norm(layer["mid"], gate=layer["gate"], post=layer["post"])
            yield "up", linear(layer["up"], "h", "g", act="swiglu")
            yield "down", linear(layer["down"], "g", "y")
        keep()
        yield "norm", norm(self.last)
        yield "result", lambda: now["h"]

    def step(self, x, state, new=1):
        """`new` further tokens of every sequence; returns [sequences * new, width]."""
        state["lengths"] += new
        result = None
        for _, run in self.calls(x, state, new):
            result = run()
        return result


def trace(model, state, new=1, repeats=16):
    """One step's kernels: a list of dicts name, grid, threads, regs, smem,
    duration (microseconds).

    The step runs `repeats` times and each launch is timed in its place there, so
    its weights and its part of the cache come from where a step finds them; its
    duration is the median."""
    with torch.cuda.device(model.device):
        x = torch.randn((state["table"].shape[0] * new, model.width), device=model.device)
        x = x.to(model.dtype)
        state["lengths"] += new
        names = []
        for name, run in model.calls(x, state, new):
            with api.rm_trace() as recorded:
                run()
            names += [name] * len(recorded.launches)
        took = []
        for _ in range(repeats):
            with api.rm_trace(len(names), timed=True) as recorded:
                for _, run in model.calls(x, state, new):
                    run()
            took.append([k["duration"] for k in recorded.launches])
    durations = np.median(np.array(took, np.float64).reshape(repeats, -1), axis=0)
    return [dict(k, name=name, duration=float(t))
            for k, name, t in zip(recorded.launches, names, durations)]


def trace_library(models, new=1):
    """Traces of (model, state) pairs as a library of kernel traces, the shape of
    workloads.make_library: for rm_pair_slowdown_matrix with workloads.MI355X."""
    traces = [trace(model, state, new) for model, state in models]
    offsets = np.zeros(len(traces) + 1, np.int64)
    offsets[1:] = np.cumsum([len(t) for t in traces])
    flat = [k for t in traces for k in t]
    out = {f: np.array([k[f] for k in flat], np.int32) for f in ("grid", "threads", "regs", "smem")}
    return dict(out, offsets=offsets, duration=np.array([k["duration"] for k in flat], np.float64))
