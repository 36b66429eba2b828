"""A served model's prompts and decode steps on the library's kernels, and their
kernel traces as the predictor takes them.

    model = DecodeModel(layers=4, width=1024, heads=8, kv_heads=2, head_dim=128,
                        hidden=2816)
    state = model.new_state(sequences=16, most_tokens=2048)
    y = model.prompt(x, state, [700, 31, ...])     # whole prompts, x [their tokens, width]
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
    gated residual between two norms, gated projection, projection.  `weights` "w4"
    (4 bits, a scale for each `group` columns) or "f8" (8-bit floating, a scale for
    each block of 128); with head_norm each head's queries and keys are normalised
    in front of the rotation."""

    def __init__(self, layers, width, heads, kv_heads, head_dim, hidden, group=128,
                 dtype=torch.bfloat16, codes=torch.int8, page_tokens=64, seed=0, device="cuda",
                 weights="w4", head_norm=False):
        if weights not in ("w4", "f8"):
            raise ValueError(f"weights: expected w4 or f8, got {weights!r}")
        self.width, self.heads, self.kv_heads, self.head_dim = width, heads, kv_heads, head_dim
        self.group, self.dtype, self.codes, self.page_tokens = group, dtype, codes, page_tokens
        self.weights, self.head_norm = weights, head_norm
        self.device = torch.device(device)
        gen = torch.Generator(device=device).manual_seed(seed)

        def projection(n, k, parts=1):
            if weights == "f8":       # each part has blocks of its own
                made = [api.rm_f8_quantize(torch.randn((n // parts, k), generator=gen,
                                                       device=device).div_(k ** 0.5).to(dtype),
                                           block_rows=128) for _ in range(parts)]
                return {"codes": torch.cat([c.view(torch.uint8) for c, _ in made]).view(
                            torch.float8_e4m3fn),
                        "scales": torch.cat([s for _, s in made])}
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
            "mid": gain(width), "up": projection(2 * hidden, width, parts=2),
            "down": projection(width, hidden)} for _ in range(layers)]
        if head_norm:
            for layer in self.layers:
                layer["q_gain"], layer["k_gain"] = gain(head_dim), gain(head_dim)
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

    def calls(self, x, state, new=1, lengths=None):
        """The step's calls in order, each a (name, function of no argument).  x
        [sequences * new, width]: `new` tokens of every sequence, counted in
        state["lengths"] already; or with `lengths` (a number for each sequence) whole
        prompts behind each other, which are all that the state then holds."""
        n = state["table"].shape[0]
        h, kv, d = self.heads, self.kv_heads, self.head_dim
        offsets, positions, tokens, most = None, None, n * new, new
        if lengths is not None:
            ends = np.cumsum([0] + list(lengths))
            tokens, most = int(ends[-1]), max([0] + list(lengths))
            offsets = torch.tensor(ends, dtype=torch.int32, device=self.device)
        elif new != 1:
            offsets = torch.arange(0, n * new + 1, new, dtype=torch.int32, device=self.device)
        if self.head_norm:
            if lengths is not None:
                positions = torch.tensor(np.concatenate([np.arange(m) for m in lengths] + [[]]),
                                         dtype=torch.int32, device=self.device)
            else:
                back = torch.arange(-new, 0, dtype=torch.int32, device=self.device)
                positions = (state["lengths"][:, None] + back).reshape(-1)
        seqs = dict(token_offsets=offsets, max_tokens=most, status=state["status"])
        none = self.inv_freq[:0]
        now = {"x": x, "y": None}

        def linear(w, source, to, act="none"):
            def run():
                if self.weights == "f8":
                    now[to] = api.rm_f8_linear(now[source], w["codes"], w["scales"], act=act)
                else:
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

        def split():
            qkv = now["qkv"].view(tokens, h + 2 * kv, d)
            return qkv[:, :h], qkv[:, h:h + kv], qkv[:, h + kv:]

        def turn(layer):
            def run():
                q, k, _ = split()
                now["q"], now["k"] = api.rm_head_norm_rotary(
                    q, k, self.inv_freq, positions, q_weight=layer["q_gain"],
                    k_weight=layer["k_gain"], rot_scale=self.rot_scale)
            return run

        def append(cache):
            def run():
                q, k, v = split()
                if self.head_norm:        # turned already
                    api.rm_rotary_append(None, now["k"], v, none, cache, state["table"],
                                         state["lengths"], **seqs)
                    return
                if lengths is not None:   # the prompt's attention takes turned keys too
                    q = now["qkv"].view(tokens, h + 2 * kv, d)[:, :h + kv]
                q = api.rm_rotary_append(q, k, v, self.inv_freq, cache, state["table"],
                                         state["lengths"], rot_scale=self.rot_scale, **seqs)
                now["q"], now["k"] = q[:, :h], q[:, h:]
            return run

        def attend(cache):
            def run():
                if lengths is not None:
                    a = api.rm_prompt_attention(now["q"], now["k"], split()[2], offsets, most,
                                                status=state["status"])
                else:
                    a = api.rm_cache_attention(now["q"], cache, state["table"], state["lengths"],
                                               **seqs)
                now["a"] = a.view(tokens, h * d)
            return run

        # a call may be run again: what it reads is set by the calls before it
        for layer, cache in zip(self.layers, state["caches"]):
            keep()
            yield "norm", norm(layer["pre"])
            yield "qkv", linear(layer["qkv"], "h", "qkv")
            if self.head_norm:
                yield "turn", turn(layer)
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

    def prompt(self, x, state, lengths):
        """Whole prompts of lengths[b] tokens, behind each other in x: every sequence
        begins anew.  Returns [sum of lengths, width].  The lengths are numbers of the
        host, whose borders each call copies to the GPU: it cannot be captured, as a
        step can."""
        if len(lengths) != state["table"].shape[0] or min(lengths, default=0) < 0:
            raise ValueError("lengths: expected a number of tokens for every sequence")
        if x.shape != (sum(lengths), self.width):
            raise ValueError(f"x: expected [{sum(lengths)}, {self.width}], got {list(x.shape)}")
        state["lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
        result = None
        for _, run in self.calls(x, state, lengths=lengths):
            result = run()
        return result


def trace(model, state, new=1, repeats=16, lengths=None):
    """One step's launches of the library: a list of dicts name, grid, threads, regs,
    smem, duration (microseconds); with `lengths` those of whole prompts.  What torch
    launches for a step's positions is not among them.

    The step runs `repeats` times and each launch is timed in its place there, so
    its weights and its part of the cache come from where a step finds them; its
    duration is the median."""
    with torch.cuda.device(model.device):
        tokens = state["table"].shape[0] * new if lengths is None else sum(lengths)
        x = torch.randn((tokens, model.width), device=model.device)
        x = x.to(model.dtype)
        if lengths is None:
            state["lengths"] += new
        else:
            model.prompt(x, state, lengths)
        names = []
        for name, run in model.calls(x, state, new, lengths):
            with api.rm_trace() as recorded:
                run()
            names += [name] * len(recorded.launches)
        took = []
        for _ in range(repeats):
            with api.rm_trace(len(names), timed=True) as recorded:
                for _, run in model.calls(x, state, new, lengths):
                    run()
            took.append([k["duration"] for k in recorded.launches])
    durations = np.median(np.array(took, np.float64).reshape(repeats, -1), axis=0)
    return [dict(k, name=name, duration=float(t))
            for k, name, t in zip(recorded.launches, names, durations)]


def trace_library(models, new=1):
    """Traces of (model, state) pairs, or of prompts as (model, state, lengths), as a
    library of kernel traces, the shape of workloads.make_library: for
    rm_pair_slowdown_matrix with workloads.MI355X."""
    traces = [trace(m[0], m[1], new, lengths=m[2] if len(m) > 2 else None) for m in models]
    offsets = np.zeros(len(traces) + 1, np.int64)
    offsets[1:] = np.cumsum([len(t) for t in traces])
    flat = [k for t in traces for k in t]
    out = {f: np.array([k[f] for k in flat], np.int32) for f in ("grid", "threads", "regs", "smem")}
    return dict(out, offsets=offsets, duration=np.array([k["duration"] for k in flat], np.float64))
