"""Timed cases of the decode-layer operators, with their inputs, their minimal
work, their plain form in elementary torch operations (32 bits, rounded once)
and their definition in 64 bits.

The operators are the kernels of one layer of a served model in the form in
which several models share a GPU: projections with 4-bit weights, rotary
positions with the append to a paged 8-bit cache, attention over that cache,
and the norms around a block.

A cache is a dict: "k" [pages, kv_heads, page_tokens, head_dim] and "v"
[pages, kv_heads, head_dim, page_tokens], int8 or float8_e4m3fn codes, and
"k_scale", "v_scale" [pages, kv_heads] float32: one scale for each page of
tokens and head.  A table [sequences, most_pages] int32 names each sequence's
pages in order, and `lengths` [sequences] int32 its tokens, the call's own
included.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
LARGEST = {"int8": 127.0, "e4m3": 448.0}
EPS = 1e-6


def listed():
    return [
        # one token through a square projection of width 4096
        dict(name="w4-one-token", op="w4", rows=1, n=4096, k=4096, group=128, zeros=False,
             bias=False, act="none", type="bf16"),
        # a few requests in flight, rows and groups that fill no tile
        dict(name="w4-few-odd", op="w4", rows=5, n=1021, k=5152, group=32, zeros=True,
             bias=True, act="none", type="f16"),
        # the gate and up projections of a batch of 16, activation included
        dict(name="w4-gated-16", op="w4", rows=16, n=28672, k=4096, group=128, zeros=True,
             bias=False, act="swiglu", type="bf16"),
        # a batch of 64 through the down projection of a large model
        dict(name="w4-batch-64", op="w4", rows=64, n=8192, k=28672, group=64, zeros=False,
             bias=False, act="none", type="bf16"),
        # one new token of each of 64 sequences, small pages that are part filled
        dict(name="append-decode", op="append", seqs=64, len_min=1, len_max=2048, new_min=1,
             new_max=1, ragged=11, heads=32, kv_heads=8, dim=128, rot=128, layout="half",
             page=16, codes="int8", type="bf16"),
        # prompts of four sequences behind what they hold, half of the head rotated
        dict(name="append-prompts", op="append", seqs=4, len_min=0, len_max=600, new_min=1200,
             new_max=2600, ragged=12, heads=32, kv_heads=8, dim=128, rot=64,
             layout="interleaved", page=64, codes="e4m3", type="f16"),
        # one sequence with a short history: latency
        dict(name="attend-one-short", op="attend", seqs=1, len_min=501, len_max=501, new_min=1,
             new_max=1, ragged=21, heads=32, kv_heads=8, dim=128, window=0, page=16,
             codes="int8", type="bf16"),
        # a served batch whose lengths differ, an empty one among them
        dict(name="attend-batch-64", op="attend", seqs=64, len_min=0, len_max=4096, new_min=1,
             new_max=1, ragged=22, heads=32, kv_heads=8, dim=128, window=0, page=64,
             codes="e4m3", type="bf16"),
        # two long documents
        dict(name="attend-two-long", op="attend", seqs=2, len_min=120001, len_max=131072,
             new_min=1, new_max=1, ragged=23, heads=64, kv_heads=8, dim=128, window=0, page=64,
             codes="int8", type="bf16"),
        # chunks of four prompts over what is held of them
        dict(name="attend-chunks", op="attend", seqs=4, len_min=700, len_max=4096, new_min=300,
             new_max=512, ragged=24, heads=32, kv_heads=8, dim=128, window=0, page=32,
             codes="int8", type="f16"),
        # one token between two blocks
        dict(name="norm-one-token", op="norm", rows=1, width=4096, kind="rms", post=True,
             gate="channel", type="bf16"),
        # the tokens of a long prompt
        dict(name="norm-prompt", op="norm", rows=8190, width=5120, kind="layer", post=True,
             gate="full", type="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _any(rng, op):
    kind = rng.choice(["bf16", "f16"])
    if op == "w4":
        group = rng.choice([32, 64, 128, 256])
        act = rng.choice(["none", "none", "swiglu"])
        n = _log(rng, 64, 28672)
        k = _log(rng, 128, 28672)
        return dict(op=op, rows=_log(rng, 1, 64), n=n + n % 2,
                    k=k if rng.random() < 0.3 else -(-k // 32) * 32, group=group,
                    zeros=rng.random() < 0.5, bias=rng.random() < 0.3, act=act, type=kind)
    if op == "norm":
        return dict(op=op, rows=_log(rng, 1, 8192), width=_log(rng, 64, 16384),
                    kind=rng.choice(["rms", "layer"]), post=rng.random() < 0.6,
                    gate=rng.choice(["none", "channel", "token", "full"]), type=kind)
    kv = rng.choice([1, 2, 4, 8])
    per = rng.choice([1, 2, 4, 5, 8] if kv > 1 else [4, 8, 16])
    dim = rng.choice([64, 128, 128, 256])
    base = dict(op=op, ragged=rng.randrange(1 << 20), heads=kv * per, kv_heads=kv, dim=dim,
                page=rng.choice([16, 32, 64, 128]), codes=rng.choice(["int8", "e4m3"]), type=kind)
    if op == "append":
        rot = rng.choice([dim, dim, dim // 2, dim // 4])
        new = 1 if rng.random() < 0.5 else _log(rng, 2, 2600)
        top = _log(rng, 2, 2048)
        return dict(base, seqs=_log(rng, 1, 64), len_min=0, len_max=top, new_min=max(1, new // 2),
                    new_max=new, rot=rot, layout=rng.choice(["half", "interleaved"]))
    new = 1 if rng.random() < 0.7 else _log(rng, 2, 512)
    top = max(new, _log(rng, 16, 131072))
    return dict(base, seqs=_log(rng, 1, 64), len_min=rng.choice([0, top // 2, top]), len_max=top,
                new_min=max(1, new // 2), new_max=new,
                window=rng.choice([0, 0, 0, _log(rng, 16, 4096)]))


def draw(rng):
    op = rng.choice(["w4", "append", "attend", "attend", "norm"])
    ours = [work(c) for c in listed() if c["op"] == op]
    most = {u: max(w[u] for w in ours) for u in ("bytes", "flops")}
    while True:
        case = _any(rng, op)
        if all(work(case)[u] <= most[u] for u in most):
            return case


def _ragged(case):
    """(tokens that each sequence holds with the call's own, the call's own)."""
    rng = random.Random(case["ragged"])
    new = [rng.randint(case["new_min"], case["new_max"]) for _ in range(case["seqs"])]
    held = [rng.randint(case["len_min"], case["len_max"]) for _ in range(case["seqs"])]
    if case["op"] == "append":
        return [h + n for h, n in zip(held, new)], new
    held[0] = max(1, held[0])
    if case["len_min"] == 0 and case["seqs"] > 1:
        held[case["seqs"] // 2] = 0      # one sequence that holds nothing
    return held, [min(n, h) for h, n in zip(held, new)]


def _visible(length, new, window):
    """Pairs (new token, token that it sees) of one sequence."""
    first = length - new + 1
    if not window or window >= length:
        return (first + length) * new // 2
    full = max(0, min(new, window - first + 1))        # rows that see fewer than the window
    return (first + first + full - 1) * full // 2 + (new - full) * window


def work(case):
    c = case
    if c["op"] == "w4":
        groups = -(-c["k"] // c["group"])
        out = c["n"] // 2 if c["act"] == "swiglu" else c["n"]
        size = (c["n"] * (c["k"] + 1) // 2 + c["n"] * groups * (3 if c["zeros"] else 2) +
                c["rows"] * c["k"] * 2 + c["rows"] * out * 2 + (c["n"] * 2 if c["bias"] else 0))
        return {"bytes": size, "flops": 2 * c["rows"] * c["n"] * c["k"]}
    if c["op"] == "norm":
        m, h = c["rows"], c["width"]
        gate = {"none": 0, "channel": h, "token": m, "full": m * h}[c["gate"]]
        gains = h * (1 + c["post"] + (c["kind"] == "layer"))
        return {"bytes": 2 * (4 * m * h + gate + gains), "flops": 14 * m * h}
    lens, new = _ragged(c)
    tokens, kv, d, t = sum(new), c["kv_heads"], c["dim"], c["page"]
    if c["op"] == "append":
        blocks = sum(_blocks(n, w, t) for n, w in zip(lens, new))
        part = sum((n - w) % t for n, w in zip(lens, new))      # older tokens of part-filled pages
        size = (tokens * (c["heads"] * 2 + kv * 2) * d * 2 + part * kv * d * 2 +
                blocks * kv * (t * d * 2 + 8) + blocks * kv * t * d * 4)
        return {"bytes": size, "flops": tokens * (c["heads"] + 2 * kv) * d * 6}
    seen = [min(n, w + c["window"] - 1) if c["window"] else n for n, w in zip(lens, new)]
    pages = sum(-(-n // t) for n in seen)
    size = sum(seen) * kv * 2 * d + pages * (kv * 8 + 4) + tokens * c["heads"] * d * 4
    pairs = sum(_visible(n, w, c["window"]) for n, w in zip(lens, new))
    return {"bytes": size, "flops": 4 * pairs * c["heads"] * d}


def _blocks(length, new, page):
    return -(-length // page) - (length - new) // page if new else 0


# --------------------------------------------------------------------------- inputs

def _codes(case, shape, gen):
    """Codes as a quantised cache holds them: near normal, the largest in use."""
    x = torch.randn(shape, generator=gen, device="cuda") * (LARGEST[case["codes"]] / 3.2)
    x = x.clamp_(-LARGEST[case["codes"]], LARGEST[case["codes"]])
    return x.round_().to(torch.int8) if case["codes"] == "int8" else x.to(torch.float8_e4m3fn)


def _cache(case, pages, gen):
    kv, t, d = case["kv_heads"], case["page"], case["dim"]
    k, v = _codes(case, (pages, kv, t, d), gen), _codes(case, (pages, kv, d, t), gen)
    scale = [3.2 / LARGEST[case["codes"]] *
             torch.exp(0.3 * torch.randn((pages, kv), generator=gen, device="cuda"))
             for _ in range(2)]
    return {"k": k, "v": v, "k_scale": scale[0], "v_scale": scale[1]}


def _frequencies(rot):
    """Base 10000, positions interpolated by 4 as for a context four times as long."""
    return [10000.0 ** (-2.0 * i / rot) / 4.0 for i in range(rot // 2)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(dt)

    st = {"case": case}
    if case["op"] == "w4":
        n, k = case["n"], case["k"]
        groups = -(-k // case["group"])
        st["x"] = normal(case["rows"], k)
        st["codes"] = torch.randint(0, 256, (n, (k + 1) // 2), generator=gen, device="cuda",
                                    dtype=torch.uint8)
        st["scales"] = (torch.exp(0.2 * torch.randn((n, groups), generator=gen, device="cuda")) *
                        (0.2 / math.sqrt(k))).to(dt)
        st["zeros"] = torch.randint(5, 11, (n, groups), generator=gen, device="cuda",
                                    dtype=torch.uint8) if case["zeros"] else None
        st["bias"] = normal(n) if case["bias"] else None
        return st
    if case["op"] == "norm":
        m, h = case["rows"], case["width"]
        st["x"], st["y"] = normal(m, h) * 3, normal(m, h)
        shape = {"none": None, "channel": (h,), "token": (m, 1), "full": (m, h)}[case["gate"]]
        st["gate"] = None if shape is None else torch.sigmoid(normal(*shape))
        st["post"] = 1 + normal(h) / 8 if case["post"] else None
        st["pre"] = 1 + normal(h) / 8
        st["pre_bias"] = normal(h) / 8 if case["kind"] == "layer" else None
        return st
    lens, new = _ragged(case)
    page, d = case["page"], case["dim"]
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    most = max(1, max(need))
    at = torch.tensor([[sum(need[:b]) + i if i < need[b] else -1 for i in range(most)]
                       for b in range(case["seqs"])], device="cuda")
    st["table"] = torch.where(at >= 0, order[at.clamp(min=0)], -1).to(torch.int32)
    st["cache"] = _cache(case, pages, gen)
    st["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    offsets = [0]
    for n in new:
        offsets.append(offsets[-1] + n)
    st["offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    st["most_new"] = max(1, max(new))
    st["q"] = normal(offsets[-1], case["heads"], d)
    if case["op"] == "attend":
        return st
    # key and value of one fused projection: views with a token stride of both
    both = normal(offsets[-1], 2 * case["kv_heads"], d)
    st["key"], st["value"] = both[:, :case["kv_heads"]], both[:, case["kv_heads"]:]
    st["inv_freq"] = torch.tensor(_frequencies(case["rot"]), dtype=torch.float32, device="cuda")
    # the pages that this call writes, in the order of the sequences
    touched, slot = [], []
    for b, (n, w) in enumerate(zip(lens, new)):
        first = (n - w) // page
        slot += [(len(touched) - first) * page + p for p in range(n - w, n)]
        touched += [at_b for at_b in range(sum(need[:b]) + first, sum(need[:b + 1]))]
    st["touched"] = order[torch.tensor(touched, device="cuda")]
    st["slot"] = torch.tensor(slot, device="cuda")     # of each token, in those pages in a row
    return st


# --------------------------------------------------------------------------- one pass

def run(state):
    return (_kernels if own else _plain)(state)


def _kernels(s):
    from paper_2607_16784_amd import api
    c = s["case"]
    if c["op"] == "w4":
        return api.rm_w4_linear(s["x"], s["codes"], s["scales"], c["group"], zeros=s["zeros"],
                                bias=s["bias"], act=c["act"])
    if c["op"] == "norm":
        x, n = api.rm_norm_residual(s["x"], s["y"], gate=s["gate"], post_weight=s["post"],
                                    pre_weight=s["pre"], pre_bias=s["pre_bias"],
                                    kind=c["kind"], alpha=0.5, eps=EPS)
        return {"x": x, "n": n}
    if c["op"] == "attend":
        return api.rm_cache_attention(s["q"], s["cache"], s["table"], s["lengths"],
                                      token_offsets=s["offsets"], max_tokens=s["most_new"],
                                      window=c["window"])
    q = api.rm_rotary_append(s["q"], s["key"], s["value"], s["inv_freq"], s["cache"], s["table"],
                             s["lengths"], token_offsets=s["offsets"], max_tokens=s["most_new"],
                             layout=c["layout"], rot_scale=1.1)
    k, v = api.rm_cache_read(s["cache"], s["touched"], s["q"].dtype)
    return {"q": q, "k": k, "v": v}


def _plain(s):
    return {"w4": _plain_w4, "norm": _plain_norm, "attend": _plain_attend,
            "append": _plain_append}[s["case"]["op"]](s)


def _plain_w4(s):
    c, codes = s["case"], s["codes"]
    n, k = c["n"], c["k"]
    w = torch.stack((codes & 15, codes >> 4), dim=2).reshape(n, -1)[:, :k].float()
    group = torch.arange(k, device="cuda") // c["group"]
    zero = 8.0 if s["zeros"] is None else s["zeros"].float()[:, group]
    w = (w - zero) * s["scales"].float()[:, group]
    t = s["x"].float() @ w.t()
    if s["bias"] is not None:
        t = t + s["bias"].float()
    if c["act"] == "swiglu":
        t = t[:, :n // 2] / (1 + torch.exp(-t[:, :n // 2])) * t[:, n // 2:]
    return t.to(s["x"].dtype)


def _normalised(x, kind):
    if kind == "layer":
        x = x - x.mean(dim=1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS)


def _plain_norm(s):
    c, dt = s["case"], s["x"].dtype
    u = s["y"].float()
    if s["post"] is not None:
        u = _normalised(u, c["kind"]) * s["post"].float()
    if s["gate"] is not None:
        u = u * s["gate"].float()
    x = s["x"].float() + 0.5 * u
    n = _normalised(x, c["kind"]) * s["pre"].float()
    if s["pre_bias"] is not None:
        n = n + s["pre_bias"].float()
    return {"x": x.to(dt), "n": n.to(dt)}


def _tokens(s):
    """Sequence, index among the sequence's new tokens and position of each new token."""
    off = s["offsets"].long()
    at = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(off[1:], at, right=True)
    i = at - off[seq]
    return seq, i, s["lengths"].long()[seq] - (off[seq + 1] - off[seq]) + i


def _gather(codes, pages):
    return codes.view(torch.uint8)[pages].view(codes.dtype).float()


def _plain_attend(s):
    c, cache = s["case"], s["cache"]
    kv, d, seqs = c["kv_heads"], c["dim"], c["seqs"]
    per, most = c["heads"] // kv, s["most_new"]
    pages = s["table"].long()                  # -1, past a sequence's end, is masked below
    k = _gather(cache["k"], pages) * cache["k_scale"][pages][..., None, None]
    v = _gather(cache["v"], pages) * cache["v_scale"][pages][..., None, None]
    k = k.permute(0, 2, 4, 1, 3).reshape(seqs * kv, d, -1)
    v = v.permute(0, 2, 1, 4, 3).reshape(seqs * kv, -1, d)
    seq, i, pos = _tokens(s)
    q = torch.zeros((seqs, most, c["heads"], d), device="cuda")
    q[seq, i] = s["q"].float() / math.sqrt(d)
    q = q.reshape(seqs, most, kv, per, d).permute(0, 2, 1, 3, 4).reshape(seqs * kv, -1, d)
    p = torch.bmm(q, k).reshape(seqs, kv, most, per, -1)
    row = torch.full((seqs, most), -1, device="cuda")
    row[seq, i] = pos
    j = torch.arange(p.shape[-1], device="cuda")
    seen = j <= row[:, :, None]
    if c["window"]:
        seen &= j > row[:, :, None] - c["window"]
    seen = seen[:, None, :, None]
    p = torch.where(seen, p, -math.inf)
    top = p.amax(dim=-1, keepdim=True)
    p = torch.exp(p - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(dim=-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    o = torch.bmm(p.reshape(seqs * kv, most * per, -1), v)
    o = o.reshape(seqs, kv, most, per, d).permute(0, 2, 1, 3, 4).reshape(seqs, most, -1, d)
    return o[seq, i].to(s["q"].dtype)


def _rotated(x, pos, s):
    c, rot = s["case"], s["case"]["rot"]
    a = (pos.float()[:, None] * s["inv_freq"])[:, None]
    cos, sin = torch.cos(a) * 1.1, torch.sin(a) * 1.1
    x = x.float()
    if c["layout"] == "half":
        u, w = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((u * cos - w * sin, u * sin + w * cos), dim=-1)
    else:
        u, w = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((u * cos - w * sin, u * sin + w * cos), dim=-1).flatten(-2)
    return torch.cat((turned, x[..., rot:]), dim=-1)


def _put(codes, scale, pages, new, fresh, older, fmt):
    """The pages [n, heads, tokens, dim] with the new tokens in them: codes and scales.
    fresh: slots of the call's own tokens, older: of those that were there."""
    top = LARGEST[fmt]
    was = torch.where(older.any(dim=1)[:, None], scale[pages], 0.0)
    now = torch.maximum(was, new.abs().amax(dim=(2, 3)) / top)
    inv = torch.where(now > 0, 1 / now, 0.0)
    old = _gather(codes, pages) * (was * inv)[..., None, None]
    x = torch.where(fresh[:, None, :, None], new * inv[..., None, None],
                    torch.where(older[:, None, :, None], old, 0.0)).clamp(-top, top)
    x = x.round().to(torch.int8) if fmt == "int8" else x.to(torch.float8_e4m3fn)
    return x, now


def _plain_append(s):
    c, cache, dt = s["case"], s["cache"], s["q"].dtype
    kv, d, page, fmt = c["kv_heads"], c["dim"], c["page"], c["codes"]
    _, _, pos = _tokens(s)
    pages, n = s["touched"].long(), s["touched"].numel()
    fresh = torch.zeros(n * page, dtype=torch.bool, device="cuda")
    fresh[s["slot"]] = True
    fresh = fresh.reshape(n, page)
    # older slots are those before the first of the call's own in its page
    older = (torch.cumsum(fresh, dim=1) == 0) & fresh.any(dim=1, keepdim=True)
    out = {"q": _rotated(s["q"], pos, s).to(dt)}
    for name, x in (("k", _rotated(s["key"], pos, s)), ("v", s["value"].float())):
        new = torch.zeros((n * page, kv, d), device="cuda")
        new[s["slot"]] = x
        new = new.reshape(n, page, kv, d).transpose(1, 2)
        scale = cache[name + "_scale"]
        held = cache[name] if name == "k" else cache[name].transpose(2, 3)
        x, now = _put(held, scale, pages, new, fresh, older, fmt)
        scale[pages] = now
        held.view(torch.uint8)[pages] = x.view(torch.uint8)
        out[name] = (x.float() * now[..., None, None]).transpose(1, 2).contiguous().to(dt)
    return out


# --------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"w4": _exact_w4, "norm": _exact_norm, "attend": _exact_attend,
            "append": _exact_append}[case["op"]](s)


def _exact_w4(s):
    c, x = s["case"], s["x"].double()
    n, k, g = c["n"], c["k"], c["group"]
    t = torch.zeros((c["rows"], n), dtype=torch.float64, device="cuda")
    for i, lo in enumerate(range(0, k, g)):
        part = s["codes"][:, lo // 2:(min(k, lo + g) + 1) // 2]
        w = torch.empty((n, 2 * part.shape[1]), dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = part.remainder(16), part.div(16, rounding_mode="floor")
        w = w[:, :min(k, lo + g) - lo]
        w -= 8 if s["zeros"] is None else s["zeros"][:, i:i + 1]
        t += (x[:, lo:lo + g] @ w.t()) * s["scales"][:, i].double()
    if s["bias"] is not None:
        t += s["bias"].double()
    if c["act"] == "swiglu":
        a, b = t.chunk(2, dim=1)
        t = a * torch.sigmoid(a) * b
    return t


def _exact_norm(s):
    c = s["case"]

    def unit(x):
        off = x.mean(1, keepdim=True) if c["kind"] == "layer" else 0.0
        return (x - off) / (((x - off) ** 2).mean(1, keepdim=True) + EPS).sqrt()

    u = s["y"].double()
    u = unit(u) * s["post"].double() if s["post"] is not None else u
    u = u * s["gate"].double() if s["gate"] is not None else u
    x = s["x"].double() + u / 2
    n = unit(x) * s["pre"].double()
    return {"x": x, "n": n + s["pre_bias"].double() if s["pre_bias"] is not None else n}


def _held(s, b, h, length):
    """Keys and values of one sequence's head, [length, dim] in 64 bits."""
    page, cache = s["case"]["page"], s["cache"]
    pages = s["table"][b, :-(-length // page)].long()
    k = cache["k"][:, h].view(torch.uint8)[pages].view(cache["k"].dtype).double()
    v = cache["v"][:, h].view(torch.uint8)[pages].view(cache["v"].dtype).double()
    k = k * cache["k_scale"][pages, h].double()[:, None, None]
    v = v * cache["v_scale"][pages, h].double()[:, None, None]
    d = s["case"]["dim"]
    return k.reshape(-1, d)[:length], v.transpose(1, 2).reshape(-1, d)[:length]


def _exact_attend(s):
    c = s["case"]
    per = c["heads"] // c["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    off = s["offsets"].tolist()
    for b, length in enumerate(s["lengths"].tolist()):
        lo, hi = off[b], off[b + 1]
        if hi == lo:
            continue
        pos = torch.arange(length - (hi - lo), length, device="cuda")[:, None]
        j = torch.arange(length, device="cuda")
        hidden = (j > pos) | ((j <= pos - c["window"]) if c["window"] else (j < 0))
        for h in range(c["heads"]):
            if h % per == 0:
                k, v = _held(s, b, h // per, length)
            p = s["q"][lo:hi, h].double() @ k.t() / c["dim"] ** 0.5
            out[lo:hi, h] = p.masked_fill(hidden, -math.inf).softmax(dim=1) @ v
    return out


def _exact_append(s):
    c, cache = s["case"], s["cache"]
    page, rot, fmt = c["page"], c["rot"], c["codes"]
    off, out = s["offsets"].tolist(), {"k": [], "v": []}
    lens = s["lengths"].tolist()
    pos = torch.cat([torch.arange(n - (off[b + 1] - off[b]), n) for b, n in enumerate(lens)])
    turn = torch.polar(torch.tensor(1.1, dtype=torch.float64, device="cuda"),
                       pos.cuda().double()[:, None] * s["inv_freq"].double())[:, None]
    if c["layout"] == "half":
        first, second = slice(0, rot // 2), slice(rot // 2, rot)
    else:
        first, second = slice(0, rot, 2), slice(1, rot, 2)

    def rotate(x):
        x = x.double().clone()
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    at = 0
    key = rotate(s["key"])
    for b, n in enumerate(lens):
        start = n - (off[b + 1] - off[b])
        for lo in range(start // page * page, n, page):
            where, at = int(s["touched"][at]), at + 1
            older, upto = max(0, start - lo), min(page, n - lo)
            mine = slice(off[b] + lo + older - start, off[b] + lo + upto - start)
            for name, x in (("k", key), ("v", s["value"].double())):
                x = x[mine].transpose(0, 1)
                held = cache[name][where].double()
                held = (held if name == "k" else held.transpose(1, 2))[:, :older]
                was = cache[name + "_scale"][where].double() if older else 0.0
                now = x.abs().amax(dim=(1, 2)) / LARGEST[fmt]
                now = torch.maximum(now, was) if older else now
                full = torch.zeros((c["kv_heads"], page, c["dim"]), dtype=torch.float64,
                                   device="cuda")
                full[:, :older] = held * (was / now)[:, None, None] if older else held
                full[:, older:upto] = x / now[:, None, None]
                q = full.round() if fmt == "int8" else full.float().to(CODES[fmt]).double()
                out[name].append((q * now[:, None, None]).transpose(0, 1))
    return {"q": rotate(s["q"]), "k": torch.stack(out["k"]), "v": torch.stack(out["v"])}
