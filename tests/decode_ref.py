"""Plain 64-bit evaluations of the decode-layer operators, on the CPU, one
sequence, head and row at a time where that is the definition."""
import math

import torch

LARGEST = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}
# half a unit in the last place over the value: 8 and 11 significant bits
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def f64(t):
    return t.detach().cpu().double() if t is not None else None


def codes_f64(t):
    return t.detach().cpu().float().double()


def weights(codes, scales, zeros, group, k):
    """The matrix that 4-bit codes stand for, [n, k]."""
    codes = codes.cpu().long()
    n = codes.shape[0]
    w = torch.zeros((n, k), dtype=torch.float64)
    for i in range(k):
        c = (codes[:, i // 2] >> (4 * (i % 2))) & 15
        z = 8 if zeros is None else zeros.cpu()[:, i // group].long()
        w[:, i] = (c - z).double() * f64(scales)[:, i // group]
    return w


def linear(x, codes, scales, group, zeros=None, bias=None, act="none"):
    w = weights(codes, scales, zeros, group, x.shape[1])
    t = f64(x) @ w.t()
    if bias is not None:
        t = t + f64(bias)
    if act == "swiglu":
        a, b = t.chunk(2, dim=1)
        t = a / (1 + torch.exp(-a)) * b
    return t


def rotate(x, positions, inv_freq, layout, scale):
    """x [tokens, heads, dim]."""
    x = f64(x).clone()
    rot = 2 * len(inv_freq)
    for t in range(x.shape[0]):
        for i in range(rot // 2):
            a = float(positions[t]) * float(inv_freq[i])
            u, w = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
            c, s = scale * math.cos(a), scale * math.sin(a)
            first, second = x[t, :, u].clone(), x[t, :, w].clone()
            x[t, :, u] = first * c - second * s
            x[t, :, w] = first * s + second * c
    return x


def cached(cache, table, length, b, h):
    """Keys and values of a sequence's kv head, [length, dim]."""
    page = cache["k"].shape[2]
    k, v = [], []
    for j in range(length):
        p, s = int(table[b, j // page]), j % page
        k.append(codes_f64(cache["k"][p, h, s]) * float(cache["k_scale"][p, h]))
        v.append(codes_f64(cache["v"][p, h, :, s]) * float(cache["v_scale"][p, h]))
    if not k:
        return [torch.zeros((0, cache["k"].shape[3]), dtype=torch.float64)] * 2
    return torch.stack(k), torch.stack(v)


def attention(q, cache, table, lengths, offsets=None, scale=None, window=0):
    """(out, mean of |value| under the weights) [tokens, heads, dim]."""
    tokens, heads, dim = q.shape
    kv = cache["k"].shape[1]
    scale = dim ** -0.5 if scale is None else scale
    cache = {n: t.cpu() for n, t in cache.items()}
    out = torch.zeros((tokens, heads, dim), dtype=torch.float64)
    size = torch.zeros_like(out)
    for b, length in enumerate(lengths):
        lo, hi = (offsets[b], offsets[b + 1]) if offsets is not None else (b, b + 1)
        for g in range(kv):
            k, v = cached(cache, table.cpu(), length, b, g)
            for t in range(lo, hi):
                p = length - (hi - lo) + t - lo
                first = max(0, p - window + 1) if window else 0
                if p < first or p < 0:
                    continue
                for h in range(g * heads // kv, (g + 1) * heads // kv):
                    w = torch.softmax(k[first:p + 1] @ f64(q[t, h]) * scale, dim=0)
                    out[t, h] = w @ v[first:p + 1]
                    size[t, h] = w @ v[first:p + 1].abs()
    return out, size


def append(cache, table, lengths, offsets, k, v):
    """The cache after the (already turned) keys k and values v, [tokens,
    kv_heads, dim] in 64 bits, in place of its CPU copy: codes in 64 bits."""
    page = cache["k"].shape[2]
    top = LARGEST[cache["k"].dtype]
    after = {"k": codes_f64(cache["k"]), "v": codes_f64(cache["v"]).transpose(2, 3).contiguous(),
             "k_scale": f64(cache["k_scale"]), "v_scale": f64(cache["v_scale"])}
    for b, length in enumerate(lengths):
        lo, hi = offsets[b], offsets[b + 1]
        start = length - (hi - lo)
        if hi == lo:
            continue
        for at in range(start // page, -(-length // page)):
            p = int(table[b, at])
            s0, s1 = max(0, start - at * page), min(page, length - at * page)
            rows = slice(lo + at * page + s0 - start, lo + at * page + s1 - start)
            for name, x in (("k", k), ("v", v)):
                for h in range(k.shape[1]):
                    new = x[rows, h]
                    was = float(after[name + "_scale"][p, h]) if s0 else 0.0
                    now = max(was, float(new.abs().max()) / top)
                    block = after[name][p, h]
                    block[:s0] = block[:s0] * (was / now) if now else 0.0
                    block[s0:s1] = new / now if now else 0.0
                    block[s1:] = 0.0
                    after[name + "_scale"][p, h] = now
    return after


def norm(x, y=None, gate=None, post=None, pre=None, bias=None, kind="rms", alpha=1.0, eps=1e-6):
    def unit(t):
        t = t - t.mean(dim=1, keepdim=True) if kind == "layer" else t
        return t / torch.sqrt((t * t).mean(dim=1, keepdim=True) + eps)

    r = f64(x)
    if y is not None:
        u = f64(y)
        u = unit(u) * f64(post) if post is not None else u
        r = r + alpha * (u * f64(gate) if gate is not None else u)
    n = unit(r)
    n = n * f64(pre) if pre is not None else n
    return r, n + f64(bias) if bias is not None else n
