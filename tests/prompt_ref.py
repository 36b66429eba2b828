"""Plain 64-bit evaluations of the prompt's operators and of the 8-bit floating
projection, on the CPU, with the sizes of the terms that tolerances count."""
import math

import torch

from decode_ref import ROUND, f64, rotate

E4M3 = torch.float8_e4m3fn


def offsets_of(lengths, first=0):
    out = [first]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def attention(q, k, v, offsets, scale=None, window=0):
    """(out, weighted mean of |value|, largest error of a logit) of rows of q
    [tokens, heads, dim]; rows of no sequence are 0."""
    tokens, heads, dim = q.shape
    scale = dim ** -0.5 if scale is None else scale
    q, k, v = f64(q), f64(k), f64(v)
    per = heads // k.shape[1]
    out, size = torch.zeros_like(q), torch.zeros_like(q)
    off = torch.zeros((tokens, heads, 1), dtype=torch.float64)
    for lo, hi in zip(offsets, offsets[1:]):
        if hi <= lo:
            continue
        i = torch.arange(hi - lo)
        hidden = i > i[:, None]
        if window:
            hidden |= i <= i[:, None] - window
        for h in range(heads):
            kh, vh, qh = k[lo:hi, h // per], v[lo:hi, h // per], q[lo:hi, h]
            p = (qh @ kh.t() * scale).masked_fill(hidden, -math.inf)
            w = torch.softmax(p, dim=1)
            out[lo:hi, h] = w @ vh
            size[lo:hi, h] = w @ vh.abs()
            # dim products and their sums in 32 bits, the factor and the exponential
            terms = (qh.abs() @ kh.abs().t() * abs(scale)).masked_fill(hidden, 0.0)
            off[lo:hi, h, 0] = terms.amax(dim=1) * (dim + 8) * 2.0 ** -24 + 2.0 ** -21
    return out, size, off


def attention_tolerance(want, size, off, lengths, dtype, top):
    """The result's rounding; each weight's in the products' type and its error from
    the logit, numerator and denominator; the sums over the keys in 32 bits; f16
    weights below the type's normal range."""
    n = max(lengths)
    tol = ROUND[dtype] * want.abs() + (ROUND[dtype] + 2 * off + (n + 8) * 2.0 ** -24) * size
    return tol * 1.01 + n * 2.0 ** -28 * top + 1e-30


def head_norm(x, weight, positions, inv_freq, layout, rot_scale, eps):
    """(turned, size of its terms) of x [tokens, heads, dim]."""
    u = f64(x)
    u = u / torch.sqrt((u * u).mean(dim=2, keepdim=True) + eps)
    u = u * f64(weight) if weight is not None else u
    turned = rotate(u, positions, inv_freq, layout, rot_scale)
    size = u.abs().amax(dim=2, keepdim=True) * (1 + 2 * abs(rot_scale))
    return turned, size.expand_as(turned)


def scale_of(top):
    """The smallest power of two, 2^-126 at least, that holds `top` within 448."""
    if top == 0:
        return 2.0 ** -126
    part, power = math.frexp(top / 448.0)
    return 2.0 ** max(power if part > 0.5 else power - 1, -126)


def blocks(x, block_rows):
    """(codes as values, scales) of x [rows, k]."""
    x = f64(x)
    rows, k = x.shape
    scales = torch.zeros((-(-rows // block_rows), -(-k // 128)), dtype=torch.float64)
    codes = torch.zeros_like(x)
    for r in range(scales.shape[0]):
        for c in range(scales.shape[1]):
            at = (slice(r * block_rows, (r + 1) * block_rows), slice(c * 128, (c + 1) * 128))
            scales[r, c] = scale_of(float(x[at].abs().max())) if torch.isfinite(x[at]).all() \
                else math.nan
            codes[at] = (x[at] / scales[r, c]).float().to(E4M3).double()
    return codes, scales


def spread(scales, rows, k, block_rows):
    s = f64(scales).repeat_interleave(block_rows, dim=0)[:rows]
    return s.repeat_interleave(128, dim=1)[:, :k]


def f8_weights(codes, scales, act):
    n, k = codes.shape
    w = codes.cpu().float().double()
    if act != "swiglu":
        return w * spread(scales, n, k, 128)
    half, bands = n // 2, scales.shape[0] // 2
    return torch.cat([w[:half] * spread(scales[:bands], half, k, 128),
                      w[half:] * spread(scales[bands:], half, k, 128)])


def alignment(x, w):
    """The matrix instruction adds the products of eight neighbouring columns as
    multiples of 2^-13 of the power of two below the largest of them (a product of
    2^-13 of it beside it counts, one of 2^-14 is lost; columns eight apart do not
    meet): each of the eight loses less than 2^-13 of that largest product, which is
    at most the largest |x| times the largest |w| of the eight."""
    def tops(t):
        t = torch.nn.functional.pad(t.abs(), (0, -t.shape[1] % 8))
        return t.unflatten(1, (-1, 8)).amax(dim=2)
    return 8 * 2.0 ** -13 * tops(x) @ tops(w).t()


def f8_linear(x, codes, scales, x_scales=None, bias=None, act="none"):
    """(result, its error in 32 bits before the last rounding)."""
    rows, k = x.shape
    if x_scales is None:
        values, s = blocks(x, 1)
        values = values * spread(s, rows, k, 1)
    else:
        values = x.cpu().float().double() * spread(x_scales, rows, k, 1)
    w = f8_weights(codes, scales, act)
    t, size = values @ w.t(), values.abs() @ w.t().abs()
    if bias is not None:
        t, size = t + f64(bias), size + f64(bias).abs()
    # a block's products and their sums, the blocks', the waves', scales and bias
    err = size * (128 + -(-k // 128) + 24) * 2.0 ** -23 + alignment(values, w)
    if act == "swiglu":
        a, b = t.chunk(2, dim=1)
        ea, eb = err.chunk(2, dim=1)
        t = a / (1 + torch.exp(-a)) * b
        # silu's slope is at most 1.1; its own error grows with |a| in the exponent
        err = 1.1 * ea * (b.abs() + eb) + a.abs() * eb + t.abs() * (a.abs() + 8) * 2.0 ** -22
    return t, err
