"""rm_prompt_attention against its 64-bit definition (tolerances: prompt_ref)."""
import pytest
import torch

import prompt_ref as ref
from paper_2607_16784_amd import api

pytestmark = pytest.mark.gpu


def inputs(tokens, heads, kv, dim, dtype, seed, sharp=1.0):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn((tokens, heads + 2 * kv, dim), generator=g)
    qkv[:, :heads] *= sharp
    qkv = qkv.to(dtype).cuda()
    return qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]


def call(q, k, v, offsets, most, **kw):
    st = api.new_status()
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    out = api.rm_prompt_attention(q, k, v, off, most, status=st, **kw)
    return out, int(st.item())


def check(got, q, k, v, offsets, dtype, **kw):
    want, size, off = ref.attention(q, k, v, offsets, **kw)
    lengths = [b - a for a, b in zip(offsets, offsets[1:])]
    tol = ref.attention_tolerance(want, size, off, lengths, dtype, float(v.float().abs().max()))
    err = (ref.f64(got) - want).abs()
    worst = float((err / tol).max()) if err.numel() else 0.0
    assert worst <= 1, worst


LENGTHS = [[1], [2, 1, 0, 3], [33], [64], [65, 63], [127, 128, 129], [1, 0, 300, 77], [0, 0, 5],
           [200, 1, 1, 1, 200, 0]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lengths", LENGTHS, ids=["-".join(map(str, n)) for n in LENGTHS])
def test_against_64_bits(lengths, dim, dtype):
    heads, kv = [(4, 4), (8, 2), (5, 1), (20, 4), (16, 2)][(sum(lengths) + dim // 64) % 5]
    offsets = ref.offsets_of(lengths)
    q, k, v = inputs(offsets[-1], heads, kv, dim, dtype, sum(lengths) + dim)
    got, st = call(q, k, v, offsets, max(lengths))
    assert st == 0
    check(got, q, k, v, offsets, dtype)


@pytest.mark.parametrize("window", [1, 2, 5, 63, 64, 65, 100, 10 ** 9])
@pytest.mark.parametrize("heads,kv", [(2, 2), (8, 2), (5, 1)])
def test_windows(window, heads, kv):
    offsets = ref.offsets_of([70, 1, 333])
    q, k, v = inputs(offsets[-1], heads, kv, 64, torch.float16, window % 1000)
    got, st = call(q, k, v, offsets, 333, window=window)
    assert st == 0
    check(got, q, k, v, offsets, torch.float16, window=window)
    if window == 1:
        assert torch.equal(got, v.repeat_interleave(heads // kv, dim=1))


@pytest.mark.parametrize("group", [1, 3, 7, 16, 40, 128, 130, 300])
def test_groups_of_heads(group):
    offsets = ref.offsets_of([5, 90, 2])
    q, k, v = inputs(97, group, 1, 64, torch.bfloat16, group)
    got, _ = call(q, k, v, offsets, 90)
    check(got, q, k, v, offsets, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0, 3.0])
def test_scales_and_sharp_rows(scale, dtype):
    offsets = ref.offsets_of([150, 40])
    q, k, v = inputs(190, 4, 2, 64, dtype, 5, sharp=2.0)
    got, _ = call(q, k, v, offsets, 150, scale=scale)
    check(got, q, k, v, offsets, dtype, scale=scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rising", [True, False])
def test_logits_that_rise_or_fall_along_the_keys(rising, dtype):
    # the running maximum moves at every step, or never again after the first
    n = 400
    q, k, v = (t.clone() for t in inputs(n, 2, 1, 64, dtype, 6))
    q[:, :, 0] = 4.0
    at = torch.arange(n, device="cuda") / 4.0
    k[:, :, 0] = (at if rising else -at)[:, None].to(dtype)
    got, _ = call(q, k, v, [0, n], n, scale=0.5)
    check(got, q, k, v, [0, n], dtype, scale=0.5)


def test_many_sequences():
    g = torch.Generator().manual_seed(3)
    lengths = torch.randint(0, 4, (5000,), generator=g).tolist()
    offsets = ref.offsets_of(lengths)
    q, k, v = inputs(offsets[-1], 2, 1, 64, torch.float16, 4)
    got, st = call(q, k, v, offsets, 3)
    assert st == 0
    check(got, q, k, v, offsets, torch.float16)


def test_rows_of_no_sequence_get_zero():
    offsets = ref.offsets_of([40, 0, 50], first=7)
    q, k, v = inputs(300, 4, 2, 128, torch.bfloat16, 8)
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    got, st = call(q, k, v, offsets, 50, out=out)
    assert got is out and st == 0
    assert torch.all(out[:7] == 0) and torch.all(out[97:] == 0)
    check(out, q, k, v, offsets, torch.bfloat16)
    for offs in ([0], [5, 5], [0, 0, 0]):
        out.fill_(float("nan"))
        got, st = call(q, k, v, offs, 0, out=out)
        assert st == 0 and torch.all(out == 0)


def test_sequences_out_of_range_are_reported():
    q, k, v = inputs(200, 4, 2, 64, torch.bfloat16, 9)
    good, _ = call(q, k, v, [0, 60, 130, 200], 70)
    # one longer than max_tokens, one past the end, one in front of the first row
    for offsets, most, keep in (([0, 60, 130, 200], 65, slice(0, 60)),
                                ([0, 60, 130, 230], 100, slice(0, 130)),
                                ([-5, 60, 130, 200], 100, slice(60, 200))):
        out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        got, st = call(q, k, v, offsets, most, out=out)
        assert st == api.ST_BAD_LENGTH
        assert torch.equal(got[keep], good[keep])
        other = torch.ones(200, dtype=torch.bool)
        other[keep] = False
        assert torch.all(got[other.cuda()] == 0)
    _, st = call(q, k, v, [0, 130, 60, 200], 200)
    assert st == api.ST_BAD_LENGTH
    _, st = call(q, k, v, [0, 2 ** 31 - 1, -2 ** 31, 200], 200)
    assert st == api.ST_BAD_LENGTH


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dim,window", [(64, 0), (128, 0), (256, 0), (64, 40)])
def test_what_a_row_does_not_see_does_not_reach_it(dim, window, bad):
    offsets = ref.offsets_of([100, 90], first=3)
    q, k, v = inputs(200, 4, 2, dim, torch.bfloat16, 10)
    clean, _ = call(q, k, v, offsets, 100, window=window)
    for at in (40, 70, 1, 102, 110, 150, 199):
        for which in "kv":
            k2, v2 = k.clone(), v.clone()
            (k2 if which == "k" else v2)[at, 1, ::3] = bad
            got, _ = call(q, k2, v2, offsets, 100, window=window)
            lo, hi = (3, 103) if 3 <= at < 103 else (103, 193) if 103 <= at < 193 else (0, 0)
            sees = torch.zeros(200, 4, dtype=torch.bool)
            sees[at if hi else 0:min(hi, at + window) if window else hi, 2:] = True
            sees = sees.cuda()
            assert torch.equal(got[~sees], clean[~sees]), (at, which)
            if which == "v" and hi:
                # all that see it have that value's weight in these channels
                assert not torch.any(torch.isfinite(got[sees][:, ::3])), (at, which)
                others = [c for c in range(dim) if c % 3]
                assert torch.equal(got[sees][:, others], clean[sees][:, others]), (at, which)


def test_strides_and_alignment():
    # rows at odd elements, heads in front of tokens, heads that are the same one
    q, k, v = inputs(90, 4, 2, 64, torch.float16, 11)
    offsets = [0, 90]
    want, _ = call(q.contiguous(), k.contiguous(), v.contiguous(), offsets, 90)

    def odd(t):
        wide = torch.full((t.shape[0], t.shape[1] * 67 + 5), float("nan"), dtype=t.dtype,
                          device="cuda")
        view = wide[:, 3:3 + t.shape[1] * 67].unflatten(1, (t.shape[1], 67))[:, :, :64]
        view.copy_(t)
        return view
    got, _ = call(odd(q), odd(k), odd(v), offsets, 90)
    assert torch.equal(got, want)
    front = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    got, _ = call(*front, offsets, 90)
    assert torch.equal(got, want)
    one = k[:, :1].expand(90, 2, 64), v[:, :1].expand(90, 2, 64)
    got, _ = call(q, *one, offsets, 90)
    want, _ = call(q, *(t.contiguous() for t in one), offsets, 90)
    assert torch.equal(got, want)


def test_a_graph_replays_other_lengths():
    q, k, v = (t.contiguous() for t in inputs(160, 4, 2, 64, torch.bfloat16, 12))
    off = torch.tensor([0, 60, 100, 160], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = api.rm_prompt_attention(q, k, v, off, 160)
    torch.cuda.current_stream().wait_stream(side)
    for offsets in ([0, 60, 100, 160], [0, 0, 160, 160], [10, 20, 30, 150], [0, 1, 2, 3]):
        off.copy_(torch.tensor(offsets, dtype=torch.int32))
        q.add_(0.5)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        want, _ = call(q, k, v, offsets, 160)
        assert torch.equal(out, want), offsets


def test_refusals():
    q, k, v = inputs(20, 4, 2, 64, torch.bfloat16, 13)
    off = torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    f = api.rm_prompt_attention
    bad = [
        (ValueError, lambda: f(q.float(), k, v, off, 20)),
        (ValueError, lambda: f(q, k.half(), v, off, 20)),
        (ValueError, lambda: f(q, k, v[:, :1], off, 20)),
        (ValueError, lambda: f(q, k[:10], v[:10], off, 20)),
        (ValueError, lambda: f(q, k[:, :, :32], v[:, :, :32], off, 20)),
        (ValueError, lambda: f(q[0], k, v, off, 20)),
        (ValueError, lambda: f(q, k, v, off.long(), 20)),
        (ValueError, lambda: f(q, k, v, off[:0], 20)),
        (ValueError, lambda: f(q, k, v, off.cpu(), 20)),
        (ValueError, lambda: f(q, k, v, off, 1 << 31)),
        (ValueError, lambda: f(q, k, v, off, 20, window=1 << 31)),
        (ValueError, lambda: f(q, k, v, off, 20, out=q)),
        (RuntimeError, lambda: f(q[:, :3], k, v, off, 20)),
        (RuntimeError, lambda: f(q, k, v, off, -1)),
        (RuntimeError, lambda: f(q, k, v, off, 20, window=-1)),
        (RuntimeError, lambda: f(q, k, v, off, 20, scale=float("inf"))),
        (RuntimeError, lambda: f(q[:, :, :32], k[:, :, :32], v[:, :, :32], off, 20)),
    ]
    for i, (error, g) in enumerate(bad):
        with pytest.raises(error):
            g()
            print("accepted", i)
    empty = f(q[:0], k[:0], v[:0], off[:1], 0)
    assert empty.shape == (0, 4, 64)
