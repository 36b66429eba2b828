"""rm_cache_attention against the 64-bit softmax, one row at a time.

Tolerance: half a unit of the output's type; the weights enter the second
product as f16 numbers (2^-11 of each, so of the mean of |value|), smaller than
2^-14 of the largest page scale they lose up to 2^-25 of it absolutely, times
the largest code; the fp32 logits are off by some 2^-20 of sums of |q k| up to
about 40, which is another 2^-14 of the weights."""
import pytest
import torch

import decode_ref as ref
from decode_common import make_cache, offsets_of
from paper_2607_16784_amd import api

pytestmark = pytest.mark.gpu
INT8, E4M3 = torch.int8, torch.float8_e4m3fn


def check(got, want, size, cache, lengths):
    top = ref.LARGEST[cache["v"].dtype] * float(cache["v_scale"][cache["v_scale"].isfinite()].max())
    tol = (ref.ROUND[got.dtype] * want.abs() + (2.0 ** -11 + 2.0 ** -13) * size +
           2.0 ** -25 * top * max(lengths + [1]) + 1e-7)
    err = (ref.f64(got) - want).abs()
    assert torch.all(err <= tol), f"worst {float((err / tol).max())}"


def run(lengths, new, heads, kv, page, dim, codes, dtype, seed, window=0, scale=None):
    cache, table, lens, _ = make_cache(lengths, kv, page, dim, codes, seed)
    g = torch.Generator().manual_seed(seed + 1)
    off = offsets_of(new)
    q = torch.randn((off[-1], heads, dim), generator=g).to(dtype).cuda()
    st = api.new_status()
    got = api.rm_cache_attention(q, cache, table, lens, status=st, window=window, scale=scale,
                                 token_offsets=torch.tensor(off, dtype=torch.int32).cuda(),
                                 max_tokens=max(new + [1]))
    assert int(st.item()) == 0
    want, size = ref.attention(q, cache, table, lengths, off, scale, window)
    check(got, want, size, cache, lengths)
    return got


DECODE = [
    # lengths, heads, kv, page, dim
    ([1], 1, 1, 16, 64),
    ([2, 15, 16, 17], 4, 4, 16, 128),
    ([63, 64, 65, 0, 128], 8, 2, 64, 128),
    ([129, 500], 5, 1, 32, 64),
    ([300, 1], 16, 1, 128, 256),
    ([700], 20, 1, 16, 128),
    ([257, 31], 34, 1, 64, 64),
    ([90, 1000, 7], 6, 3, 128, 128),
]


@pytest.mark.parametrize("codes", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("case", range(len(DECODE)))
def test_one_token_a_sequence(case, dtype, codes):
    lengths, heads, kv, page, dim = DECODE[case]
    run(lengths, [min(1, n) for n in lengths], heads, kv, page, dim, codes, dtype, seed=case)


CHUNKS = [
    # lengths, new, heads, kv, page, dim, window
    ([5], [5], 1, 1, 16, 64, 0),
    ([70, 33], [3, 33], 4, 2, 32, 128, 0),
    ([150], [40], 8, 2, 64, 128, 0),
    ([150, 90], [100, 17], 3, 1, 16, 64, 20),
    ([140], [30], 10, 5, 128, 256, 64),
    ([200, 200], [1, 50], 2, 2, 64, 128, 1),
    ([260], [70], 4, 1, 32, 256, 0),
    ([130], [130], 2, 1, 16, 128, 65),
]


@pytest.mark.parametrize("codes", [INT8, E4M3], ids=["int8", "e4m3"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("case", range(len(CHUNKS)))
def test_chunks_and_windows(case, dtype, codes):
    lengths, new, heads, kv, page, dim, window = CHUNKS[case]
    run(lengths, new, heads, kv, page, dim, codes, dtype, seed=40 + case, window=window)


def test_a_long_sequence_is_joined_from_its_parts():
    # too long for the row-by-row reference on the CPU: 64 bits on the GPU
    n, kv, page, dim, heads = 50001, 2, 64, 128, 8
    cache, table, lens, _ = make_cache([n], kv, page, dim, INT8, 60)
    q = torch.randn((1, heads, dim), device="cuda").bfloat16() * 3
    got = api.rm_cache_attention(q, cache, table, lens)
    p = table[0].long()
    k = cache["k"][p].double() * cache["k_scale"][p].double()[..., None, None]
    v = cache["v"][p].double() * cache["v_scale"][p].double()[..., None, None]
    k = k.transpose(0, 1).reshape(kv, -1, dim)[:, :n]
    v = v.permute(1, 0, 3, 2).reshape(kv, -1, dim)[:, :n]
    w = torch.softmax(torch.bmm(q[0].double().reshape(kv, heads // kv, dim),
                                k.transpose(1, 2).contiguous()) * dim ** -0.5, dim=-1)
    want = torch.bmm(w, v).reshape(1, heads, dim).cpu()
    size = torch.bmm(w, v.abs()).reshape(1, heads, dim).cpu()
    check(got, want, size, cache, [n])
    # the same whether or not the token axis is split over workgroups: a second
    # call gives the same bits
    assert torch.equal(got, api.rm_cache_attention(q, cache, table, lens))


def test_scale_and_sharp_softmax():
    run([200, 30], [1, 4], 4, 2, 32, 64, INT8, torch.float16, 61, scale=2.0)
    run([200], [1], 4, 2, 32, 64, E4M3, torch.bfloat16, 62, scale=-0.3)


def test_a_very_large_logit_in_every_place():
    # the running maximum moves late or early
    cache, table, lens, _ = make_cache([300], 1, 16, 64, INT8, 63)
    q = torch.randn((1, 1, 64), device="cuda").bfloat16()
    for at in (0, 15, 64, 200, 299):
        c = {n: t.clone() for n, t in cache.items()}
        page = int(table[0, at // 16])
        c["k"][page, 0, at % 16] = torch.where(q[0, 0] > 0, 127, -127).to(torch.int8)
        c["k_scale"][page, 0] *= 20
        got = api.rm_cache_attention(q, c, table, lens)
        want, size = ref.attention(q, c, table, [300])
        check(got, want, size, c, [300])


def test_page_scales_far_apart():
    cache, table, lens, _ = make_cache([200], 2, 16, 64, E4M3, 64)
    cache["v_scale"] *= torch.exp2(torch.randint(-20, 20, cache["v_scale"].shape).float()).cuda()
    cache["v_scale"][0] = 0.0
    q = torch.randn((1, 4, 64), device="cuda").half() * 0.1
    got = api.rm_cache_attention(q, cache, table, lens).double().cpu()
    want, size = ref.attention(q, cache, table, [200])
    fits = want.abs() < 60000
    top = 448 * float(cache["v_scale"].max())
    tol = ref.ROUND[torch.float16] * want.abs() + 2.0 ** -10 * size + 2.0 ** -25 * top * 200
    assert torch.all(((got - want).abs() <= tol)[fits])


@pytest.mark.parametrize("codes", [INT8, E4M3], ids=["int8", "e4m3"])
def test_what_is_not_seen_may_hold_anything(codes):
    # slots behind the last token, unused pages and pages before the window
    # hold the largest code or NaN, their scales NaN
    lengths, new, window = [37, 150], [3, 10], 40
    cache, table, lens, spare = make_cache(lengths, 2, 16, 64, codes, 65, spare=4)
    off = offsets_of(new)
    q = torch.randn((off[-1], 4, 64), device="cuda").bfloat16()
    kw = dict(token_offsets=torch.tensor(off, dtype=torch.int32, device="cuda"), max_tokens=10,
              window=window)
    want, size = ref.attention(q, cache, table, lengths, off, None, window)
    check(api.rm_cache_attention(q, cache, table, lens, **kw), want, size, cache, lengths)
    for b, n in enumerate(lengths):
        last = int(table[b, (n - 1) // 16])
        cache["k"].view(torch.uint8)[last, :, (n - 1) % 16 + 1:] = 0x7F
        cache["v"].view(torch.uint8)[last, :, :, (n - 1) % 16 + 1:] = 0x7F
    first = (lengths[1] - new[1] + 1 - window) // 16     # pages of sequence 1 before any window
    for p in spare.tolist() + table[1, :first].tolist():
        cache["k"].view(torch.uint8)[p] = 0x7F
        cache["v"].view(torch.uint8)[p] = 0x7F
        cache["k_scale"][p] = float("nan")
        cache["v_scale"][p] = float("nan")
    check(api.rm_cache_attention(q, cache, table, lens, **kw), want, size, cache, lengths)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("window", [0, 24])
def test_scales_that_are_not_finite_stay_with_the_rows_that_see_them(bad, window):
    # a chunk whose rows end in different pages: one page's scales spoil the
    # rows that see it and no others
    length, new = 90, 60
    cache, table, lens, _ = make_cache([length], 2, 16, 64, INT8, 71)
    q = torch.randn((new, 4, 64), device="cuda").bfloat16()
    kw = dict(token_offsets=torch.tensor([0, new], dtype=torch.int32, device="cuda"),
              max_tokens=new, window=window)
    want, size = ref.attention(q, cache, table, [length], [0, new], None, window)
    for page in range(6):
        for name in ("k_scale", "v_scale"):
            c = {n: t.clone() for n, t in cache.items()}
            c[name][int(table[0, page])] = bad
            got = api.rm_cache_attention(q, c, table, lens, **kw)
            pos = torch.arange(length - new, length)
            sees = (pos >= page * 16) & ((pos - window < page * 16 + 15) | (window == 0))
            free = (~sees).nonzero()[:, 0]
            check(got[free], want[free], size[free], cache, [length])
            # codes of 0 and +inf of the wrong sign aside, a seen one shows
            assert not torch.isfinite(got.cpu()[sees]).all() or not sees.any()


def test_small_weights_beside_a_large_one():
    # 4000 weights of 2^-20 to 2^-22 of the largest one: together 10^-3 of the
    # sum, on values that are all alike and 100 times the large one's
    cache, table, lens, _ = make_cache([4001], 1, 64, 64, INT8, 72)
    cache["k"].zero_()
    cache["v"].fill_(100)
    cache["k_scale"].fill_(1.0)
    cache["v_scale"].fill_(1.0)
    cache["k"][int(table[0, 5]), 0, 7, 0] = 112
    cache["v"][int(table[0, 5]), 0, :, 7] = 1
    q = torch.zeros((1, 1, 64), device="cuda").half()
    q[0, 0, 0] = 1.0
    w = 1 / (4000 * 2.718281828459045 ** -14 + 1)        # 112 / 8
    want = w * 1 + (1 - w) * 100
    got = api.rm_cache_attention(q, cache, table, lens).double()
    # f16 rounding of the output and of the weights, 2^-11 each
    assert float((got - want).abs().max()) < 2.0 ** -10 * want


def test_pages_that_no_row_sees_are_not_reported():
    cache, table, lens, _ = make_cache([200], 2, 16, 64, INT8, 73)
    q = torch.randn((1, 4, 64), device="cuda").bfloat16()
    want = api.rm_cache_attention(q, cache, table, lens, window=20)
    st = api.new_status()
    t = table.clone()
    t[0, :11] = -1                       # tokens 180 and later are seen
    got = api.rm_cache_attention(q, cache, t, lens, window=20, status=st)
    assert int(st.item()) == 0 and torch.equal(got, want)
    t[0, 11] = -1
    api.rm_cache_attention(q, cache, t, lens, window=20, status=st)
    assert int(st.item()) == api.ST_BAD_PAGE


def test_sequences_without_tokens_and_out_of_range():
    cache, table, lens, _ = make_cache([20, 40, 30, 50], 2, 16, 64, INT8, 66)
    q = torch.randn((4, 4, 64), device="cuda").bfloat16()
    good = api.rm_cache_attention(q, cache, table, lens)
    st = api.new_status()
    bad = lens.clone()
    bad[1], bad[2] = 0, 10 ** 6
    out = torch.full_like(q, 7.0)
    got = api.rm_cache_attention(q, cache, table, bad, out=out, status=st)
    assert torch.all(got[1:3] == 0) and torch.equal(got[[0, 3]], good[[0, 3]])
    assert int(st.item()) == api.ST_BAD_LENGTH
    # a page out of range is not seen: the result is that of the other tokens
    t = table.clone()
    t[3, 1] = cache["k"].shape[0]
    t[0, 0], t[0, 1] = -7, 10 ** 9
    st.zero_()
    got = api.rm_cache_attention(q, cache, t, lens, status=st)
    assert int(st.item()) == api.ST_BAD_PAGE
    assert torch.all(got[0] == 0) and torch.equal(got[1:3], good[1:3])
    short = {n: x.clone() for n, x in cache.items()}
    page = int(table[3, 1])
    keep = [j for j in range(50) if j // 16 != 1]
    k, v = (torch.stack([ref.cached({n: x.cpu() for n, x in short.items()}, table.cpu(), 50, 3,
                                    g)[i] for g in range(2)]) for i in range(2))
    for h in range(4):
        w = torch.softmax(k[h // 2, keep] @ ref.f64(q[3, h]) / 8, dim=0)
        assert float((w @ v[h // 2, keep] - ref.f64(got[3, h])).abs().max()) < 0.02
    assert page >= 0
    # with offsets, more tokens than the sequence holds: zeros
    st.zero_()
    out.fill_(7.0)
    off = torch.tensor([0, 3, 3, 3, 4], dtype=torch.int32, device="cuda")
    two = torch.tensor([2, 40, 30, 50], dtype=torch.int32, device="cuda")
    got = api.rm_cache_attention(q, cache, table, two, token_offsets=off, max_tokens=3, out=out,
                                 status=st)
    assert int(st.item()) == api.ST_BAD_LENGTH
    assert torch.all(got[:3] == 0) and torch.equal(got[3], good[3])


def test_infinite_and_nan_queries_stay_in_their_rows():
    cache, table, lens, _ = make_cache([100, 100], 1, 16, 64, INT8, 67)
    q = torch.randn((2, 3, 64), device="cuda").bfloat16()
    good = api.rm_cache_attention(q, cache, table, lens)
    q[0, 1, 3] = float("nan")
    q[1, 2] = float("inf")
    got = api.rm_cache_attention(q, cache, table, lens)
    assert torch.all(torch.isnan(got[0, 1])) and torch.all(torch.isnan(got[1, 2]))
    assert torch.equal(got[0, [0, 2]], good[0, [0, 2]]) and torch.equal(got[1, :2], good[1, :2])


def test_strided_queries():
    cache, table, lens, _ = make_cache([80, 33], 2, 32, 128, E4M3, 68)
    fused = torch.randn((2, 8, 128), device="cuda").half()
    q = fused[:, 1:5]
    got = api.rm_cache_attention(q, cache, table, lens)
    assert torch.equal(got, api.rm_cache_attention(q.contiguous(), cache, table, lens))


def test_many_heads_and_sequences():
    lengths = [(7 * i) % 90 for i in range(150)]
    run(lengths, [min(1, n) for n in lengths], 8, 4, 32, 64, INT8, torch.bfloat16, 69)


def test_refusals():
    cache, table, lens, _ = make_cache([20], 2, 16, 64, INT8, 70)
    q = torch.randn((1, 4, 64), device="cuda").bfloat16()

    def call(**kw):
        a = dict(q=q, cache=cache, table=table, lengths=lens)
        a.update(kw)
        return api.rm_cache_attention(**a)
    call()
    for kind, kw in [
            (ValueError, dict(q=q.float())), (ValueError, dict(q=q[:, :3])),
            (ValueError, dict(q=q[:, :, :32])), (ValueError, dict(q=q.cpu())),
            (ValueError, dict(lengths=lens.long())), (ValueError, dict(table=table[0])),
            (ValueError, dict(out=q.half())), (ValueError, dict(cache=api.new_cache(2, 2, 24, 64))),
            (RuntimeError, dict(window=-1)), (RuntimeError, dict(scale=float("nan"))),
            (RuntimeError, dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda")))]:
        with pytest.raises(kind):
            call(**kw)
    empty = torch.zeros((1, 4, 64), device="cuda").bfloat16()[:0]
    assert call(q=empty, lengths=lens, token_offsets=torch.zeros(2, dtype=torch.int32,
                                                                 device="cuda")).shape[0] == 0
