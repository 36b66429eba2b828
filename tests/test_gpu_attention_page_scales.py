"""rm_cache_attention where finite page scales lie far apart: a page has no say in
the precision of rows that do not see it, or that give it next to no weight.

Tolerance: half a unit of bf16; the f16 weights (2^-11 of each) and the fp32
logits (2^-13) are relative to the mean of |value| under the weights; weights
below 2^-28 of the row's largest weight times scale lose up to 2^-39 of that each,
times the largest code: `cap` holds the sum of weight times scale times that code."""
import pytest
import torch

import decode_ref as ref
from decode_common import make_cache
from paper_2607_16784_amd import api

pytestmark = pytest.mark.gpu
INT8, E4M3 = torch.int8, torch.float8_e4m3fn
BOTH = pytest.mark.parametrize("codes", [INT8, E4M3], ids=["int8", "e4m3"])


def check(got, q, cache, table, lengths, offsets, window, rows=slice(None)):
    want, size = ref.attention(q, cache, table, lengths, offsets, None, window)
    top = ref.LARGEST[cache["v"].dtype]
    full = dict(cache, v=torch.full(cache["v"].shape, top).to(cache["v"].dtype))
    cap = ref.attention(q, full, table, lengths, offsets, None, window)[1]
    tol = (ref.ROUND[got.dtype] * want.abs() + (2.0 ** -11 + 2.0 ** -13) * size +
           2.0 ** -38 * max(lengths) * cap)
    err = (ref.f64(got) - want).abs()
    assert torch.all((err <= tol)[rows]), f"worst {float((err / tol)[rows].max())}"


@BOTH
@pytest.mark.parametrize("window", [0, 24])
@pytest.mark.parametrize("factor", [2.0 ** 40, 2.0 ** -40])
def test_a_page_of_another_magnitude(factor, window, codes):
    # a chunk whose rows end in different pages, some before the one that differs
    length, new = 90, 60
    cache, table, lens, _ = make_cache([length], 2, 16, 64, codes, 81)
    q = torch.randn((new, 4, 64), device="cuda").bfloat16()
    for page in range(6):
        c = dict(cache, v_scale=cache["v_scale"].clone())
        c["v_scale"][int(table[0, page])] *= factor
        got = api.rm_cache_attention(
            q, c, table, lens, max_tokens=new, window=window,
            token_offsets=torch.tensor([0, new], dtype=torch.int32, device="cuda"))
        check(got, q, c, table, [length], [0, new], window)


@BOTH
@pytest.mark.parametrize("at", [0, 3, 18])
def test_a_large_page_with_next_to_no_weight(at, codes):
    # keys of one page give logits of -60: weights of e^-60 on values 2^40 larger
    length = 300
    cache, table, lens, _ = make_cache([length], 1, 16, 64, codes, 82)
    q = torch.ones((1, 2, 64), device="cuda").bfloat16()
    cache["k"].view(torch.uint8).zero_()
    page = int(table[0, at])
    cache["k"][page] = torch.full((1, 16, 64), -60.0).to(codes).cuda()
    cache["k_scale"][page] = 60 / (60 * 64 / 8)
    cache["v_scale"][page] *= 2.0 ** 40
    got = api.rm_cache_attention(q, cache, table, lens)
    check(got, q, cache, table, [length], None, 0)


@BOTH
def test_a_page_that_only_the_window_of_earlier_rows_holds(codes):
    # the blocks behind a large page: rows whose window has left it
    length, new, window = 400, 300, 40
    cache, table, lens, _ = make_cache([length], 1, 16, 64, codes, 83)
    cache["v_scale"][int(table[0, 4])] *= 2.0 ** 40
    q = torch.randn((new, 1, 64), device="cuda").bfloat16()
    got = api.rm_cache_attention(
        q, cache, table, lens, max_tokens=new, window=window,
        token_offsets=torch.tensor([0, new], dtype=torch.int32, device="cuda"))
    check(got, q, cache, table, [length], [0, new], window)
