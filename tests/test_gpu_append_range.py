"""rm_rotary_append over the whole range of bf16: the largest values, and those
whose page scale is small.

Tolerances: those of test_gpu_cache_append (half a step of a code and 2^-20 of the
quotient).  A scale below 2^-126 is a subnormal fp32 number: it is within half of
2^-149 of the quotient, and the codes count in the scale that is stored."""
import pytest
import torch

import decode_ref as ref
from paper_2607_16784_amd import api
from test_gpu_cache_append import check_cache, step_of

pytestmark = pytest.mark.gpu
INT8, E4M3 = torch.int8, torch.float8_e4m3fn
BOTH = pytest.mark.parametrize("codes", [INT8, E4M3], ids=["int8", "e4m3"])


def tokens(tops, kv, dim, seed):
    """bf16 [tokens, kv, dim], token t's largest magnitude tops[t]; every channel
    another part of it, both signs, the largest itself among them."""
    g = torch.Generator().manual_seed(seed)
    x = torch.rand((len(tops), kv, dim), generator=g, dtype=torch.float64) * 2 - 1
    x[..., 3], x[..., dim - 2] = 1, -1
    return (x * torch.tensor(tops, dtype=torch.float64)[:, None, None]).to(torch.bfloat16)


def append(cache, x, start):
    """Appends x to the only sequence, whose pages are 0, 1, ..."""
    n = x.shape[0]
    table = torch.arange(cache["k"].shape[0], dtype=torch.int32, device="cuda")[None]
    api.rm_rotary_append(None, x.cuda(), x.cuda(), torch.zeros(0, device="cuda"), cache, table,
                         torch.tensor([start + n], dtype=torch.int32, device="cuda"),
                         token_offsets=torch.tensor([0, n], dtype=torch.int32, device="cuda"),
                         max_tokens=n)
    return table.cpu()


@BOTH
@pytest.mark.parametrize("tops", [[3e36], [3e38], [1e36, 3e38, 8e35], [2e37, 3e36, 1.0]])
def test_the_largest_values_keep_their_sign(tops, codes):
    cache = api.new_cache(2, 2, 16, 64, codes)
    x = tokens(tops, 2, 64, 1)
    table = append(cache, x, 0)
    check_cache(cache, ref.append(api.new_cache(2, 2, 16, 64, codes, device="cpu"), table,
                                  [len(tops)], [0, len(tops)], ref.f64(x), ref.f64(x)))


@BOTH
@pytest.mark.parametrize("first,second", [(1e30, 3e37), (3e37, 1e37), (5.0, 3.3e38)])
def test_large_values_behind_older_ones(first, second, codes):
    cache = api.new_cache(1, 2, 16, 64, codes)
    append(cache, tokens([first], 2, 64, 2), 0)
    before = {n: t.cpu().clone() for n, t in cache.items()}
    x = tokens([second, second / 4], 2, 64, 3)
    table = append(cache, x, 1)
    check_cache(cache, ref.append(before, table, [3], [0, 2], ref.f64(x), ref.f64(x)))


@BOTH
@pytest.mark.parametrize("first,second", [(4.5e-34, 4e-34), (4.5e-34, 6e-34), (4e-35, 3e-35),
                                          (4e-36, 1e-36), (1e-36, 4e-36)])
def test_small_values_beside_older_ones(first, second, codes):
    cache = api.new_cache(1, 2, 16, 64, codes)
    append(cache, tokens([first], 2, 64, 4), 0)
    before = {n: t.cpu().clone() for n, t in cache.items()}
    x = tokens([second, second / 2], 2, 64, 5)
    table = append(cache, x, 1)
    check_cache(cache, ref.append(before, table, [3], [0, 2], ref.f64(x), ref.f64(x)))


@BOTH
@pytest.mark.parametrize("top", [1e-36, 3e-37, 1e-38, 1e-39, 1e-40])
def test_codes_count_in_the_scale_that_is_stored(top, codes):
    cache = api.new_cache(1, 1, 16, 64, codes)
    x = tokens([top, top / 3], 1, 64, 6)
    append(cache, x, 0)
    for name in ("k", "v"):
        scale = float(cache[name + "_scale"][0, 0])
        largest = float(ref.f64(x).abs().max())
        assert abs(scale - largest / ref.LARGEST[codes]) <= 2.0 ** -150 + 2.0 ** -20 * scale
        c = ref.codes_f64(cache[name])[0, 0]
        c = (c if name == "k" else c.t())[:2]
        q = (ref.f64(x)[:, 0] / scale).clamp(-ref.LARGEST[codes], ref.LARGEST[codes])
        assert torch.all((c - q).abs() <= step_of(q, codes) * 0.5 + q.abs() * 2.0 ** -20)
