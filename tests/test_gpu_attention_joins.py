"""rm_cache_attention where the token axis is split over workgroups and joined:
tiles of 16 and of 32 rows, several of them, every head size, windows that leave
parts empty, sequences without tokens or out of range.

Tolerance: test_gpu_cache_attention, check."""
import pytest
import torch

import decode_ref as ref
from decode_common import make_cache, offsets_of
from paper_2607_16784_amd import api
from test_gpu_cache_attention import check

pytestmark = pytest.mark.gpu
INT8, E4M3 = torch.int8, torch.float8_e4m3fn

CASES = [
    # lengths, new, heads, kv, page, dim
    ([1500, 0, 900], [70, 0, 1], 4, 2, 16, 64),
    ([1500, 0, 900], [70, 0, 1], 2, 1, 64, 128),
    ([1500, 0, 900], [40, 0, 1], 2, 1, 32, 256),
    ([1300], [9], 8, 1, 128, 256),
    ([1030, 1], [1, 1], 40, 1, 16, 128),
    ([2100, 64, 65], [33, 64, 1], 3, 3, 64, 64),
]


def run(case, codes, dtype, window, seed):
    lengths, new, heads, kv, page, dim = case
    cache, table, lens, _ = make_cache(lengths, kv, page, dim, codes, seed)
    off = offsets_of(new)
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn((off[-1], heads, dim), generator=g).to(dtype).cuda()
    kw = dict(token_offsets=torch.tensor(off, dtype=torch.int32, device="cuda"),
              max_tokens=max(new), window=window)
    return q, cache, table, lens, off, kw


@pytest.mark.parametrize("codes,dtype", [(INT8, torch.bfloat16), (E4M3, torch.float16),
                                         (E4M3, torch.bfloat16), (INT8, torch.float16)])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_joined_parts(case, window, codes, dtype):
    q, cache, table, lens, off, kw = run(CASES[case], codes, dtype, window, 110 + case)
    st = api.new_status()
    with api.rm_trace() as t:
        got = api.rm_cache_attention(q, cache, table, lens, status=st, **kw)
    assert len(t.launches) == 2 and int(st.item()) == 0
    want, size = ref.attention(q, cache, table, CASES[case][0], off, None, window)
    check(got, want, size, cache, CASES[case][0])


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 300])
def test_one_part_and_several(window, dim):
    # a table that could name more pages splits the same tokens
    case = ([700, 300], [50, 1], 4, 2, 32, dim)
    q, cache, table, lens, off, kw = run(case, INT8, torch.bfloat16, window, 120)
    with api.rm_trace() as one:
        a = api.rm_cache_attention(q, cache, table, lens, **kw)
    wide = torch.full((2, 200), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    with api.rm_trace() as several:
        b = api.rm_cache_attention(q, cache, wide, lens, **kw)
    assert len(one.launches) == 1 and len(several.launches) == 2
    want, size = ref.attention(q, cache, table, case[0], off, None, window)
    check(a, want, size, cache, case[0])
    check(b, want, size, cache, case[0])


@pytest.mark.parametrize("dim", [64, 256])
def test_bad_pages_and_lengths_among_joined_parts(dim):
    case = ([1500, 900, 1000, 800], [40, 1, 3, 2], 4, 2, 16, dim)
    q, cache, table, lens, off, kw = run(case, E4M3, torch.bfloat16, 0, 130)
    good = api.rm_cache_attention(q, cache, table, lens, **kw)
    bad, st = lens.clone(), api.new_status()
    bad[1] = 10 ** 6
    t = table.clone()
    t[2, :] = -1                          # sequence 2 has no page in range
    out = torch.full_like(q, 7.0)
    got = api.rm_cache_attention(q, cache, t, bad, out=out, status=st, **kw)
    assert int(st.item()) == api.ST_BAD_LENGTH | api.ST_BAD_PAGE
    assert torch.all(got[off[1]:off[3]] == 0)
    assert torch.equal(got[:off[1]], good[:off[1]]) and torch.equal(got[off[3]:], good[off[3]:])
    # one page of many is not seen: the result of the other tokens
    t = table.clone()
    t[3, 20] = cache["k"].shape[0]
    st.zero_()
    got = api.rm_cache_attention(q, cache, t, lens, status=st, **kw)
    assert int(st.item()) == api.ST_BAD_PAGE
    assert torch.equal(got[:off[3]], good[:off[3]])
    host = {n: x.cpu() for n, x in cache.items()}
    for g in range(2):
        k, v = ref.cached(host, table.cpu(), 800, 3, g)
        for row, last in ((off[3], 799), (off[3] + 1, 800)):
            keep = [j for j in range(last) if j // 16 != 20]
            for h in (2 * g, 2 * g + 1):
                w = torch.softmax(k[keep] @ ref.f64(q[row, h]) * dim ** -0.5, dim=0)
                want, size = w @ v[keep], w @ v[keep].abs()
                tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -13) * size + 1e-5
                assert torch.all((ref.f64(got[row, h]) - want).abs() <= tol)
