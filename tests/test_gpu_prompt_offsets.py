"""rm_prompt_attention with offsets that decrease and a window: reported, and nothing
outside of `out` is touched (which rows a workgroup takes: test_prompt_slots)."""
import random

import pytest
import torch

from paper_2607_16784_amd import api

pytestmark = pytest.mark.gpu


def cases():
    yield [0, 1000, 1200, 500, 600, 700, 1500], 1500, 64, 4
    yield [0, 900, 1000, 0, 0, 1000], 1000, 64, 4
    rng = random.Random(3)
    for turn in range(12):
        tokens = rng.choice([130, 700, 1500])
        offsets = [rng.randint(0, tokens) for _ in range(rng.randint(3, 90))]
        if offsets == sorted(offsets):
            offsets.reverse()
        yield offsets, tokens, rng.choice([1, 64, 100]), rng.choice([1, 4, 5])


CASES = list(cases())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_offsets_that_decrease(case, dim):
    offsets, tokens, window, group = CASES[case]
    g = torch.Generator().manual_seed(case)
    qkv = torch.randn((tokens, 2 * group + 4, dim), generator=g).bfloat16().cuda()
    q, k, v = qkv.split([2 * group, 2, 2], dim=1)
    off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    wide = torch.full((tokens + 64, 2 * group, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    st = api.new_status()
    api.rm_prompt_attention(q, k, v, off, tokens, window=window, out=wide[32:32 + tokens],
                            status=st)
    assert int(st.item()) == api.ST_BAD_LENGTH
    assert torch.all(wide[:32] == 7) and torch.all(wide[32 + tokens:] == 7)
    # the same call with the offsets in order is none the worse
    order, st = off.sort()[0].int(), api.new_status()
    got = api.rm_prompt_attention(q, k, v, order, tokens, window=window, status=st)
    assert int(st.item()) == 0 and torch.all(torch.isfinite(got))
