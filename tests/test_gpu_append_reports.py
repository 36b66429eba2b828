"""rm_rotary_append reports sequences that are out of range also where it has no
pages to write."""
import pytest
import torch

from decode_common import make_cache
from paper_2607_16784_amd import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("queries", [True, False])
@pytest.mark.parametrize("offsets,bad", [([0, 2, 4], True), ([0, 0, 3], True), ([0, 0, 0], False)])
def test_max_tokens_of_0(offsets, bad, queries):
    cache, table, lens, _ = make_cache([20, 30], 2, 16, 64, torch.int8, 96)
    before = {n: t.clone() for n, t in cache.items()}
    k = torch.randn((4, 2, 64), device="cuda").bfloat16()
    st = api.new_status()
    api.rm_rotary_append(k if queries else None, k, k, torch.ones(32, device="cuda"), cache, table,
                         lens, max_tokens=0, status=st,
                         token_offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"))
    assert int(st.item()) == (api.ST_BAD_LENGTH if bad else 0)
    for n in cache:
        assert torch.equal(cache[n].view(torch.uint8), before[n].view(torch.uint8)), n
