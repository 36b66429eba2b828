"""rm_cache_attention over values near the largest that bf16 holds: a weighted mean
of them is one of them, however many tokens there are.

Tolerance: test_gpu_attention_page_scales, check."""
import pytest
import torch

from decode_common import make_cache
from paper_2607_16784_amd import api
from test_gpu_attention_page_scales import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("codes", [torch.int8, torch.float8_e4m3fn], ids=["int8", "e4m3"])
@pytest.mark.parametrize("largest", [1e30, 1e36, 2e38])
@pytest.mark.parametrize("length,new", [(200, 1), (3000, 1), (90, 40), (2500, 20)])
def test_means_of_large_values(length, new, largest, codes):
    cache, table, lens, _ = make_cache([length], 1, 16, 64, codes, 85)
    cache["v_scale"].mul_(largest / (float(cache["v_scale"].max()) *
                                     (127 if codes == torch.int8 else 448)))
    # values of one sign: their mean is as large as they are
    cache["v"].view(torch.uint8).copy_(cache["v"].float().abs().to(codes).view(torch.uint8))
    q = torch.randn((new, 2, 64), device="cuda").bfloat16() * 0.1
    offsets = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    got = api.rm_cache_attention(q, cache, table, lens, token_offsets=offsets, max_tokens=new)
    assert torch.all(torch.isfinite(got))
    check(got, q, cache, table, [length], [0, new], 0)
