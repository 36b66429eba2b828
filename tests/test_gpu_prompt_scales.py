"""rm_prompt_attention with scales at the ends of fp32's range (tolerances: prompt_ref)."""
import pytest
import torch

from test_gpu_prompt_attention import call, check, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1e-45, -1e-45, 2.3e38])
def test_logits_near_zero(scale):
    offsets = [0, 90, 150]
    q, k, v = (t.clone() for t in inputs(150, 4, 2, 64, torch.bfloat16, 40))
    if scale > 1:
        q.zero_()
    got, _ = call(q, k, v, offsets, 90, scale=scale)
    check(got, q, k, v, offsets, torch.bfloat16, scale=scale)


def test_a_scale_beyond_the_exponentials():
    q, k, v = inputs(20, 4, 2, 64, torch.bfloat16, 41)
    for scale in (2.4e38, -3e38):
        with pytest.raises(RuntimeError):
            call(q, k, v, [0, 20], 20, scale=scale)
