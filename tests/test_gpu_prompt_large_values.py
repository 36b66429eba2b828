"""rm_prompt_attention over values near the largest of their type: a weighted mean of
them is within them, however many tokens there are (tolerances: prompt_ref)."""
import pytest
import torch

from test_gpu_prompt_attention import call, check, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("largest", [1e30, 1e36, 2e38, float(torch.finfo(torch.bfloat16).max)])
@pytest.mark.parametrize("lengths,window", [([1], 0), ([200, 70], 0), ([3000], 0), ([700], 130)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_means_of_large_values(dim, lengths, window, largest):
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    q, k, v = inputs(offsets[-1], 2, 1, dim, torch.bfloat16, 30)
    # values of one sign: their mean is as large as they are
    v = (v.double().abs() / float(v.abs().max()) * largest).to(torch.bfloat16)
    got, st = call(q, k, v, offsets, max(lengths), window=window)
    assert st == 0 and torch.all(torch.isfinite(got))
    check(got, q, k, v, offsets, torch.bfloat16, window=window)


@pytest.mark.parametrize("rising", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sign", [1, -1])
def test_the_largest_value_everywhere(sign, dtype, rising):
    # weights are rounded, their sum is not: the quotient may not leave the type
    n = 900
    q, k, v = (t.clone() for t in inputs(n, 2, 1, 64, dtype, 31))
    q[:, :, 0] = 4.0
    at = torch.arange(n, device="cuda") / 64.0
    k[:, :, 0] = (at if rising else -at)[:, None].to(dtype)
    v.fill_(sign * torch.finfo(dtype).max)
    v[:, :, 5] = 1.0
    v[300, :, 5] = -float("inf")
    got, _ = call(q, k, v, [0, n], n, scale=0.5)
    assert torch.all(torch.isfinite(got[:300])) and not torch.any(torch.isfinite(got[300:, :, 5]))
    # weights down to e^-27 (the rising logits and the others' spread): 0 in f16
    assert dtype is torch.float16 or torch.all(got[300:, :, 5] == -float("inf"))
    rest = [c for c in range(64) if c != 5]
    v[:, :, 5] = 1.0
    got[:, :, 5] = 1.0
    assert torch.all(torch.isfinite(got[:, :, rest]))
    check(got, q, k, v, [0, n], dtype, scale=0.5)


@pytest.mark.parametrize("power", [100, 110, -60])
def test_powers_of_two_pass_through(power):
    q, k, v = inputs(600, 4, 2, 64, torch.bfloat16, 32)
    want, _ = call(q, k, v, [0, 250, 600], 350)
    got, _ = call(q, k, torch.ldexp(v.float(), torch.tensor(power, device="cuda")).bfloat16(),
                  [0, 250, 600], 350)
    assert torch.equal(got.double(), want.double() * 2.0 ** power)
