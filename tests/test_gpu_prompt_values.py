"""rm_prompt_attention over values that are not finite, against the definition: a row
gets what it sees of them, and the other channels and rows their finite results
(tolerances: prompt_ref)."""
import pytest
import torch

import prompt_ref as ref
from test_gpu_prompt_attention import call, inputs

pytestmark = pytest.mark.gpu


def check(got, q, k, v, offsets, dtype, window=0):
    """Every weight that a row gives is above 0 in q's type."""
    clean = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    want, size, off = ref.attention(q, k, clean, offsets, window=window)
    lengths = [b - a for a, b in zip(offsets, offsets[1:])]
    tol = ref.attention_tolerance(want, size, off, lengths, dtype, float(clean.abs().max()))
    odd, per = ref.f64(torch.where(torch.isfinite(v), 0 * clean, v)), q.shape[1] // k.shape[1]
    for t, g, c in torch.nonzero(odd).tolist():
        for lo, hi in zip(offsets, offsets[1:]):
            if lo <= t < hi:
                rows = slice(t, min(hi, t + window) if window else hi)
                want[rows, g * per:(g + 1) * per, c] += odd[t, g, c]
    got, finite = ref.f64(got), torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf])
    assert torch.all((got - want).abs()[finite] <= tol[finite])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,window", [(64, 0), (128, 0), (256, 0), (64, 40), (128, 100)])
@pytest.mark.parametrize("aligned", [True, False])
def test_infinite_values(dim, window, dtype, aligned):
    offsets = ref.offsets_of([400, 1, 70], first=2)
    q, k, v = inputs(480, 4, 2, dim, dtype, 20)
    v = v.clone() if aligned else torch.nn.functional.pad(v, (1, 0))[:, :, 1:]
    inf = float("inf")
    # first rows, both sides of a step's border, the last row, one of no sequence
    for at, c, bad in ((2, 0, inf), (2, 7, -inf), (65, 9, inf), (66, 3, -inf), (130, 9, -inf),
                       (300, 5, inf), (401, 1, inf), (402, 2, -inf), (403, 2, inf),
                       (440, 63, float("nan")), (472, 4, inf), (478, 6, inf)):
        v[at, 1, c] = bad
    got, st = call(q, k, v, offsets, 400, window=window)
    assert st == 0
    check(got, q, k, v, offsets, dtype, window)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_one_token(dtype):
    q, k, v = inputs(3, 2, 1, 64, dtype, 21)
    v = v.clone()
    v[0, 0, :3] = v.new_tensor([float("inf"), -float("inf"), float("nan")])
    got, _ = call(q, k, v, [0, 1, 2, 3], 1)
    assert torch.equal(got[1:], v[1:].expand(2, 2, 64))
    assert torch.equal(torch.nan_to_num(got[0], nan=5.0),
                       torch.nan_to_num(v[0].expand(2, 64), nan=5.0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128])
def test_infinite_values_of_weight_zero(dim, dtype):
    # a logit of -infinity: 0 times infinity, wherever the rows stand
    n, at = 330, 70
    q, k, v = (t.clone() for t in inputs(n, 4, 2, dim, dtype, 22))
    q[:, :, 0] = 1.0
    k[at, 1, 0] = -float("inf")
    v[at, 1, 5] = float("inf")
    got, _ = call(q, k, v, [0, n], n)
    assert torch.all(torch.isnan(got[at:, 2:, 5]))
    rest = [c for c in range(dim) if c != 5]
    assert torch.all(torch.isfinite(got[:, :, rest])) and torch.all(torch.isfinite(got[:at]))
    # the heads of that key: the other channels are those of the tokens without it
    keep = [t for t in range(n) if t != at]
    want, size, off = ref.attention(q[keep], k[keep], v[keep], [0, n - 1])
    tol = ref.attention_tolerance(want, size, off, [n - 1], dtype, float(v[keep].abs().max()))
    assert torch.all(((ref.f64(got[keep]) - want).abs() <= tol)[:, 2:, rest])
