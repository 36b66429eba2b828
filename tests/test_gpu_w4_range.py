"""rm_w4_linear over the whole range of bf16 inputs.

Tolerance: that of test_gpu_w4_linear (half a unit of the output, 2^-19 of the sum
of |x| scale times 143) without its absolute term; in its place what fp32
subnormals can lose: the terms are held 2^-15 low, so a rounding is 2^-135 of the
scale, and 24 of them a group are allowed."""
import pytest
import torch

import decode_ref as ref
from paper_2607_16784_amd import api
from test_gpu_w4_linear import inputs

pytestmark = pytest.mark.gpu

# rows, n, k, group: every form of the kernel, ends that no batch covers among them
SIZES = [(1, 40, 300, 64), (4, 16500, 256, 128), (9, 130, 700, 32), (16, 8300, 544, 128),
         (20, 500, 2100, 96), (33, 270, 640, 64), (40, 65550, 160, 32)]


def check(x, codes, scales, group, z, b, got):
    n, k = codes.shape[0], x.shape[1]
    want = ref.linear(x, codes, scales, group, z, b)
    s = ref.f64(scales).repeat_interleave(group, dim=1)[:, :k]
    lost = 2.0 ** -19 * 143 * (ref.f64(x).abs() @ s.t())
    small = 24 * 2.0 ** -135 * ref.f64(scales).sum(dim=1)[None] + 2.0 ** -133
    tol = ref.ROUND[x.dtype] * want.abs() + lost + small
    err = (ref.f64(got) - want).abs()
    assert torch.all(err <= tol), f"worst {float((err / tol).max())}"


@pytest.mark.parametrize("size", SIZES, ids=["x".join(map(str, s)) for s in SIZES])
@pytest.mark.parametrize("big", [1e34, 4e36, 1e38])
def test_large_inputs(big, size):
    rows, n, k, group = size
    x, codes, scales, z, _ = inputs(rows, n, k, group, torch.bfloat16, True, False, seed=rows + n)
    x = (ref.f64(x) * big).clamp(-3.3e38, 3.3e38).bfloat16().cuda()
    scales = (scales.float() * 2.0 ** -9).bfloat16()
    got = api.rm_w4_linear(x, codes, scales, group, zeros=z)
    check(x, codes, scales, group, z, None, got)


@pytest.mark.parametrize("rows", [1, 16, 40])
def test_the_largest_input_everywhere(rows):
    k, n = 8192, 64
    x = torch.full((rows, k), 3.3895e38, dtype=torch.bfloat16, device="cuda")
    codes = torch.full((n, k // 2), 0xFF, dtype=torch.uint8, device="cuda")
    codes[1::2] = 0x00
    scales = torch.full((n, k // 128), 2.0 ** -17, dtype=torch.bfloat16, device="cuda")
    got = api.rm_w4_linear(x, codes, scales, 128)
    check(x, codes, scales, 128, None, None, got)


def test_large_inputs_behind_a_gate():
    x, codes, scales, z, _ = inputs(5, 80, 300, 64, torch.bfloat16, True, False, seed=3, big=1e37)
    scales = scales.float()
    scales[:40] *= 2.0 ** -120                   # gates of some 1
    got = api.rm_w4_linear(x, codes, scales.bfloat16(), 64, zeros=z, act="swiglu")
    want = ref.linear(x, codes, scales.bfloat16(), 64, z, None, "swiglu")
    # bf16 ends at 3.39e38; a few products of gate and value are beyond
    fits, beyond = want.abs() < 3.38e38, want.abs() > 3.41e38
    assert int(beyond.sum()) == 5 and torch.all(fits | beyond)
    got = ref.f64(got)
    assert torch.all(torch.isfinite(got[fits])) and torch.all(got[beyond] == want[beyond] * float("inf"))
    # what 143 times the terms loses in fp32, of terms that partly cancel
    assert float((got - want)[fits].norm() / want[fits].norm()) < 2.0 ** -8


@pytest.mark.parametrize("size", SIZES, ids=["x".join(map(str, s)) for s in SIZES])
@pytest.mark.parametrize("small", [1e-30, 1e-34, 1e-36, 1e-38])
def test_small_inputs(small, size):
    rows, n, k, group = size
    x, codes, scales, z, _ = inputs(rows, n, k, group, torch.bfloat16, True, False, seed=rows + n)
    x = (ref.f64(x) * small).bfloat16().cuda()
    got = api.rm_w4_linear(x, codes, scales, group, zeros=z)
    check(x, codes, scales, group, z, None, got)
