"""The prompt's operators and the 8-bit floating projection where offsets pass 2^31
elements or bytes."""
import pytest
import torch

import prompt_ref as ref
from paper_2607_16784_amd import api

pytestmark = pytest.mark.gpu


def test_rows_far_apart():
    # 20 000 rows 131 072 elements apart: 5 GB, the last rows beyond 2^31 elements
    n, wide = 20000, 131072
    rows = torch.zeros((n, wide), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(1)
    part = torch.randn((n, 4 * 64), generator=g).bfloat16().cuda()
    rows[:, 1000:1256] = part
    far = rows[:, 1000:1256].unflatten(1, (4, 64))
    near = part.view(n, 4, 64)
    off = torch.tensor([0, 19000, 19950, n], dtype=torch.int32, device="cuda")
    got = api.rm_prompt_attention(far[:, :2], far[:, 2:3], far[:, 3:], off, 19000, window=300)
    want = api.rm_prompt_attention(near[:, :2], near[:, 2:3], near[:, 3:], off, 19000, window=300)
    assert torch.equal(got, want)
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    f = (10000.0 ** (-torch.arange(0, 64, 2) / 64)).float().cuda()
    want = api.rm_head_norm_rotary(near[:, :2], near[:, 2:], f, at)
    q, k = far[:, :2], far[:, 2:]
    api.rm_head_norm_rotary(q, k, f, at, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    x = rows[:, 900:1300]
    codes, scales = api.rm_f8_quantize(x)
    again = api.rm_f8_quantize(x.contiguous())
    assert torch.equal(codes.view(torch.uint8), again[0].view(torch.uint8))
    assert torch.equal(scales, again[1])


def test_results_beyond_31_bits():
    rows, n, k = 40000, 60000, 128
    g = torch.Generator().manual_seed(2)
    x = torch.randn((rows, k), generator=g).bfloat16().cuda()
    codes, scales = api.rm_f8_quantize(torch.randn((n, k), generator=g).bfloat16().cuda(), 128)
    y = api.rm_f8_linear(x, codes, scales)
    for lo in (0, 17000, rows - 20):
        want, err = ref.f8_linear(x[lo:lo + 20], codes[n - 300:], scales[(n - 300) // 128:]) \
            if (n - 300) % 128 == 0 else ref.f8_linear(x[lo:lo + 20], codes, scales)
        got = ref.f64(y[lo:lo + 20])[:, -want.shape[1]:]
        tol = ref.ROUND[torch.bfloat16] * (want.abs() + err) * 1.01 + err
        assert torch.all((got - want).abs() <= tol), lo


@pytest.mark.parametrize("act", ["none", "swiglu"])
@pytest.mark.parametrize("given", [False, True])
def test_weights_whose_rows_are_far_apart(given, act):
    # rows 2^28 bytes apart: more than sixteen rows of x go sixteen at a time
    n, k, rows = 6, 200, 37
    g = torch.Generator().manual_seed(3)
    wide = torch.zeros((n, 1 << 28), dtype=torch.uint8, device="cuda")
    w = torch.randn((n, k), generator=g).bfloat16().cuda()
    codes, scales = api.rm_f8_quantize(w, 128)
    scales = scales.repeat(2, 1) if act == "swiglu" else scales
    wide[:, 100:100 + k] = codes.view(torch.uint8)
    far = wide.view(torch.float8_e4m3fn)[:, 100:100 + k]
    x = torch.randn((rows, k), generator=g).half().cuda()
    kw = dict(act=act, dtype=torch.float16)
    if given:
        x, kw["x_scales"] = api.rm_f8_quantize(x)
    got = api.rm_f8_linear(x, far, scales, **kw)
    one = {n_: v for n_, v in kw.items() if n_ != "x_scales"}
    for m in (0, 15, 16, 36):
        if given:
            one["x_scales"] = kw["x_scales"][m:m + 1].contiguous()
        assert torch.equal(got[m:m + 1], api.rm_f8_linear(x[m:m + 1], codes, scales, **one))
