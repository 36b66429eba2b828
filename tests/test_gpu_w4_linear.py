"""rm_w4_linear against the 64-bit product with the weights the codes stand for.

Tolerance: half a unit of the output's type, plus what fp32 sums of terms of the
expanded codes can lose.  bf16 expands a code to 128 + code, so a partial sum is
up to 143 / 1 times sum |x| scale; 16 roundings of a group's sum (the matrix
instructions of a group and the subtraction) bound it by 2^-20 of that, and the
sum over groups adds as much.  f16 subtracts before the product: at most 15."""
import pytest
import torch

import decode_ref as ref
from paper_2607_16784_amd import api

pytestmark = pytest.mark.gpu


def inputs(rows, n, k, group, dtype, zeros, bias, seed, big=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((rows, k), generator=g) * big).to(dtype).cuda()
    codes = torch.randint(0, 256, (n, (k + 1) // 2), generator=g, dtype=torch.uint8).cuda()
    groups = -(-k // group)
    scales = (torch.rand((n, groups), generator=g) * 0.02 + 0.001).to(dtype).cuda()
    z = torch.randint(0, 16, (n, groups), generator=g, dtype=torch.uint8).cuda() if zeros else None
    b = torch.randn((n,), generator=g).to(dtype).cuda() if bias else None
    return x, codes, scales, z, b


def check(x, codes, scales, group, z, b, act, got):
    n, k = codes.shape[0], x.shape[1]
    want = ref.linear(x, codes, scales, group, z, b, act)
    s = ref.f64(scales).repeat_interleave(group, dim=1)[:, :k]
    size = ref.f64(x).abs() @ s.t() * (143 if x.dtype == torch.bfloat16 else 15)
    lost = 2.0 ** -19 * size
    if act == "swiglu":
        # |d silu(a)/da| < 1.1 and |silu(a)| <= |a|
        t = ref.linear(x, codes, scales, group, z, b)
        a, c = t.chunk(2, dim=1)
        lost = 1.1 * lost[:, :n // 2] * c.abs() + lost[:, n // 2:] * a.abs() + 2.0 ** -20 * want.abs()
    tol = ref.ROUND[x.dtype] * want.abs() + lost + 1e-7
    err = (ref.f64(got) - want).abs()
    assert torch.all(err <= tol), f"worst {float((err / tol).max())}"


CASES = [
    # rows, n, k, group, zeros, bias, act
    (1, 16, 128, 128, False, False, "none"),
    (1, 1, 1, 32, True, True, "none"),
    (2, 3, 31, 32, False, True, "none"),
    (1, 64, 4096, 128, True, False, "none"),
    (3, 17, 161, 32, True, False, "none"),
    (15, 33, 257, 64, False, False, "none"),
    (16, 100, 1000, 96, True, True, "none"),
    (17, 50, 512, 64, True, False, "swiglu"),
    (33, 34, 640, 256, False, True, "swiglu"),
    (64, 48, 1152, 128, True, False, "none"),
    (65, 65, 384, 32, False, False, "none"),
    (130, 20, 200, 224, True, False, "swiglu"),
    (5, 2, 2048, 1024, True, True, "swiglu"),
    (1, 200, 9001, 128, True, False, "none"),
    # every form: whole in LDS, wide, streams of one, two and four tiles, split
    (2, 16500, 300, 32, True, False, "none"),
    (3, 33000, 260, 128, False, True, "swiglu"),
    (16, 8300, 1056, 64, True, False, "none"),
    (9, 16600, 320, 32, False, False, "swiglu"),
    (16, 96, 11000, 128, False, False, "none"),
    (16, 64, 24000, 32, True, False, "none"),
    (20, 500, 9000, 96, True, True, "none"),
    (32, 130, 5000, 256, True, False, "swiglu"),
    (64, 300, 4100, 32, True, True, "none"),
    (61, 260, 9216, 128, True, False, "swiglu"),
    (200, 270, 2600, 64, False, True, "none"),
    # 64 rows a workgroup, in one part of the columns and in eight
    (40, 65550, 160, 64, True, False, "none"),
    (61, 65540, 140, 32, False, True, "swiglu"),
    (33, 8200, 8300, 128, True, False, "none"),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}x{c[1]}x{c[2]}-g{c[3]}-{c[6]}" for c in CASES])
def test_against_64_bits(case, dtype):
    rows, n, k, group, zeros, bias, act = case
    x, codes, scales, z, b = inputs(rows, n, k, group, dtype, zeros, bias, seed=rows * n + k)
    got = api.rm_w4_linear(x, codes, scales, group, zeros=z, bias=b, act=act)
    check(x, codes, scales, group, z, b, act, got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_strided_rows_and_unaligned_starts(dtype):
    # x a column range of a wider tensor at an odd element, codes a byte range
    # of wider rows at an odd byte, the output a column range too
    x, codes, scales, z, b = inputs(6, 40, 300, 64, dtype, True, True, seed=5)
    wide = torch.full((6, 411), float("nan"), dtype=dtype, device="cuda")
    wide[:, 5:305] = x
    rows = torch.full((40, 175), 255, dtype=torch.uint8, device="cuda")
    rows[:, 3:153] = codes
    out = torch.full((6, 90), 7.0, dtype=dtype, device="cuda")
    got = api.rm_w4_linear(wide[:, 5:305], rows[:, 3:153], scales, 64, zeros=z, bias=b,
                           out=out[:, 11:51])
    check(x, codes, scales, 64, z, b, "none", got)
    assert torch.all(out[:, :11] == 7) and torch.all(out[:, 51:] == 7)
    assert torch.equal(got, api.rm_w4_linear(x, codes, scales, 64, zeros=z, bias=b))


def test_nothing_is_read_behind_a_row():
    # the columns behind k hold NaN, and so do the rows behind the last one
    x, codes, scales, z, b = inputs(3, 20, 133, 32, torch.bfloat16, False, False, seed=6)
    wide = torch.full((5, 200), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:3, :133] = x
    got = api.rm_w4_linear(wide[:3, :133], codes, scales, 32)
    check(x, codes, scales, 32, None, None, "none", got)


def test_the_same_result_every_time():
    x, codes, scales, z, b = inputs(9, 500, 7000, 128, torch.bfloat16, True, False, seed=7)
    first = api.rm_w4_linear(x, codes, scales, 128, zeros=z)
    for _ in range(3):
        assert torch.equal(first, api.rm_w4_linear(x, codes, scales, 128, zeros=z))


def test_a_row_does_not_depend_on_the_others():
    x, codes, scales, z, b = inputs(4, 64, 512, 128, torch.float16, True, False, seed=8)
    x[1] = float("nan")
    x[2, 5] = float("inf")
    got = api.rm_w4_linear(x, codes, scales, 128, zeros=z)
    assert torch.all(torch.isnan(got[1])) and not torch.any(torch.isfinite(got[2]))
    check(x[[0, 3]], codes, scales, 128, z, None, "none", got[[0, 3]])


def test_large_sums_stay_in_32_bits():
    # 8192 products of one sign near f16's largest: partial sums beyond 65504
    x = torch.full((1, 8192), 60.0, dtype=torch.float16, device="cuda")
    codes = torch.full((16, 4096), 0xFF, dtype=torch.uint8, device="cuda")
    scales = torch.full((16, 64), 0.015625, dtype=torch.float16, device="cuda")
    got = api.rm_w4_linear(x, codes, scales, 128)
    assert torch.all(got == torch.tensor(8192 * 60 * 7 * 0.015625, dtype=torch.float16))


def test_refusals():
    x, codes, scales, z, b = inputs(2, 8, 64, 32, torch.bfloat16, True, True, seed=9)
    ok = dict(zeros=z, bias=b)
    api.rm_w4_linear(x, codes, scales, 32, **ok)
    bad = [
        (ValueError, lambda: api.rm_w4_linear(x.float(), codes, scales, 32)),
        (ValueError, lambda: api.rm_w4_linear(x.cpu(), codes, scales, 32)),
        (ValueError, lambda: api.rm_w4_linear(x, codes[:, :31], scales, 32)),
        (ValueError, lambda: api.rm_w4_linear(x, codes, scales.half(), 32)),
        (ValueError, lambda: api.rm_w4_linear(x, codes, scales, 48)),
        (ValueError, lambda: api.rm_w4_linear(x, codes, scales[:, :1], 32)),
        (ValueError, lambda: api.rm_w4_linear(x, codes, scales, 32, zeros=z.int())),
        (ValueError, lambda: api.rm_w4_linear(x, codes, scales, 32, bias=b[:4])),
        (ValueError, lambda: api.rm_w4_linear(x, codes, scales, 32, act="relu")),
        (ValueError, lambda: api.rm_w4_linear(x.t().contiguous().t(), codes, scales, 32)),
        (ValueError, lambda: api.rm_w4_linear(x[:1].expand(2, 64), codes, scales, 32)),
        (ValueError, lambda: api.rm_w4_linear(x, codes, scales, 32, out=x)),
        (RuntimeError, lambda: api.rm_w4_linear(x, codes[:7], scales[:7], 32, act="swiglu")),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [1, 16, 40])
def test_a_group_of_any_size_beyond_k_is_one_group(rows, dtype):
    x, codes, scales, z, b = inputs(rows, 96, 1100, 1120, dtype, True, True, seed=95)
    want = api.rm_w4_linear(x, codes, scales, 1120, zeros=z, bias=b)
    check(x, codes, scales, 1120, z, b, "none", want)
    for group in (1 << 20, (1 << 31) - 32):
        assert torch.equal(api.rm_w4_linear(x, codes, scales, group, zeros=z, bias=b), want)


def test_no_rows():
    x, codes, scales, z, b = inputs(2, 8, 64, 32, torch.bfloat16, False, False, seed=9)
    assert api.rm_w4_linear(x[:0], codes, scales, 32).shape == (0, 8)
