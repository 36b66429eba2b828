"""rm_head_norm_rotary against its 64-bit definition.

Tolerance: half a unit of the output's type plus 2^-19 of the result's largest
terms: squares summed in a tree of at most 14 levels (2^-20), the root and the
quotient, the angle (1.3e-7 and 9e-8) and three products."""
import pytest
import torch

import prompt_ref as ref
from paper_2607_16784_amd import api

pytestmark = pytest.mark.gpu


def inputs(tokens, heads, kv, dim, rot, dtype, seed, far=4096):
    g = torch.Generator().manual_seed(seed)

    def r(*shape):
        return torch.randn(shape, generator=g)
    qkv = (r(tokens, heads + 2 * kv, dim) * torch.exp(r(tokens, heads + 2 * kv, 1))).to(dtype).cuda()
    return dict(q=qkv[:, :heads], k=qkv[:, heads:heads + kv],
                q_weight=(1 + r(dim) / 4).to(dtype).cuda(),
                k_weight=(1 + r(dim) / 4).to(dtype).cuda(),
                positions=torch.randint(0, far, (tokens,), generator=g, dtype=torch.int32).cuda(),
                inv_freq=(10000.0 ** (-torch.arange(0, rot, 2) / max(rot, 1))).float().cuda())


def check(got, x, weight, p, dtype, layout="half", rot_scale=1.0, eps=1e-6):
    want, size = ref.head_norm(x, weight, p["positions"].tolist(), p["inv_freq"].tolist(), layout,
                               rot_scale, eps)
    tol = ref.ROUND[dtype] * want.abs() + 2.0 ** -19 * size
    err = (ref.f64(got) - want).abs()
    worst = float((err / tol).max()) if err.numel() else 0.0
    assert worst <= 1, worst


SIZES = [(1, 1, 1, 8, 8), (1, 32, 8, 128, 128), (3, 5, 1, 16, 4), (7, 4, 4, 24, 16), (2, 3, 2, 64, 64),
         (5, 20, 4, 80, 36), (9, 7, 1, 96, 48), (4, 64, 8, 128, 64), (33, 6, 2, 256, 256),
         (2, 2, 1, 264, 128), (3, 3, 1, 512, 512), (2, 16, 2, 72, 72), (2, 17, 16, 128, 2),
         (3, 4, 2, 64, 0), (1, 200, 1, 64, 32), (700, 8, 2, 64, 64)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("size", SIZES, ids=["x".join(map(str, s)) for s in SIZES])
def test_against_64_bits(size, layout, dtype):
    tokens, heads, kv, dim, rot = size
    p = inputs(tokens, heads, kv, dim, rot, dtype, sum(size))
    q, k = api.rm_head_norm_rotary(p["q"], p["k"], p["inv_freq"], p["positions"],
                                   q_weight=p["q_weight"], k_weight=p["k_weight"], layout=layout,
                                   rot_scale=1.25, eps=1e-5)
    assert q.shape == p["q"].shape and k.shape == p["k"].shape
    check(q, p["q"], p["q_weight"], p, dtype, layout, 1.25, 1e-5)
    check(k, p["k"], p["k_weight"], p, dtype, layout, 1.25, 1e-5)


@pytest.mark.parametrize("rot", [64, 40, 20])
def test_one_side_without_weights_and_far_positions(rot):
    p = inputs(6, 4, 2, 64, rot, torch.float16, 7, far=2 ** 31 - 1)
    q, none = api.rm_head_norm_rotary(p["q"], None, p["inv_freq"], p["positions"])
    assert none is None
    check(q, p["q"], None, p, torch.float16)
    none, k = api.rm_head_norm_rotary(None, p["k"], p["inv_freq"], p["positions"])
    assert none is None
    check(k, p["k"], None, p, torch.float16)
    both = api.rm_head_norm_rotary(p["q"], p["k"], p["inv_freq"], p["positions"])
    assert torch.equal(both[0], q) and torch.equal(both[1], k)


def test_negative_positions_turn_back():
    p = inputs(4, 2, 1, 64, 64, torch.bfloat16, 8)
    p["positions"] = -p["positions"]
    q, _ = api.rm_head_norm_rotary(p["q"], None, p["inv_freq"], p["positions"])
    check(q, p["q"], None, p, torch.bfloat16)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [128, 64, 36])
def test_in_place_and_strided(layout, rot):
    # in the fused projection's rows, at an address that is no multiple of 16
    p = inputs(50, 6, 3, 128, rot, torch.bfloat16, 9)
    kw = dict(q_weight=p["q_weight"], k_weight=p["k_weight"], layout=layout)
    want = api.rm_head_norm_rotary(p["q"], p["k"], p["inv_freq"], p["positions"], **kw)
    rows = torch.zeros((50, 12 * 128 + 9), dtype=torch.bfloat16, device="cuda")
    qkv = rows[:, 3:3 + 12 * 128].unflatten(1, (12, 128))
    qkv[:, :6].copy_(p["q"])
    qkv[:, 6:9].copy_(p["k"])
    qkv[:, 9:].fill_(7.0)
    q, k = qkv[:, :6], qkv[:, 6:9]
    got = api.rm_head_norm_rotary(q, k, p["inv_freq"], p["positions"], q_out=q, k_out=k, **kw)
    assert got[0] is q and got[1] is k
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.all(qkv[:, 9:] == 7.0) and torch.all(rows[:, :3] == 0)
    assert torch.all(rows[:, 3 + 12 * 128:] == 0)
    # heads in front of the tokens
    turned = torch.empty((6, 50, 128), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    api.rm_head_norm_rotary(p["q"], p["k"], p["inv_freq"], p["positions"], q_out=turned, **kw)
    assert torch.equal(turned, want[0])


def test_what_is_not_finite_stays_in_its_head():
    p = inputs(4, 4, 2, 128, 64, torch.float16, 10)
    clean, _ = api.rm_head_norm_rotary(p["q"], None, p["inv_freq"], p["positions"])
    q = p["q"].clone()
    q[1, 2, 5], q[2, 0, 100], q[3, 3, 127] = float("nan"), float("inf"), -float("inf")
    got, _ = api.rm_head_norm_rotary(q, None, p["inv_freq"], p["positions"])
    bad = torch.zeros(4, 4, dtype=torch.bool)
    bad[1, 2] = bad[2, 0] = bad[3, 3] = True
    assert torch.all(torch.isnan(got[1, 2]))
    assert torch.equal(got[~bad.cuda()], clean[~bad.cuda()])
    zero = torch.zeros_like(q)
    got, _ = api.rm_head_norm_rotary(zero, None, p["inv_freq"], p["positions"])
    assert torch.all(got == 0)


def test_no_tokens():
    p = inputs(3, 4, 2, 64, 64, torch.float16, 11)
    q, k = api.rm_head_norm_rotary(p["q"][:0], p["k"][:0], p["inv_freq"], p["positions"][:0])
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)


def test_refusals():
    p = inputs(3, 4, 2, 64, 64, torch.bfloat16, 12)
    q, k, f, at = p["q"], p["k"], p["inv_freq"], p["positions"]
    call = api.rm_head_norm_rotary
    wide = torch.zeros((3, 1, 8, 64), dtype=torch.bfloat16, device="cuda")
    bad = [
        (ValueError, lambda: call(None, None, f, at)),
        (ValueError, lambda: call(q.float(), k, f, at)),
        (ValueError, lambda: call(q, k.half(), f, at)),
        (ValueError, lambda: call(q, k[:2], f, at)),
        (ValueError, lambda: call(q, k[:, :, :32], f, at)),
        (ValueError, lambda: call(q[0], k, f, at)),
        (ValueError, lambda: call(q, k, f.double(), at)),
        (ValueError, lambda: call(q, k, f, at.long())),
        (ValueError, lambda: call(q, k, f, at[:2])),
        (ValueError, lambda: call(q, k, f, at, q_weight=p["q_weight"][:5])),
        (ValueError, lambda: call(q, k, f, at, layout="both")),
        (ValueError, lambda: call(q.transpose(1, 2), None, f, at)),
        (ValueError, lambda: call(q, k, f, at, q_out=wide.expand(3, 4, 8, 64)[:, :, 0])),
        (RuntimeError, lambda: call(q, k, f)),
        (RuntimeError, lambda: call(q, k, torch.ones(33, device="cuda"), at)),
        (RuntimeError, lambda: call(q, k, f, at, eps=float("nan"))),
        (RuntimeError, lambda: call(q[:, :, :36].contiguous(), None, f[:4], at)),
    ]
    for i, (error, f_) in enumerate(bad):
        with pytest.raises(error):
            f_()
            print("accepted", i)
