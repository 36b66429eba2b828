"""Sines and cosines of rm_rotary_append, read through pairs (0, 1) and (1, 0).

Tolerance: half a unit of f16 (2^-11) and 2^-20 of the value: sine and cosine
are fp32 numbers with a relative error of a few of their last places, also near
their zeros, where the angle itself (rounded to fp32 once the whole turns are
off) sets what is left; results lie in the normal range of f16."""
import math

import pytest
import torch

from paper_2607_16784_amd import api

pytestmark = pytest.mark.gpu


def turned(freq, positions, scale):
    """(cosine, sine) * scale of position * freq for each pair, fp64 [tokens, 32]."""
    n = len(positions)
    q = torch.zeros((n, 1, 64), dtype=torch.float16, device="cuda")
    q[..., :32] = 1.0
    cache = api.new_cache(1, 1, 128, 64)
    k = torch.zeros((n, 1, 64), dtype=torch.float16, device="cuda")
    inv = torch.tensor(freq, dtype=torch.float32, device="cuda")
    out = api.rm_rotary_append(
        q, k, k, inv, cache, torch.zeros((1, 1), dtype=torch.int32, device="cuda"),
        torch.tensor([n], dtype=torch.int32, device="cuda"), max_tokens=n, rot_scale=scale,
        token_offsets=torch.tensor([0, n], dtype=torch.int32, device="cuda"),
        positions=torch.tensor(positions, dtype=torch.int32, device="cuda"))
    out = out[:, 0].double().cpu()
    return out[:, :32], out[:, 32:], inv.double().cpu()


@pytest.mark.parametrize("scale", [4096.0, 1024.0])
def test_small_angles(scale):
    # angles from 3e-4 to 0.5, both signs
    freq = [3e-4 * 1.27 ** i for i in range(32)]
    positions = [1, -1]
    cs, sn, inv = turned(freq, positions, scale)
    for t, p in enumerate(positions):
        for i in range(32):
            a = float(inv[i]) * p
            want = math.sin(a) * scale
            assert abs(float(sn[t, i]) - want) <= (2.0 ** -11 + 2.0 ** -20) * abs(want), (p, i)
            want = math.cos(a) * scale
            assert abs(float(cs[t, i]) - want) <= (2.0 ** -11 + 2.0 ** -20) * abs(want), (p, i)


def test_all_around_the_turn():
    freq = [(i + 0.37) * 2 * math.pi / 32 for i in range(32)]
    positions = list(range(1, 120, 7))
    cs, sn, inv = turned(freq, positions, 2048.0)
    for t, p in enumerate(positions):
        for i in range(32):
            a = float(inv[i]) * p
            for got, want in ((sn, math.sin(a)), (cs, math.cos(a))):
                # near a zero the turn, rounded to fp32, is off by 2^-25 of half a turn
                tol = (2.0 ** -11 + 2.0 ** -20) * abs(want) + 2.0 ** -22
                assert abs(float(got[t, i]) / 2048.0 - want) <= tol, (p, i)
