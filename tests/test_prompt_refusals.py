"""Host-side argument checks of the prompt's operators and the 8-bit floating
projection; these need no GPU."""
import ctypes

import pytest

from paper_2607_16784_amd import api

P = ctypes.c_void_p(256)


@pytest.fixture(scope="module")
def lib():
    return api.library()


def test_head_norm_rotary(lib):
    def call(type=0, tokens=3, heads=4, kv=2, dim=64, q=P, k=P, at=P, inv=P, rot=64, layout=0,
             scale=1.0, eps=1e-6, qo=P, ko=P):
        return lib.rm_head_norm_rotary(type, tokens, heads, kv, dim, q, 256, 64, k, 128, 64, None,
                                       None, at, inv, rot, layout, scale, eps, qo, 256, 64, ko,
                                       128, 64, None)
    assert call(tokens=0) == 0 and call(heads=0, kv=0) == 0
    for kw in (dict(type=2), dict(tokens=-1), dict(heads=-1), dict(kv=-1), dict(dim=0),
               dict(rot=3), dict(rot=66), dict(rot=-2), dict(layout=2), dict(scale=float("nan")),
               dict(eps=float("inf")), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None),
               dict(at=None), dict(inv=None)):
        assert call(**kw) == 1, kw
    for kw in (dict(dim=68), dict(dim=520), dict(heads=65536), dict(kv=65536)):
        assert call(**kw) == 3, kw


def test_prompt_attention(lib):
    def call(type=0, tokens=3, heads=4, kv=2, dim=64, q=P, k=P, v=P, off=P, n=1, most=3,
             scale=0.1, window=0, out=P):
        return lib.rm_prompt_attention(type, tokens, heads, kv, dim, q, 256, 64, k, 128, 64, v,
                                       128, 64, off, n, most, scale, window, out, None, None)
    assert call(tokens=0) == 0
    for kw in (dict(type=-1), dict(tokens=-1), dict(n=-1), dict(most=-1), dict(kv=0),
               dict(heads=0), dict(heads=3), dict(window=-1), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(q=None), dict(k=None), dict(v=None), dict(off=None),
               dict(out=None)):
        assert call(**kw) == 1, kw
    for kw in (dict(dim=32), dict(dim=96), dict(n=65536), dict(heads=65536),
               dict(most=0x7fffff00), dict(tokens=0x7fffffff, heads=65534)):
        assert call(**kw) == 3, kw


def test_f8(lib):
    def quantise(type=0, rows=2, k=200, x=P, xs=200, block=1, codes=P, cs=200, scales=P):
        return lib.rm_f8_quantize(type, rows, k, x, xs, block, codes, cs, scales, None)
    assert quantise(rows=0) == 0
    for kw in (dict(type=2), dict(rows=-1), dict(k=0), dict(xs=199), dict(cs=199), dict(block=2),
               dict(x=None), dict(codes=None), dict(scales=None)):
        assert quantise(**kw) == 1, kw
    assert quantise(k=1 << 22, xs=1 << 22, cs=1 << 22) == 3

    def call(type=0, rows=1, n=8, k=64, x=P, xs=64, codes=P, cs=64, scales=P, act=0, y=P, ys=8,
             ws=None, size=0):
        return lib.rm_f8_linear(type, rows, n, k, x, xs, None, codes, cs, scales, None, act, y, ys,
                                ws, size, None)
    assert call(rows=0) == 0
    for kw in (dict(type=2), dict(rows=-1), dict(n=0), dict(k=0), dict(xs=63), dict(cs=63),
               dict(ys=7), dict(act=2), dict(act=1, n=7), dict(x=None), dict(codes=None),
               dict(scales=None), dict(y=None)):
        assert call(**kw) == 1, kw
    assert call(k=1 << 22, xs=1 << 22, cs=1 << 22) == 3
    assert call(n=1 << 30, ys=1 << 30) == 3
    assert call(rows=1 << 23) == 3
    for kw in (dict(rows=0), dict(n=0), dict(k=0), dict(rows=1 << 23), dict(n=1 << 30),
               dict(k=1 << 22)):
        s = dict(dict(rows=500, n=8, k=64), **kw)
        assert lib.rm_f8_linear_workspace_bytes(s["rows"], s["n"], s["k"], 0) == 0
    need = lib.rm_f8_linear_workspace_bytes(500, 8, 64, 0)
    assert need >= 500 * (128 + 4)
    assert lib.rm_f8_linear_workspace_bytes(api.F8_FEW_ROWS, 1 << 20, 1 << 20, 0) == 0
    assert lib.rm_f8_linear_workspace_bytes(api.F8_FEW_ROWS + 1, 8, 64, 0) > 0
    # few tiles: the columns' parts are in it
    assert lib.rm_f8_linear_workspace_bytes(64, 128, 12800, 0) >= 64 * 12800 + 16 * 64 * 128 * 4
    for kw in (dict(), dict(ws=P, size=need - 1), dict(ws=ctypes.c_void_p(257), size=need)):
        assert call(rows=500, **kw) == 2, kw
