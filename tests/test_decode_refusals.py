"""Host-side argument checks of the decode-layer entry points; these need no GPU.
Pointers that a check must not follow are small odd numbers."""
import ctypes

import pytest
import torch

from paper_2607_16784_amd import api

P = ctypes.c_void_p(256)


@pytest.fixture(scope="module")
def lib():
    return api.library()


def cache(**kw):
    c = dict(k=256, v=256, k_scale=256, v_scale=256, n_pages=4, kv_heads=2, page_tokens=16,
             head_dim=64, codes=0)
    c.update(kw)
    return api.Cache(*(c[n] for n, _ in api.Cache._fields_))


def seqs(**kw):
    s = dict(table=256, lengths=256, token_offsets=256, n_seqs=2, table_stride=3, n_tokens=2,
             max_tokens=1)
    s.update(kw)
    return api.Sequences(*(s[n] for n, _ in api.Sequences._fields_))


def test_w4_linear(lib):
    def call(type=0, rows=1, n=8, k=64, x=P, xs=64, codes=P, cs=32, group=32, scales=P, act=0,
             y=P, ys=8, ws=None, size=0):
        return lib.rm_w4_linear(type, rows, n, k, x, xs, codes, cs, group, scales, None, None,
                                act, y, ys, ws, size, None)
    assert call(rows=0) == 0
    for kw in (dict(type=2), dict(rows=-1), dict(n=0), dict(k=0), dict(xs=63), dict(cs=31),
               dict(group=0), dict(group=40), dict(act=2), dict(act=1, n=7, ys=7), dict(ys=7),
               dict(x=None), dict(codes=None), dict(scales=None), dict(y=None)):
        assert call(**kw) == 1, kw
    assert call(k=1 << 25, xs=1 << 25, cs=1 << 24) == 3
    assert call(n=(1 << 30) + 1, ys=1 << 31) == 3
    assert call(rows=1 << 23) == 3 and lib.rm_w4_linear_workspace_bytes(1 << 23, 8, 64, 0) == 0
    # sizes whose columns are split need a workspace
    big = dict(rows=64, n=512, k=8192, xs=8192, cs=4096, ys=512)
    need = lib.rm_w4_linear_workspace_bytes(64, 512, 8192, 0)
    assert need > 0 and need % 4 == 0
    assert lib.rm_w4_linear_workspace_bytes(1, 512, 8192, 0) == 0
    assert lib.rm_w4_linear_workspace_bytes(0, 512, 8192, 0) == 0
    for kw in (dict(), dict(ws=P, size=need - 1), dict(ws=ctypes.c_void_p(257), size=need)):
        assert call(**big, **kw) == 2, kw


BAD_CACHES = [(dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(n_pages=0), 1),
              (dict(kv_heads=0), 1), (dict(codes=2), 1), (dict(k=264), 1), (dict(v=257), 1),
              (dict(page_tokens=8), 3), (dict(page_tokens=48), 3), (dict(head_dim=96), 3),
              (dict(kv_heads=65536), 3)]
BAD_SEQS = [(dict(n_seqs=-1), 1), (dict(table_stride=-1), 1), (dict(n_tokens=-1), 1),
            (dict(max_tokens=-1), 1), (dict(lengths=None), 1), (dict(table=None), 1),
            (dict(token_offsets=None, n_tokens=3), 1), (dict(token_offsets=None, max_tokens=0), 1),
            (dict(n_seqs=65536), 3), (dict(table_stride=1 << 28), 3)]


def test_rotary_append(lib):
    def call(c=None, s=None, type=0, heads=4, q=P, k=P, v=P, inv=P, rot=64, layout=0, out=P):
        return lib.rm_rotary_append(type, c or cache(), s or seqs(), heads, q, 64, 64, k, 64, 64,
                                    v, 64, 64, None, inv, rot, layout, 1.0, out, None, None)
    assert call(s=seqs(n_tokens=0)) == 0
    for kw in (dict(type=-1), dict(heads=-1), dict(q=None), dict(k=None), dict(v=None),
               dict(inv=None), dict(rot=3), dict(rot=66), dict(rot=-2), dict(layout=2),
               dict(out=None)):
        assert call(**kw) == 1, kw
    assert call(heads=65536) == 3
    for kw, code in BAD_CACHES:
        assert call(c=cache(**kw)) == code, kw
    for kw, code in BAD_SEQS:
        assert call(s=seqs(**kw)) == code, kw


def test_cache_read(lib):
    def call(c=None, type=0, n=1, pages=P, k=P, v=P):
        return lib.rm_cache_read(type, c or cache(), n, pages, k, v, None, None)
    assert call(n=0) == 0
    for kw in (dict(type=2), dict(n=-1), dict(pages=None), dict(k=None), dict(v=None)):
        assert call(**kw) == 1, kw
    for kw, code in BAD_CACHES:
        assert call(c=cache(**kw)) == code, kw


def test_cache_attention(lib):
    def call(c=None, s=None, type=0, heads=4, q=P, scale=1.0, window=0, out=P, ws=P, size=1 << 40):
        return lib.rm_cache_attention(type, c or cache(), s or seqs(), heads, q, 64, 64, scale,
                                      window, out, ws, size, None, None)
    assert call(s=seqs(n_tokens=0)) == 0
    for kw in (dict(type=2), dict(heads=0), dict(heads=3), dict(q=None), dict(out=None),
               dict(scale=float("inf")), dict(window=-1)):
        assert call(**kw) == 1, kw
    for kw in (dict(ws=None), dict(size=0), dict(ws=ctypes.c_void_p(264))):
        assert call(**kw) == 2, kw
    for kw, code in BAD_CACHES:
        assert call(c=cache(**kw)) == code, kw
    for kw, code in BAD_SEQS:
        assert call(s=seqs(**kw)) == code, kw


def test_rows_of_a_sequence_beyond_31_bits(lib):
    s = seqs(max_tokens=1 << 30)
    assert lib.rm_cache_attention(0, cache(), s, 4, P, 64, 64, 1.0, 0, P, P, 1 << 60, None,
                                  None) == 3
    assert lib.rm_cache_attention_workspace_bytes(cache(), s, 4) == 0


def test_cache_attention_workspace(lib):
    f = lib.rm_cache_attention_workspace_bytes
    assert f(cache(), seqs(), 4) > 0
    assert f(cache(), seqs(), 3) == 0 and f(cache(), seqs(), 0) == 0
    assert f(cache(head_dim=80), seqs(), 4) == 0 and f(cache(), seqs(lengths=None), 4) == 0


def test_norm_residual(lib):
    def call(type=0, kind=0, rows=1, width=8, x=P, xs=8, y=P, ys=8, gate=None, gs=0, gw=8,
             post=None, alpha=1.0, eps=0.0, x_out=P, n_out=P):
        return lib.rm_norm_residual(type, kind, rows, width, x, xs, y, ys, gate, gs, gw, post,
                                    None, None, alpha, eps, x_out, n_out, None)
    assert call(rows=0) == 0
    for kw in (dict(type=2), dict(kind=2), dict(rows=-1), dict(width=0), dict(x=None),
               dict(xs=7), dict(ys=7), dict(y=None, gate=P), dict(y=None, post=P),
               dict(gate=P, gw=4), dict(gate=P, gs=7), dict(alpha=float("nan")),
               dict(eps=float("inf")), dict(x_out=None, n_out=None)):
        assert call(**kw) == 1, kw
    assert call(width=32769, xs=32769, ys=32769) == 3


def test_trace(lib):
    n = ctypes.c_int32()
    assert lib.rm_trace_end(ctypes.byref(n)) == 1
    records = (api.Launch * 2)()
    assert lib.rm_trace_begin(None, 2) == 1 and lib.rm_trace_begin(records, -1) == 1
    assert lib.rm_trace_begin(records, 2) == 0
    assert lib.rm_trace_begin(records, 2) == 1
    assert lib.rm_trace_end(None) == 1
    assert lib.rm_trace_end(ctypes.byref(n)) == 0 and n.value == 0
    with api.rm_trace(4) as t:
        pass
    assert t.launches == []


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu():
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        api.rm_norm_residual(x)
    with pytest.raises(ValueError):
        api.rm_w4_linear(x, torch.zeros((4, 32), dtype=torch.uint8), x, 32)
    c = api.new_cache(2, 1, 16, 64, device="cpu")
    t = torch.zeros((2, 1), dtype=torch.int32)
    k = torch.zeros((2, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        api.rm_cache_attention(k, c, t, t[:, 0])
    with pytest.raises(ValueError):
        api.rm_rotary_append(k, k, k, torch.zeros(32), c, t, t[:, 0])
    with pytest.raises(ValueError):
        api.rm_cache_read(c, t[:, 0])
