"""Calls whose workgroups have 2^32 threads or more: a dispatch holds fewer, so the
norms stride over the rows and the cache calls come in several launches."""
import pytest
import torch

from decode_common import make_cache
from paper_2607_16784_amd import api

pytestmark = pytest.mark.gpu


def fit(launches, at_least):
    threads = [k["grid"] * k["threads"] for k in launches]
    assert max(threads) < 1 << 32 and sum(threads) >= 1 << 32 and len(launches) >= at_least


def test_norm_of_many_rows():
    rows, width = (1 << 26) + 3, 8
    x = torch.empty((rows, width), dtype=torch.bfloat16, device="cuda")
    step = 1 << 22
    for at in range(0, rows, step):
        part = x[at:at + step]
        part.copy_(torch.randn(part.shape, device="cuda"))
    _, n = api.rm_norm_residual(x)
    for at in range(0, rows, step):
        part = x[at:at + step].float()
        want = part / torch.sqrt(part.square().mean(dim=1, keepdim=True) + 1e-6)
        err = (n[at:at + step].float() - want).abs()
        # half a unit of bf16 and a few roundings of fp32
        assert torch.all(err <= (2.0 ** -8 + 2.0 ** -20) * want.abs())


def one_long(sequences, length, kv, dim, seed):
    """Sequences of one new token, the last of them of `length` new ones."""
    lengths = [20] * (sequences - 1) + [length]
    cache, table, lens, _ = make_cache(lengths, kv, 16, dim, torch.int8, seed)
    offsets = torch.arange(sequences + 1, dtype=torch.int32, device="cuda")
    offsets[-1] = sequences - 1 + length
    return cache, table, lens, offsets


def test_attention_over_a_long_prompt_among_many_sequences():
    n, length, kv, heads = 520, 32768, 8, 32
    cache, table, lens, offsets = one_long(n, length, kv, 64, 101)
    tokens = n - 1 + length
    q = torch.randn((tokens, heads, 64), device="cuda").bfloat16()
    st = api.new_status()
    with api.rm_trace() as t:
        got = api.rm_cache_attention(q, cache, table, lens, token_offsets=offsets,
                                     max_tokens=length, window=64, status=st)
    assert int(st.item()) == 0
    fit(t.launches, 2)
    # the sequences of one token, and the prompt, by calls of their own
    few = api.rm_cache_attention(q[:n - 1].contiguous(), cache, table[:n - 1].contiguous(),
                                 lens[:n - 1].contiguous(), window=64)
    alone = api.rm_cache_attention(
        q[n - 1:].contiguous(), cache, table[n - 1:].contiguous(), lens[n - 1:].contiguous(),
        token_offsets=torch.tensor([0, length], dtype=torch.int32, device="cuda"),
        max_tokens=length, window=64)
    for a, b in ((got[:n - 1], few), (got[n - 1:], alone)):
        a, b = a.float(), b.float()
        # each within a unit of bf16 and 2^-11 of the mean of |value|, at most 3 * 127 / 127
        assert torch.all((a - b).abs() <= 2.0 ** -7 * b.abs() + 4 * 2.0 ** -10)


def test_append_of_a_long_prompt_among_many_sequences():
    n, length, kv = 2200, 32768, 8
    cache, table, lens, offsets = one_long(n, length, kv, 64, 102)
    other = {name: c.clone() for name, c in cache.items()}
    k, v = (torch.randn((n - 1 + length, kv, 64), device="cuda").bfloat16() for _ in range(2))
    inv = torch.tensor([10000.0 ** (-i / 32) for i in range(32)], device="cuda")
    st = api.new_status()
    with api.rm_trace() as t:
        q = api.rm_rotary_append(k, k, v, inv, cache, table, lens, token_offsets=offsets,
                                 max_tokens=length, status=st)
    assert int(st.item()) == 0
    fit(t.launches, 2)
    few = api.rm_rotary_append(k[:n - 1], k[:n - 1], v[:n - 1], inv, other,
                               table[:n - 1].contiguous(), lens[:n - 1].contiguous())
    alone = api.rm_rotary_append(
        k[n - 1:], k[n - 1:], v[n - 1:], inv, other, table[n - 1:].contiguous(),
        lens[n - 1:].contiguous(), max_tokens=length,
        token_offsets=torch.tensor([0, length], dtype=torch.int32, device="cuda"))
    assert torch.equal(q, torch.cat([few, alone]))
    for name in cache:
        assert torch.equal(cache[name].view(torch.uint8), other[name].view(torch.uint8)), name
