"""Sizes whose launches do not fit are refused by the host; these need no GPU."""
from test_decode_refusals import P, cache, lib, seqs  # noqa: F401


def test_attention_beyond_31_bits_of_workgroups(lib):  # noqa: F811
    s = seqs(n_seqs=65535, max_tokens=1 << 20, n_tokens=1 << 30)
    assert lib.rm_cache_attention(0, cache(), s, 4, P, 64, 64, 1.0, 0, P, P, 1 << 60, None,
                                  None) == 3
    assert lib.rm_cache_attention_workspace_bytes(cache(), s, 4) == 0


def test_a_workspace_serves_calls_of_fewer_tokens(lib):  # noqa: F811
    for n, most, stride in ((2, 1, 3), (9, 700, 4000), (3, 64, 100000), (64, 512, 300)):
        need = {lib.rm_cache_attention_workspace_bytes(
            cache(kv_heads=4), seqs(n_seqs=n, max_tokens=most, table_stride=stride,
                                    n_tokens=tokens), 16)
            for tokens in (1, 7, n, most, n * most)}
        assert len(need) == 1 and min(need) > 0


def test_append_beyond_31_bits_of_workgroups(lib):  # noqa: F811
    s = seqs(n_seqs=65535, max_tokens=1 << 30, n_tokens=1 << 30)
    assert lib.rm_rotary_append(0, cache(), s, 4, P, 64, 64, P, 64, 64, P, 64, 64, None, P, 64, 0,
                                1.0, P, None, None) == 3


def test_outputs_of_a_projection(lib):  # noqa: F811
    # 64 outputs a workgroup of 512 threads: fewer than 2^23 of them
    n = 536870849
    assert lib.rm_w4_linear(0, 1, n, 64, P, 64, P, 32, 32, P, None, None, 0, P, n, None, 0,
                            None) == 3
    assert lib.rm_w4_linear_workspace_bytes(64, n, 8192, 0) == 0
