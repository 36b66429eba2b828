"""Sizes whose launches do not fit are refused by the host; these need no GPU."""
from test_decode_refusals import P, cache, lib, seqs  # noqa: F401


def test_attention_beyond_31_bits_of_workgroups(lib):  # noqa: F811
    s = seqs(n_seqs=65535, max_tokens=1 << 20, n_tokens=1 << 30)
    assert lib.rm_cache_attention(0, cache(), s, 4, P, 64, 64, 1.0, 0, P, P, 1 << 60, None,
                                  None) == 3
    assert lib.rm_cache_attention_workspace_bytes(cache(), s, 4) == 0
    # the bound on a sequence's tokens is that of the call where it is larger
    s = seqs(n_seqs=65535, max_tokens=1 << 20, n_tokens=1 << 10)
    assert lib.rm_cache_attention_workspace_bytes(cache(), s, 4) > 0


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
