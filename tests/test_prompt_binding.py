"""What the binding of the prompt's operators hands to the library, with the
stand-ins of test_decode_binding: which GPU a call goes to, and what it refuses.
These need no GPU."""
import pytest
import torch

from paper_2607_16784_amd import api
from test_decode_binding import BF16, F32, I32, Tensor, calls  # noqa: F401

E4M3 = torch.float8_e4m3fn


def headnorm():
    return api.rm_head_norm_rotary, dict(
        q=Tensor((3, 4, 64), BF16), k=Tensor((3, 2, 64), BF16), inv_freq=Tensor((32,), F32),
        positions=Tensor((3,), I32), q_weight=Tensor((64,), BF16), k_weight=Tensor((64,), BF16),
        q_out=Tensor((3, 4, 64), BF16), k_out=Tensor((3, 2, 64), BF16))


def attention():
    return api.rm_prompt_attention, dict(
        q=Tensor((3, 4, 64), BF16), k=Tensor((3, 2, 64), BF16), v=Tensor((3, 2, 64), BF16),
        token_offsets=Tensor((3,), I32), max_tokens=2, out=Tensor((3, 4, 64), BF16),
        status=Tensor((1,), I32))


def linear():
    return api.rm_f8_linear, dict(
        x=Tensor((3, 200), E4M3), x_scales=Tensor((3, 2), F32), codes=Tensor((300, 200), E4M3),
        scales=Tensor((3, 2), F32), bias=Tensor((300,), BF16), out=Tensor((3, 300), BF16),
        workspace=Tensor((512,), torch.uint8))


CALLS = [headnorm, attention, linear]


@pytest.mark.parametrize("make", CALLS)
def test_a_call_goes_to_the_gpu_of_its_tensors(calls, make):  # noqa: F811
    f, kw = make()
    f(**kw)
    (name, gpu, args), = calls
    assert name == f.__name__ and gpu == 1 and args[-1] == 1001
    with torch.cuda.device(1):
        f(**kw)
    assert calls[1][1] == 1 and calls[1][2][-1] == 1001


@pytest.mark.parametrize("make", CALLS)
@pytest.mark.parametrize("gpu", [0, -1])
def test_all_tensors_of_a_call_are_on_one_gpu(calls, make, gpu):  # noqa: F811
    f, kw = make()
    for n in [n for n, t in kw.items() if isinstance(t, Tensor)]:
        _, bad = make()
        bad[n].gpu = gpu
        before = len(calls)
        with pytest.raises(ValueError):
            f(**bad)
        assert len(calls) == before, n


def test_numbers_beyond_31_bits(calls):  # noqa: F811
    big = 1 << 31
    cases = [
        (headnorm, dict(q=Tensor((big, 4, 64), BF16), q_out=Tensor((big, 4, 64), BF16),
                        k=Tensor((big, 2, 64), BF16), k_out=Tensor((big, 2, 64), BF16))),
        (headnorm, dict(inv_freq=Tensor((1 << 30,), F32))),
        (attention, dict(max_tokens=big)), (attention, dict(window=big)),
        (attention, dict(q=Tensor((big, 4, 64), BF16), k=Tensor((big, 2, 64), BF16),
                         v=Tensor((big, 2, 64), BF16), out=Tensor((big, 4, 64), BF16))),
        (linear, dict(x=Tensor((big, 200), E4M3))), (linear, dict(codes=Tensor((big, 200), E4M3))),
    ]
    for make, kw in cases:
        f, args = make()
        args.update(kw)
        with pytest.raises(ValueError, match="beyond 31 bits"):
            f(**args)
    assert calls == []


def test_outputs_whose_rows_overlap(calls):  # noqa: F811
    for strides in ((100, 64, 1), (256, 32, 1), (0, 64, 1)):
        f, kw = headnorm()
        kw["q_out"] = Tensor((3, 4, 64), BF16, strides=strides)
        with pytest.raises(ValueError, match="overlap"):
            f(**kw)
    for strides in ((256, 64, 1), (999, 80, 1), (64, 192, 1)):
        f, kw = headnorm()
        kw["q_out"] = Tensor((3, 4, 64), BF16, strides=strides)
        f(**kw)
    f, kw = linear()
    kw["out"] = Tensor((3, 300), BF16, strides=(299, 1))
    with pytest.raises(ValueError, match="overlap"):
        f(**kw)
