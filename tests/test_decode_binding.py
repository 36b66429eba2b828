"""What the binding of the decode-layer operators hands to the library, seen with
stand-ins for tensors on two GPUs and for the library: which GPU a call goes to,
and what it refuses.  These need no GPU."""
import contextlib

import pytest
import torch

from paper_2607_16784_amd import api

BF16, F32, I32, U8, I8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.int8


class Tensor:
    def __init__(self, shape, dtype, gpu=1, strides=None):
        self.shape, self.dtype, self.gpu = torch.Size(shape), dtype, gpu
        dense = [1] * len(shape)
        for i in range(len(shape) - 2, -1, -1):
            dense[i] = dense[i + 1] * shape[i + 1]
        self.strides, self.dense = tuple(strides or dense), tuple(dense)

    is_cuda = property(lambda t: t.gpu >= 0)
    device = property(lambda t: f"cuda:{t.gpu}" if t.gpu >= 0 else "cpu")
    get_device = lambda t: t.gpu                                     # noqa: E731
    dim = lambda t: len(t.shape)                                     # noqa: E731
    stride = lambda t: t.strides                                     # noqa: E731
    is_contiguous = lambda t: t.strides == t.dense                   # noqa: E731
    data_ptr = lambda t: 4096                                        # noqa: E731
    numel = lambda t: t.shape.numel()                                # noqa: E731
    element_size = lambda t: torch.empty(0, dtype=t.dtype).element_size()   # noqa: E731


@pytest.fixture
def calls(monkeypatch):
    """(entry point, current GPU, its arguments) of every call."""
    made, current = [], [0]

    class Library:
        def __getattr__(self, name):
            def call(*args):
                if name.endswith("_bytes"):
                    return 256
                made.append((name, current[0], args))
                return 0
            return call

    @contextlib.contextmanager
    def device(gpu):
        before, current[0] = current[0], gpu
        yield
        current[0] = before

    monkeypatch.setattr(api, "_lib", Library())
    monkeypatch.setattr(api, "_raw_stream", lambda gpu: 1000 + gpu)
    monkeypatch.setattr(api, "_current_gpu", lambda: current[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    return made


def cache():
    return {"k": Tensor((4, 2, 16, 64), I8), "v": Tensor((4, 2, 64, 16), I8),
            "k_scale": Tensor((4, 2), F32), "v_scale": Tensor((4, 2), F32)}


def linear():
    return api.rm_w4_linear, dict(
        x=Tensor((3, 64), BF16), codes=Tensor((8, 32), U8), scales=Tensor((8, 2), BF16), group=32,
        zeros=Tensor((8, 2), U8), bias=Tensor((8,), BF16), out=Tensor((3, 8), BF16),
        workspace=Tensor((512,), U8))


def append():
    return api.rm_rotary_append, dict(
        q=Tensor((3, 4, 64), BF16), k=Tensor((3, 2, 64), BF16), v=Tensor((3, 2, 64), BF16),
        inv_freq=Tensor((32,), F32), cache=cache(), table=Tensor((2, 2), I32),
        lengths=Tensor((2,), I32), token_offsets=Tensor((3,), I32), max_tokens=2,
        positions=Tensor((3,), I32), q_out=Tensor((3, 4, 64), BF16), status=Tensor((1,), I32))


def attention():
    return api.rm_cache_attention, dict(
        q=Tensor((3, 4, 64), BF16), cache=cache(), table=Tensor((2, 2), I32),
        lengths=Tensor((2,), I32), token_offsets=Tensor((3,), I32), max_tokens=2,
        workspace=Tensor((512,), U8), out=Tensor((3, 4, 64), BF16), status=Tensor((1,), I32))


def norm():
    return api.rm_norm_residual, dict(
        x=Tensor((3, 64), BF16), y=Tensor((3, 64), BF16), gate=Tensor((3, 1), BF16),
        post_weight=Tensor((64,), BF16), pre_weight=Tensor((64,), BF16),
        pre_bias=Tensor((64,), BF16), x_out=Tensor((3, 64), BF16), n_out=Tensor((3, 64), BF16))


CALLS = [linear, append, attention, norm]


@pytest.mark.parametrize("make", CALLS)
def test_a_call_goes_to_the_gpu_of_its_tensors(calls, make):
    f, kw = make()
    f(**kw)
    (name, gpu, args), = calls
    assert name == f.__name__ and gpu == 1 and args[-1] == 1001
    with torch.cuda.device(1):
        f(**kw)
    assert calls[1][1] == 1 and calls[1][2][-1] == 1001


@pytest.mark.parametrize("make", CALLS)
@pytest.mark.parametrize("gpu", [0, -1])
def test_all_tensors_of_a_call_are_on_one_gpu(calls, make, gpu):
    f, kw = make()
    names = [n for n, t in kw.items() if isinstance(t, Tensor) and n != "workspace"]
    names += [("cache", n) for n in kw.get("cache", {})]
    assert len(names) > 5
    for n in names:
        _, bad = make()
        if isinstance(n, tuple):
            bad["cache"][n[1]].gpu = gpu
        else:
            bad[n].gpu = gpu
        with pytest.raises(ValueError):
            f(**bad)
    assert calls == []
    _, bad = make()
    if "gate" in bad:
        bad["gate"] = Tensor((64,), BF16, gpu)
        with pytest.raises(ValueError):
            f(**bad)


def test_cache_read_goes_to_the_gpu_of_its_tensors(calls, monkeypatch):
    pages = Tensor((2,), I32)
    both = type("Both", (), {"unbind": lambda t: (Tensor((2, 16, 2, 64), BF16),) * 2})()
    monkeypatch.setattr(api.torch, "empty", lambda *a, **kw: both)
    api.rm_cache_read(cache(), pages)
    assert calls[0][1] == 1 and calls[0][2][-1] == 1001
    for n in cache():
        bad = cache()
        bad[n].gpu = 0
        with pytest.raises(ValueError):
            api.rm_cache_read(bad, pages)
    for gpu in (0, -1):
        with pytest.raises(ValueError):
            api.rm_cache_read(cache(), Tensor((2,), I32, gpu))
    every = cache()
    for t in every.values():
        t.gpu = -1
    with pytest.raises(ValueError):
        api.rm_cache_read(every, Tensor((2,), I32, -1))
    assert len(calls) == 1


@pytest.mark.parametrize("make", [linear, attention])
@pytest.mark.parametrize("workspace", [Tensor((512,), U8, gpu=-1), Tensor((512,), U8, gpu=0),
                                       Tensor((512,), U8, strides=(2,)),
                                       Tensor((8, 64), U8, strides=(128, 1))])
def test_a_workspace_that_no_kernel_may_write(calls, make, workspace):
    f, kw = make()
    with pytest.raises(ValueError, match="workspace"):
        f(**dict(kw, workspace=workspace))
    assert calls == []


@pytest.mark.parametrize("make", [linear, attention])
def test_a_workspace_counts_in_bytes(calls, make):
    f, kw = make()
    f(**dict(kw, workspace=Tensor((256,), F32)))
    f(**dict(kw, workspace=Tensor((8, 128), torch.float64)))
    # the size stands behind the workspace's address
    sizes = [args[-2] if f.__name__ == "rm_w4_linear" else args[-3] for _, _, args in calls]
    assert sizes == [1024, 8192]


BEYOND = [1 << 31, (1 << 32) + 32, -(1 << 32) + 32, -(1 << 31) - 1]


@pytest.mark.parametrize("value", BEYOND)
def test_numbers_beyond_32_bits_are_refused(calls, value):
    # the C entry points take int32: 2^32 + 32 would arrive as 32
    f, kw = linear()
    with pytest.raises(ValueError):
        f(**dict(kw, group=value, scales=Tensor((8, 1), BF16), zeros=Tensor((8, 1), U8)))
    f, kw = attention()
    for name in ("window", "max_tokens"):
        with pytest.raises(ValueError, match=name):
            f(**dict(kw, **{name: value}))
    f, kw = append()
    with pytest.raises(ValueError, match="max_tokens"):
        f(**dict(kw, max_tokens=value))
    assert calls == []


def test_sizes_beyond_32_bits_are_refused(calls):
    many = (1 << 32) + 3
    f, kw = linear()
    with pytest.raises(ValueError, match="sizes"):
        f(**dict(kw, x=Tensor((many, 64), BF16), out=Tensor((many, 8), BF16)))
    f, kw = norm()
    wide = {n: Tensor((many, 64), BF16) for n in ("x", "y", "x_out", "n_out")}
    with pytest.raises(ValueError, match="sizes"):
        f(**dict(kw, gate=None, **wide))
    f, kw = attention()
    with pytest.raises(ValueError, match="sizes"):
        f(**dict(kw, table=Tensor((2, many), I32)))
    with pytest.raises(ValueError, match="sizes"):
        f(**dict(kw, q=Tensor((many, 4, 64), BF16), out=Tensor((many, 4, 64), BF16)))
    f, kw = append()
    tall = {n: Tensor((many, 4, 64), BF16) for n in ("q", "q_out")}
    tall |= {n: Tensor((many, 2, 64), BF16) for n in ("k", "v")}
    with pytest.raises(ValueError, match="sizes"):
        f(**dict(kw, positions=None, **tall))
    with pytest.raises(ValueError, match="sizes"):
        api.rm_cache_read(cache(), Tensor((many,), I32))
    assert calls == []


def test_the_largest_numbers_pass(calls):
    f, kw = attention()
    f(**dict(kw, window=(1 << 31) - 1, max_tokens=(1 << 31) - 1))
    f(**dict(kw, window=-1))            # the library's to refuse
    f, kw = linear()
    f(**dict(kw, group=(1 << 31) - 32, scales=Tensor((8, 1), BF16), zeros=Tensor((8, 1), U8)))
    assert len(calls) == 3


def test_a_recording_with_times_is_refused_without_room_for_them():
    import ctypes
    lib, n = api.library(), ctypes.c_int32()
    records, times = (api.Launch * 2)(), (ctypes.c_float * 2)()
    for args in ((None, times, 2), (records, None, 2), (records, times, -1)):
        assert lib.rm_trace_begin_timed(*args) == 1
    assert lib.rm_trace_begin_timed(records, times, 2) == 0
    assert lib.rm_trace_begin_timed(records, times, 2) == 1 and lib.rm_trace_begin(records, 2) == 1
    assert lib.rm_trace_end(ctypes.byref(n)) == 0 and n.value == 0
    assert lib.rm_trace_begin_timed(None, None, 0) == 0
    assert lib.rm_trace_end(ctypes.byref(n)) == 0
