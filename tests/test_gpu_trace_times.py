"""Times of a recording and of a traced step: what each launch takes, where the
step has it."""
import pytest
import torch

from paper_2607_16784_amd import api, decode

pytestmark = pytest.mark.gpu


def step_time(model, state, n):
    """Microseconds of a captured step (the least of a few replays)."""
    x = torch.randn((n, model.width), device="cuda").bfloat16()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for _, run in model.calls(x, state):
            run()
    torch.cuda.current_stream().wait_stream(side)
    took = []
    for _ in range(6):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        graph.replay()
        end.record()
        end.synchronize()
        took.append(begin.elapsed_time(end) * 1e3)
    return min(took)


def test_launches_of_one_call_have_times_of_their_own():
    # the projection down reads 117 MB of codes, its join 17 MB of sums, with the
    # same number of threads
    model = decode.DecodeModel(layers=1, width=8192, heads=8, kv_heads=2, head_dim=64,
                               hidden=28672)
    state = model.new_state(64, 64)
    down = [k for k in decode.trace(model, state) if k["name"] == "down"]
    assert len(down) == 2
    assert down[0]["grid"] * down[0]["threads"] == down[1]["grid"] * down[1]["threads"]
    assert down[0]["duration"] > 3 * down[1]["duration"] > 0
    # the codes cannot arrive faster than 8 TB/s
    assert down[0]["duration"] > 28672 * 8192 / 2 / 8e6


def test_a_step_is_the_sum_of_its_launches():
    # 350 MB of weights: more than the last level of cache
    model = decode.DecodeModel(layers=4, width=4096, heads=32, kv_heads=8, head_dim=128,
                               hidden=14336)
    state = model.new_state(1, 128)
    model.step(torch.randn((100, 4096), device="cuda").bfloat16(), state, 100)
    kernels = decode.trace(model, state)
    assert len(kernels) == 33
    total, whole = sum(k["duration"] for k in kernels), step_time(model, state, 1)
    # a captured step has gaps between its launches beside
    assert 0.8 * whole < total < 1.1 * whole, (total, whole)


def test_a_recording_with_times():
    x = torch.randn((4096, 4096), device="cuda").bfloat16()
    api.rm_norm_residual(x)
    with api.rm_trace() as plain:
        want = api.rm_norm_residual(x)[1]
    with api.rm_trace(3, timed=True) as t:
        got = [api.rm_norm_residual(x)[1] for _ in range(3)]
    assert all(torch.equal(g, want) for g in got)
    for k in t.launches:
        # 67 MB to and from memory
        assert 67.1e6 / 8e6 < k.pop("duration") < 1e3
    assert t.launches == plain.launches * 3 and "duration" not in plain.launches[0]
    with pytest.raises(RuntimeError, match="room for 1"):
        with api.rm_trace(1, timed=True):
            api.rm_norm_residual(x)
            api.rm_norm_residual(x)
    with api.rm_trace(timed=True) as t:
        pass
    assert t.launches == []


def test_times_are_refused_in_a_capture():
    x = torch.randn((4, 64), device="cuda").bfloat16()
    out = torch.full_like(x, 3.0)
    api.rm_norm_residual(x, n_out=out)
    want = out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with api.rm_trace(timed=True) as t:
            with pytest.raises(RuntimeError):
                api.rm_norm_residual(x, n_out=out)
        api.rm_norm_residual(x, n_out=out)
    assert t.launches == []
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
