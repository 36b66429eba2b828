"""A decode step through all operators together: in a graph, on another stream,
one token at a time against whole prompts, and as a trace for the predictor."""
import numpy as np
import pytest
import torch

from paper_2607_16784_amd import api, decode
from paper_2607_16784_amd import workloads as W

pytestmark = pytest.mark.gpu


def small(codes=torch.int8, dtype=torch.bfloat16, seed=1):
    return decode.DecodeModel(layers=2, width=256, heads=4, kv_heads=2, head_dim=64, hidden=512,
                              group=64, dtype=dtype, codes=codes, page_tokens=16, seed=seed)


def hidden(model, n, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, model.width), generator=g).to(model.dtype).cuda()


@pytest.mark.parametrize("codes", [torch.int8, torch.float8_e4m3fn], ids=["int8", "e4m3"])
def test_a_prompt_at_once_and_token_by_token(codes):
    # the same tokens in the cache; a page filled token by token is rescaled on
    # the way, which moves its codes by a step at most, so the last outputs agree
    # to a few steps of the cache: 1/127 of the largest value (int8) or 1/16
    model, n, tokens = small(codes, torch.float16), 3, 21
    x = hidden(model, n * tokens, 2).view(n, tokens, -1)
    whole = model.new_state(n, 64)
    y = model.step(x.reshape(n * tokens, -1), whole, tokens).view(n, tokens, -1)[:, -1]
    single = model.new_state(n, 64)
    for t in range(tokens):
        z = model.step(x[:, t].contiguous(), single)
    assert torch.equal(whole["lengths"], single["lengths"])
    assert int(whole["status"].item()) == 0 and int(single["status"].item()) == 0
    step = 1 / 127 if codes == torch.int8 else 1 / 16
    off = (y.double() - z.double()).norm() / y.double().norm()
    assert float(off) < 4 * step, float(off)
    assert torch.all(torch.isfinite(y))


def test_a_captured_step_replays_as_the_eager_one():
    model, n = small(), 5
    state, other = model.new_state(n, 64), model.new_state(n, 64)
    for s in (state, other):
        model.step(hidden(model, n * 9, 3), s, 9)
    x = hidden(model, n, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = model.step(x, state)               # counts its token in the graph too
    torch.cuda.current_stream().wait_stream(side)
    for t in range(4):
        new = hidden(model, n, 50 + t)
        x.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        want = model.step(new, other)
        assert torch.equal(y, want), t
        assert torch.equal(state["lengths"], other["lengths"])
        for a, b in zip(state["caches"], other["caches"]):
            for k in a:
                assert torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)), (t, k)


def test_on_another_stream():
    model, n = small(), 4
    state, other = model.new_state(n, 64), model.new_state(n, 64)
    x = hidden(model, n * 12, 5)
    want = model.step(x, other, 12)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    # work queued on the side stream before the step must be seen by it
    y = torch.zeros_like(x)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        y.copy_(x)
        got = model.step(y, state, 12)
    side.synchronize()
    assert torch.equal(got, want)


def test_a_recording_holds_the_launches_and_changes_nothing():
    model, n = small(), 2
    state, other = model.new_state(n, 64), model.new_state(n, 64)
    x = hidden(model, n, 6)
    want = model.step(x, other)
    with api.rm_trace() as t:
        got = model.step(x, state)
    assert torch.equal(got, want)
    assert len(t.launches) == 2 * 8 + 1
    for k in t.launches:
        assert k["grid"] > 0 and k["threads"] % 64 == 0 and 64 <= k["threads"] <= 1024
        assert 0 < k["regs"] <= 512 and 0 <= k["smem"] <= 160 * 1024
    with api.rm_trace() as t:
        model.step(x[:0], model.new_state(0, 64))
    assert t.launches == []
    with pytest.raises(RuntimeError, match="room for 3"):
        with api.rm_trace(3):
            model.step(x, state)


def test_the_predictor_takes_the_traces():
    models = []
    for seed, n in ((1, 2), (2, 7)):
        model = small(seed=seed)
        state = model.new_state(n, 64)
        model.step(hidden(model, n * 20, seed), state, 20)
        models.append((model, state))
    lib = decode.trace_library(models)
    assert lib["offsets"].tolist() == [0, 17, 34]
    assert np.all(lib["duration"] > 0) and np.all(lib["duration"] < 1e4)
    L = api.library_to_device(lib)
    st = api.new_status()
    occ = api.rm_occupancy(W.MI355X, L["grid"], L["threads"], L["regs"], L["smem"], status=st)
    out = api.rm_pair_slowdown_matrix(W.MI355X, L["offsets"], L["grid"], L["threads"], L["regs"],
                                      L["smem"], L["duration"], status=st)
    assert int(st.item()) == 0
    assert torch.all(occ["blocks_per_sm"] > 0)
    assert torch.all(out["slowdown"] >= 0) and torch.all(out["iso_time"] > 0)
    for _, state in models:
        assert int(state["status"].item()) == 0


def test_frequencies():
    f, s = decode.rotary_frequencies(8)
    assert s == 1.0 and torch.allclose(f, 10000.0 ** (-torch.arange(0, 8, 2) / 8))
    g, _ = decode.rotary_frequencies(8, scaling="linear", factor=4.0)
    assert torch.allclose(g, f / 4)
    g, _ = decode.rotary_frequencies(8, scaling="ntk", factor=4.0)
    assert torch.isclose(g[0], f[0]) and torch.isclose(g[-1], f[-1] / 4)
    g, s = decode.rotary_frequencies(64, scaling="parts", factor=4.0, trained=4096)
    f, _ = decode.rotary_frequencies(64)
    assert torch.isclose(g[0], f[0]) and torch.isclose(g[-1], f[-1] / 4) and s > 1
    with pytest.raises(ValueError):
        decode.rotary_frequencies(8, scaling="best")
