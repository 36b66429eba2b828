"""The prompt's operators together, as a served model runs them: prompts of
different lengths against the same tokens one at a time, decode steps behind
them, in a graph, and as traces for the predictor."""
import numpy as np
import pytest
import torch

from paper_2607_16784_amd import api, decode
from paper_2607_16784_amd import workloads as W

pytestmark = pytest.mark.gpu
FORMS = [("w4", False), ("w4", True), ("f8", False), ("f8", True)]


def small(weights, head_norm, dtype=torch.float16, seed=1):
    return decode.DecodeModel(layers=2, width=256, heads=4, kv_heads=2, head_dim=64, hidden=320,
                              group=64, dtype=dtype, page_tokens=16, seed=seed, weights=weights,
                              head_norm=head_norm)


def hidden(model, n, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((n, model.width), generator=g).to(model.dtype).cuda()


@pytest.mark.parametrize("weights,head_norm", FORMS)
def test_a_prompt_at_once_and_token_by_token(weights, head_norm):
    # A prompt attends to its own keys and values, a step to those of the cache, off
    # by half a code of 1/127 of a page's largest.  In 8-bit floating weights a
    # changed input moves codes of the activations, 2^-4 of one each, in the seven
    # projections of two layers.
    model = small(weights, head_norm)
    lengths = [21, 1, 34, 0, 7]
    x = hidden(model, sum(lengths), 2)
    whole = model.new_state(5, 64)
    y = model.prompt(x, whole, lengths)
    assert y.shape == x.shape and torch.all(torch.isfinite(y))
    assert whole["lengths"].tolist() == lengths and int(whole["status"].item()) == 0
    at = 0
    for b, n in enumerate(lengths):
        single = model.new_state(1, 64)
        for t in range(n):
            z = model.step(x[at + t:at + t + 1], single)
        at += n
        if n:
            off = (y[at - 1].double() - z[0].double()).norm() / y[at - 1].double().norm()
            assert float(off) < (4 / 127 if weights == "w4" else 1 / 8), (b, float(off))


@pytest.mark.parametrize("weights,head_norm", FORMS)
def test_prompts_do_not_depend_on_their_neighbours(weights, head_norm):
    model = small(weights, head_norm)
    lengths = [40, 3, 50]
    x = hidden(model, 93, 3)
    state = model.new_state(3, 64)
    y = model.prompt(x, state, lengths)
    alone = model.new_state(3, 64)
    z = model.prompt(x[40:43], alone, [0, 3, 0])
    off = (y[40:43].double() - z.double()).norm() / z.double().norm()
    assert float(off) < 1e-2       # projections of 3 rows and of 93 sum in another order
    # the steps behind the prompts read what these have left in the cache
    new = hidden(model, 3, 4)
    after = model.step(new, state)
    assert torch.all(torch.isfinite(after)) and state["lengths"].tolist() == [41, 4, 51]
    assert int(state["status"].item()) == 0


def test_keys_of_a_prompt_are_in_the_cache():
    model = small("f8", True)
    x = hidden(model, 30, 5)
    state = model.new_state(2, 64)
    model.prompt(x, state, [20, 10])
    again = model.new_state(2, 64)
    model.prompt(x, again, [20, 10])
    for a, b in zip(state["caches"], again["caches"]):
        for k in a:
            assert torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8))
    pages = state["table"][0, :2].contiguous()
    k, v = api.rm_cache_read(state["caches"][0], pages, torch.float16)
    norms = k.view(32, 2, 64).float()[:20].square().mean(dim=2).sqrt()
    assert torch.all((norms > 0.8) & (norms < 1.25))      # normalised, gains near 1
    assert torch.all(k.view(32, 2, 64)[20:] == 0) and torch.all(v.view(32, 2, 64)[20:] == 0)


@pytest.mark.parametrize("weights,head_norm", FORMS)
def test_a_captured_step_replays_as_the_eager_one(weights, head_norm):
    model, n = small(weights, head_norm, torch.bfloat16), 3
    state, other = model.new_state(n, 64), model.new_state(n, 64)
    for s in (state, other):
        model.prompt(hidden(model, 30, 6), s, [10, 5, 15])
    x = hidden(model, n, 7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = model.step(x, state)
    torch.cuda.current_stream().wait_stream(side)
    for t in range(3):
        new = hidden(model, n, 60 + t)
        x.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, model.step(new, other)), t


def test_on_another_stream():
    model = small("f8", True)
    x = hidden(model, 100, 8)
    want = model.prompt(x, model.new_state(2, 64), [64, 36])
    state = model.new_state(2, 64)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y = torch.zeros_like(x)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        y.copy_(x)
        got = model.prompt(y, state, [64, 36])
    side.synchronize()
    assert torch.equal(got, want)


def test_two_calls_at_once():
    # on two streams, again and again, without workspaces of the caller's
    g = torch.Generator().manual_seed(10)
    x = torch.randn((300, 640), generator=g).bfloat16().cuda()
    w, s = api.rm_f8_quantize(torch.randn((900, 640), generator=g).bfloat16().cuda(), 128)
    qkv = torch.randn((400, 8, 128), generator=g).bfloat16().cuda()
    off = torch.tensor([0, 150, 400], dtype=torch.int32, device="cuda")

    def calls():
        return (api.rm_f8_linear(x, w, s), api.rm_f8_linear(x[:40], w, s),
                api.rm_prompt_attention(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], off, 250))
    want = calls()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for turn in range(20):
        with torch.cuda.stream(streams[turn % 2]):
            got.append(calls())
    torch.cuda.synchronize()
    for turn, outs in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), turn


def test_the_predictor_takes_prompts_and_steps():
    models = []
    for seed, (weights, head_norm) in enumerate(FORMS):
        model = small(weights, head_norm, seed=seed)
        lengths = [30, 50, 10]
        state = model.new_state(3, 64)
        model.prompt(hidden(model, 90, seed), state, lengths)
        models += [(model, state), (model, model.new_state(3, 64), lengths)]
    lib = decode.trace_library(models)
    counts = np.diff(lib["offsets"])
    # 8-bit floating weights: 90 rows are quantised in a launch of their own
    assert counts.tolist() == [17, 17, 19, 19, 17, 25, 19, 27]
    assert np.all(lib["duration"] > 0)
    dev = api.library_to_device(lib)
    st = api.new_status()
    occ = api.rm_occupancy(W.MI355X, dev["grid"], dev["threads"], dev["regs"], dev["smem"],
                           status=st)
    out = api.rm_pair_slowdown_matrix(W.MI355X, dev["offsets"], dev["grid"], dev["threads"],
                                      dev["regs"], dev["smem"], dev["duration"], status=st)
    assert int(st.item()) == 0 and torch.all(occ["blocks_per_sm"] > 0)
    assert torch.all(out["slowdown"] >= 0)


def test_refusals():
    with pytest.raises(ValueError):
        small("w8", False)
    model = small("w4", False)
    state = model.new_state(2, 64)
    for lengths in ([3], [3, -1], [1, 1, 1]):
        with pytest.raises(ValueError):
            model.prompt(hidden(model, 3, 9), state, lengths)
