"""rm_f8_linear with many outputs: few rows in the largest tiles, results beyond 2^31
elements, and the largest tiles in a graph (tolerances: test_gpu_f8_linear, check)."""
import pytest
import torch

from paper_2607_16784_amd import api
from test_gpu_f8_linear import check, normal, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [17, 33, 64])
@pytest.mark.parametrize("act", ["none", "swiglu"])
@pytest.mark.parametrize("given", [False, True], ids=["x", "codes"])
def test_few_rows_of_a_wide_projection(rows, act, given):
    n, k = 37008, 256
    codes, scales = weights(n, k, act, rows)
    x, x_scales = normal((rows, k), rows, torch.bfloat16), None
    if given:
        x, x_scales = api.rm_f8_quantize(x)
    y = api.rm_f8_linear(x, codes, scales, x_scales=x_scales, act=act, dtype=torch.bfloat16)
    check(y, x, codes, scales, torch.bfloat16, x_scales=x_scales, act=act)


def test_results_beyond_31_bits():
    rows, n, k = 40000, 60000, 128
    codes, scales = api.rm_f8_quantize(normal((n, k), 2, torch.bfloat16), 128)
    x = normal((rows, k), 3, torch.bfloat16)
    y = api.rm_f8_linear(x, codes, scales)
    first = n // 128 * 128 - 128
    for lo in (0, 17000, rows - 20):
        check(y[lo:lo + 20, first:], x[lo:lo + 20], codes[first:], scales[first // 128:],
              torch.bfloat16)


@pytest.mark.parametrize("rows,n,k", [(300, 40960, 256), (200, 20000, 256), (100, 20000, 250),
                                      (64, 256, 12800)])
def test_large_tiles_in_a_graph(rows, n, k):
    codes, scales = weights(n, k, "none", 4)
    x = normal((rows, k), 5, torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = api.rm_f8_linear(x, codes, scales)
    torch.cuda.current_stream().wait_stream(side)
    for turn in range(3):
        x.add_(0.25)
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, api.rm_f8_linear(x, codes, scales)), turn
