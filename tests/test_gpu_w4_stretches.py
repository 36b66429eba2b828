"""rm_w4_linear where x does not fit in LDS whole and goes by in stretches.

Tolerance: that of test_gpu_w4_linear."""
import pytest
import torch

from paper_2607_16784_amd import api
from test_gpu_w4_linear import check, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,n,k,group,act", [
    (4, 16500, 4129, 32, "none"), (3, 16400, 9001, 128, "none"), (4, 32900, 4096, 64, "swiglu"),
    (1, 16384, 17000, 32, "none"), (4, 48, 24001, 32, "none"), (16, 80, 9000, 96, "none"),
    (16, 64, 4864, 32, "swiglu"), (2, 32, 60000, 128, "none")])
def test_stretches(rows, n, k, group, act, dtype):
    x, codes, scales, z, b = inputs(rows, n, k, group, dtype, True, True, seed=rows + n + k)
    got = api.rm_w4_linear(x, codes, scales, group, zeros=z, bias=b, act=act)
    keep = torch.arange(0, n // 2 if act == "swiglu" else n, max(1, n // 400))
    rows_of = torch.cat([keep, keep + n // 2]) if act == "swiglu" else keep
    # the reference of some outputs: all of them would take minutes
    check(x, codes[rows_of.cuda()], scales[rows_of.cuda()], group, z[rows_of.cuda()],
          b[rows_of.cuda()], act, got[:, keep.cuda()])
