"""Arguments of the prompt's calls at the ends of their ranges; these need no GPU."""
import numpy as np

from test_prompt_refusals import lib  # noqa: F401


def test_scales_whose_logits_leave_fp32(lib):  # noqa: F811
    # the exponentials take scale times log2(e), which times a product of 0 has to be 0
    def call(scale):                      # of no tokens
        return lib.rm_prompt_attention(0, 0, 4, 2, 64, None, 256, 64, None, 128, 64, None, 128, 64,
                                       None, 1, 3, scale, 0, None, None, None)
    most = float(np.finfo(np.float32).max) * np.log(2.0)
    for scale in (most * 1.00001, 3e38, -3e38):
        assert call(scale) == 1, scale
    for scale in (most * 0.9999, -2.3e38, 1e-45, 0.0):
        assert call(scale) == 0, scale
