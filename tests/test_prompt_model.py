"""What DecodeModel.prompt refuses before it changes a state; these need no GPU."""
import pytest
import torch

from paper_2607_16784_amd import decode


class Small(decode.DecodeModel):
    """A model without weights: only the checks of a prompt are asked."""

    def __init__(self):
        self.width, self.dtype, self.device = 64, torch.bfloat16, torch.device("cpu")

    def calls(self, x, state, new=1, lengths=None):
        yield "result", lambda: x


def test_rows_that_are_not_the_prompts():
    model = Small()
    state = {"table": torch.zeros((2, 4), dtype=torch.int32),
             "lengths": torch.tensor([7, 9], dtype=torch.int32)}
    x = torch.zeros((12, 64), dtype=torch.bfloat16)
    for lengths, rows in (([3, 4], x), ([8, 4], x[:11]), ([8, 4], x[:, :32]), ([6, 6], x[0]),
                          ([0, 0], x)):
        with pytest.raises(ValueError):
            model.prompt(rows, state, lengths)
        assert state["lengths"].tolist() == [7, 9]
    assert model.prompt(x, state, [8, 4]) is x and state["lengths"].tolist() == [8, 4]
    assert model.prompt(x[:0], state, [0, 0]).shape == (0, 64)
