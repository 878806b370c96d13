"""What the binding of the linear layers refuses before the library is called: no GPU needed."""
import pytest
import torch

from paper_2409_02097_amd import layers

HEAD = (-1, torch.float32)   # tensors in host memory


def test_rows_of_a_weight():
    w = torch.zeros(16, 24)
    assert layers._matrix("w", w, (16, 24), HEAD) == 24
    assert layers._matrix("w", torch.zeros(16, 32)[:, 8:], (16, 24), HEAD) == 32
    assert layers._matrix("w", torch.zeros(1, 24), (1, 24), HEAD) == 24


@pytest.mark.parametrize("w", [torch.zeros(1, 24).expand(16, 24), torch.zeros(24).expand(16, 24), torch.zeros(400).as_strided((16, 24), (8, 1)),
                               torch.zeros(24, 16).t(), torch.zeros(16, 16), torch.zeros(16, 24, dtype=torch.float16)],
                         ids=["one row for all", "one vector for all", "rows in one another", "transposed", "another width", "another type"])
def test_weights_that_are_no_rows_one_behind_the_other(w):
    """A stride of 0 would be read as that of contiguous rows, far behind the one row that is there."""
    with pytest.raises(ValueError, match="^w"):
        layers._matrix("w", w, (16, 24), HEAD)
