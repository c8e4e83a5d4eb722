"""A table or upstream gradient that is not rows of one width is refused by name (no GPU needed)."""
import pytest
import torch

from paper_1711_06505_amd import ams


@pytest.mark.parametrize("shape", [(), (8,), (2, 4, 2)])
def test_not_rows(shape):
    i32 = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match=r"table is .*\[rows, width\] needed"):
        ams.ams_lookup_fwd(i32, torch.zeros(shape), torch.zeros((4, 8)))
    with pytest.raises(ValueError, match=r"dout is .*\[rows, width\] needed"):
        ams.ams_lookup_bwd(i32, i32, i32, i32, i32, 4, torch.zeros(shape), torch.zeros((4, 8)), torch.zeros(1))
