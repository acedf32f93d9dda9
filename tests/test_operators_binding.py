"""What the operators' Python side refuses before it needs a GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


@pytest.mark.parametrize("out", [dict(), dict(h=None, h_last=None), dict(h=None, h_last=None, carry=None)])
def test_a_carry_that_has_no_place(apex, out):
    """Asked for, and left out in silence, it would be missed by the gradient."""
    x = torch.zeros((1, 2, 3))
    with pytest.raises(ValueError, match="carry"):
        apex.gated_scan(x, x, carry=True, out=out, workspace=x)
