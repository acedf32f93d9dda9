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


@pytest.mark.parametrize("temperature", [1e-45, 1e-40, 4e-39])
def test_temperatures_whose_reciprocal_is_no_number(apex, temperature):
    """log2(e) / temperature is beyond 32 bits: logits times that would be infinite or NaN."""
    a = 1 << 20
    assert apex.lib.apex_distill_topk(1, 8, 1, 0, a, 8, a, 0, a, None, None, temperature, a, None, None, 0, None, None) == apex.ERR_INVALID_ARG
