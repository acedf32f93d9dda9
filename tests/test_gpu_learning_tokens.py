"""Tokens of any shape (GPU)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


@pytest.mark.parametrize("shape", [(), (1,), (24,), (4, 6), (2, 3, 4), (2, 3, 2, 2), (1, 2, 3, 2, 2)], ids=str)
def test_tokens_of_any_shape(apex, shape):
    """One token, and as many dimensions as there are: the rows are those of the tokens one after the other."""
    g = torch.Generator("cuda:0").manual_seed(0)
    table = torch.randn((9, 5), generator=g, device="cuda:0")
    token = torch.randint(0, 9, shape, generator=g, device="cuda:0", dtype=torch.int32)
    N = token.numel()
    rc, out = apex.embedding(table, token)
    assert rc == apex.OK and torch.equal(out["out"], table[token.view(-1).long()])
    dout = torch.randn((N, 5), generator=g, device="cuda:0")
    rc, out = apex.embedding_backward(dout, token, 9)
    assert rc == apex.OK
    rc, flat = apex.embedding_backward(dout, token.view(-1), 9)
    assert rc == apex.OK and torch.equal(out["dtable"], flat["dtable"])


def test_tokens_that_do_not_lie_one_after_the_other_are_refused(apex):
    table = torch.zeros((9, 5), device="cuda:0")
    token = torch.zeros((2, 3, 2, 4), dtype=torch.int32, device="cuda:0")
    with pytest.raises(AssertionError, match="token"):
        apex.embedding(table, token[0, :, :, 0])
    with pytest.raises(RuntimeError, match="view"):
        apex.embedding(table, token.transpose(0, 3))
