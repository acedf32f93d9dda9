"""What the operators' binding refuses before anything is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


def scan_inputs(S, T, D):
    return torch.zeros((S, T, D), device="cuda:0"), torch.ones((S, T, D), device="cuda:0")


def test_workspaces_that_are_too_small(apex):
    """One made for smaller sizes, and one a byte short; the smallest that is enough, and a larger one, are taken."""
    S, T, D = 3, 700, 200
    g, x = scan_inputs(S, T, D)
    dh = torch.ones_like(x)
    whole = apex.gated_scan_workspace(S, T, D)
    rc, out = apex.gated_scan(g, x, carry=True, workspace=whole)
    assert rc == apex.OK
    larger = torch.zeros(whole.numel() + 512, dtype=torch.uint8, device="cuda:0")
    for space in (whole, larger):
        assert apex.gated_scan(g, x, workspace=space)[0] == apex.OK
        assert apex.gated_scan_backward(g, x, dh, out["carry"], workspace=space)[0] == apex.OK
    for space in (whole[:-1], whole[:256], apex.gated_scan_workspace(S, T - 64, D), apex.gated_scan_workspace(S - 1, T, D),
                  apex.gated_scan_workspace(S, T, D - 100)):
        with pytest.raises(AssertionError, match="workspace"):
            apex.gated_scan(g, x, workspace=space)
        with pytest.raises(AssertionError, match="workspace"):
            apex.gated_scan_backward(g, x, dh, out["carry"], workspace=space)
    # where no workspace is needed one of any size is taken
    assert apex.gated_scan(g[:, :100], x[:, :100], workspace=whole[:256])[0] == apex.OK
    B, G, V = 5, 2, 3000
    target, draft = torch.rand((B, G + 1, V), device="cuda:0"), torch.rand((B, G, V), device="cuda:0")
    token = torch.zeros((B, G), dtype=torch.int32, device="cuda:0")
    rnd = torch.zeros((B, G + 1), dtype=torch.int64, device="cuda:0")
    whole = apex.verify_draft_workspace(B, V)
    assert apex.verify_draft(target, draft, token, rnd, workspace=whole)[0] == apex.OK
    for space in (whole[:-1], apex.verify_draft_workspace(B - 1, V)):
        with pytest.raises(AssertionError, match="workspace"):
            apex.verify_draft(target, draft, token, rnd, workspace=space)
    torch.cuda.synchronize()


def test_tickets_that_are_none_of_the_call_are_dropped(apex):
    """A workspace whose counters are far from zero: no tile is any of the call's, so nothing but the workspace's own counters is
    written, and nothing waits."""
    for S, T, D, back in ((1, 300, 70, False), (1, 300, 70, True), (2, 1000, 300, False), (2, 1000, 300, True)):
        g, x = scan_inputs(S, T, D)
        n = apex.gated_scan_workspace(S, T, D).numel()
        held = torch.full((n + 4096,), 0, dtype=torch.uint8, device="cuda:0")
        for taken in (1 << 20, 0x7fffff00):
            held.zero_()
            counters = held[256:256 + 1024 * 128].view(torch.int32).view(1024, 32)
            counters[:, 0] = taken
            had = held.clone()
            carry = torch.full(apex.gated_scan_carry_shape(S, T, D), 7.0, device="cuda:0")
            written = [torch.full((S, T, D), 7.0, device="cuda:0") for _ in range(2)] + [torch.full((S, D), 7.0, device="cuda:0")]
            if back:
                rc, _ = apex.gated_scan_backward(g, x, torch.ones_like(x), carry, workspace=held[:n],
                                                 out=dict(dg=written[0], dx=written[1], dh0=written[2]))
            else:
                rc, _ = apex.gated_scan(g, x, workspace=held[:n], out=dict(h=written[0], h_last=written[2], carry=carry))
            assert rc == apex.OK
            torch.cuda.synchronize()
            assert all((t == 7.0).all() for t in written + [carry])
            taken_by = held[256:256 + 1024 * 128].view(torch.int32).view(1024, 32)[:, 0] - taken
            assert int(taken_by.sum()) == S * -(-T // 64) * -(-D // 128)
            counters[:, 0] = taken
            assert torch.equal(held, had)


def test_arrays_without_elements_are_not_taken_for_none(apex):
    """An empty tensor has no address, like None; where an array of some size belongs it is refused all the same."""
    S, T, D = 2, 20, 8
    g, x = scan_inputs(S, T, D)
    nothing, no_ints = torch.empty(0, device="cuda:0"), torch.empty(0, dtype=torch.int32, device="cuda:0")
    for name, a in (("discount", nothing), ("length", no_ints), ("h0", nothing)):
        with pytest.raises(AssertionError, match=name):
            apex.gated_scan(g, x, **{name: a})
    rc, out = apex.gated_scan(g, x, carry=True)
    for name in ("h_last", "carry"):
        with pytest.raises(AssertionError, match=name):
            apex.gated_scan(g, x, out={**out, name: nothing})
    with pytest.raises(AssertionError, match="dh_last"):
        apex.gated_scan_backward(g, x, x, out["carry"], dh_last=nothing)
    logits, index, value = torch.zeros((3, 40), device="cuda:0"), torch.zeros((3, 2), dtype=torch.int32, device="cuda:0"), torch.zeros((3, 2), device="cuda:0")
    for name in ("weight", "top_lse"):
        with pytest.raises(AssertionError, match=name):
            apex.distill_topk(logits, index, value, **{name: nothing})
    loss = torch.zeros(3, device="cuda:0")
    for name in ("lse", "grad"):
        with pytest.raises(AssertionError, match=name):
            apex.distill_topk(logits, index, value, out=dict(loss=loss, **{name: nothing}))
    target, rnd = torch.rand((3, 1, 40), device="cuda:0"), torch.zeros((3, 1), dtype=torch.int64, device="cuda:0")
    with pytest.raises(AssertionError, match="length"):
        apex.verify_draft(target, None, None, rnd, length=no_ints)
    # a draft of no tokens has no tokens, of whatever type
    draft = torch.empty((3, 0, 40), device="cuda:0")
    for dtype in (torch.int32, torch.int64):
        assert apex.verify_draft(target, draft, torch.empty((3, 0), dtype=dtype, device="cuda:0"), rnd)[0] == apex.OK
    torch.cuda.synchronize()
