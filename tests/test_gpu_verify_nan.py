"""Verification where the probabilities of a row that is drawn from are no numbers: NaN has no mass, in the target's row or in the
draft's, whose tokens then keep all of the target's."""
import numpy as np
import pytest
import torch

import operators_plain as plain

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("B,V", [(40, 9), (40, 1003), (30, 9001), (2, 300007)])
@pytest.mark.parametrize("share", [0.0005, 0.3, 1.0])
def test_rows_with_nan(apex, dtype, B, V, share):
    """Every drafted token is turned down (the target gives it nothing), with NaN at others in the draft's row, in the target's, and
    in both; values below 0 and above 1 among them."""
    rng = np.random.default_rng(V)
    G = 2
    target, draft = rng.dirichlet(np.ones(V), (B, G + 1)), rng.dirichlet(np.ones(V), (B, G))
    token = rng.integers(0, V, (B, G)).astype(np.int32)
    rnd = rng.integers(1 << 40, 1 << 64, (B, G + 1), dtype=np.uint64)
    for a, rows in ((draft, slice(0, None, 2)), (target, slice(1, None, 3))):
        a[rows][rng.random(a[rows].shape) < share] = np.nan
    draft[:, :, V // 2], target[:, :, V // 3] = -1.0, 3.0
    np.put_along_axis(target[:, :G], token[:, :, None].astype(np.int64), 0.0, 2)
    np.put_along_axis(draft, token[:, :, None].astype(np.int64), 0.9, 2)
    dev = lambda a, *t: torch.from_numpy(a).to("cuda:0", *t)  # noqa: E731
    target, draft = dev(target, DTYPES[dtype]), dev(draft, DTYPES[dtype])
    want = plain.verify(plain.f64(target), plain.f64(draft), token, rnd)
    rc, out = apex.verify_draft(target, draft, dev(token), dev(rnd.view(np.int64)))
    assert rc == apex.OK
    assert (want[0] == 0).all()
    assert np.array_equal(out["accepted"].cpu().numpy(), want[0]) and np.array_equal(out["token"].cpu().numpy(), want[1])
