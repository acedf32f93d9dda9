"""What the gated delta rule leaves for its gradient, where an episode ends on a piece's last step (GPU)."""
import pytest
import torch

import learning_plain as plain
from test_gpu_learning import Delta, apex, check  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes", [(2, 300, 1, 2, 40, 50), (1, 257, 1, 1, 128, 128), (9, 200, 4, 4, 128, 120)], ids=str)
def test_nothing_passes_into_a_piece_behind_an_episodes_end(apex, sizes, dtype):  # noqa: F811
    """The carry is what passes into a piece's first step: zeros behind an end, the state (to the bit what it is without the end) where
    there is none, and the gradient is that of either."""
    S, T, _, H, Dk, Dv = sizes
    c = Delta(*sizes, dtype, seed=T, cut=True, ragged=True)
    for at in (63, 127, 191):
        c.discount[:, at] = 0.99
    open_ended = c.run(apex)["carry"]
    c.discount[0, 63] = c.discount[-1, 127] = 0.0
    want = c.want()
    got = c.run(apex)
    c.check(got, want)

    def states(carry):
        x = carry.permute(0, 1, 2, 4, 6, 5, 3, 7)
        return x.reshape(*x.shape[:3], x.shape[3] * 32, -1)
    carry = states(got["carry"])
    length = c.length.cpu()
    seen = 0
    for s in range(S):
        for piece in range(-(-int(length[s]) // 64)):
            part = dict(want, carry=want["carry"][s:s + 1, piece], h_last_mag=want["h_last_mag"][s:s + 1])
            check(carry[s:s + 1, piece, :, :Dk, :Dv], part["carry"], plain.delta_bound("h_last", part, Dk, Dv), torch.float32, "carry %d %d" % (s, piece))
            if piece and c.discount[s, piece * 64 - 1] == 0:
                assert (carry[s, piece] == 0).all()
                seen += 1
            elif piece < 2 and (s, piece) != (0, 1):
                assert torch.equal(got["carry"][s, piece], open_ended[s, piece])
    assert seen and (carry[0, 1] == 0).all()
