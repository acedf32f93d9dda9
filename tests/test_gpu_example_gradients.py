"""Gradients of the example's model whose memory is a matrix per head, block by block, against the model in 64 bits: by its derivatives,
and by differences of its loss along directions that know nothing of the gradient.  (A direction that is the computed gradient itself
would not see a part of it that is missing.)"""
import pytest
import torch

from test_gpu_example_matrix import example  # noqa: F401

V, D, H, T = 40, 32, 2, 70
SIDE = D // H
# Roundings on a number's way, each 2^-24 of it: products with D, 3 D and 2 D terms, the unit length over SIDE, two pieces of the recurrence
# and of its gradient as in learning_plain (SIDE + 3 * 64, twice, + SIDE), the sum over the rows.  Steps are contractions, so that they add
# up; a sum of n rows of either sign is smaller than its terms' magnitudes by up to sqrt(n).
ROWS = 4 * T
LIMIT = (6 * D + SIDE + 2 * ((SIDE + 192) * 2 + SIDE) + ROWS) * ROWS ** 0.5 * 2.0 ** -24   # 1.4e-3 of a block's length


def reference(params, token, state, length):
    """The model step by step, in the type of its parameters, on the CPU."""
    table, projection, gates, head = params
    x = torch.where(((token >= 0) & (token < V))[..., None], table[token.clamp(0, V - 1)], 0.0)
    q, k, v = ((x @ projection).unflatten(2, (3, H, SIDE))).unbind(2)
    q, k = (torch.nn.functional.normalize(p, dim=3) for p in (q, k))
    decay, strength = (x @ gates).chunk(2, 2)
    keep, beta = torch.sigmoid(decay + 3.0), torch.sigmoid(strength)
    S, out = state.view(-1, H, SIDE, SIDE), []
    for t in range(token.shape[1]):
        left = keep[:, t, :, None, None] * S
        u = beta[:, t, :, None] * (v[:, t] - (left * k[:, t, :, :, None]).sum(2))
        new = left + k[:, t, :, :, None] * u[:, :, None]
        here = (t < length)[:, None, None, None]
        out.append(torch.where(here[..., 0], (new * q[:, t, :, :, None]).sum(2) * SIDE ** -0.5, 0.0))
        S = torch.where(here, new, S)
    return torch.cat((torch.stack(out, 1).flatten(2), x), 2) @ head, S.flatten(1)


def blocks():
    """name -> (parameter, part of it)."""
    b = {"row %d" % v: (0, (v,)) for v in range(V)}
    for i, n in enumerate("qkv"):
        for h in range(H):
            b["%s of head %d" % (n, h)] = (1, (slice(None), slice(i * D + h * SIDE, i * D + (h + 1) * SIDE)))
    for i, n in enumerate(("decay", "strength")):
        for h in range(H):
            b["%s of head %d" % (n, h)] = (2, (slice(None), i * H + h))
    for h in range(H):
        b["output of head %d" % h] = (3, (slice(h * SIDE, (h + 1) * SIDE),))
    b["output of the tokens' rows"] = (3, (slice(D, 2 * D),))
    return b


def loss_of(model, up, up_state, *inputs):
    logits, last = model(*inputs)
    return (logits * up).sum() + (last * up_state).sum()


def case():
    g = torch.Generator().manual_seed(3)
    token = torch.randint(-1, V + 1, (4, T), generator=g, dtype=torch.int32)
    length = torch.tensor([T, 0, 33, 1], dtype=torch.int32)
    inside = (torch.arange(T) < length[:, None])[:, :, None]
    state, up_state = (torch.randn(4, H * SIDE * SIDE, generator=g) for _ in range(2))
    return token, length, state, torch.randn(4, T, V, generator=g) * inside, up_state


def derivatives(params, token, length, state, up, up_state):
    params = [p.detach().double().cpu().requires_grad_(True) for p in params]
    loss = loss_of(lambda: reference(params, token.long(), state.double(), length.long()), up.double(), up_state.double())
    return torch.autograd.grad(loss, params)


def slopes(params, grads, token, length, state, up, up_state):
    """(block, slope of the 64-bit loss by differences along a random direction in it, what the gradients say, both lengths)."""
    params = [p.detach().double().cpu() for p in params]
    g = torch.Generator().manual_seed(5)

    def loss():
        with torch.no_grad():
            return float(loss_of(lambda: reference(params, token.long(), state.double(), length.long()), up.double(), up_state.double()))
    for name, (i, part) in blocks().items():
        if name.startswith("row") and name not in ("row 0", "row 7", "row 39"):
            continue
        for _ in range(2):
            d = torch.randn(params[i][part].shape, generator=g, dtype=torch.float64)
            step, at = 1e-6, params[i][part].clone()
            params[i][part] = at + step * d
            above = loss()
            params[i][part] = at - step * d
            slope = (above - loss()) / (2 * step)
            params[i][part] = at
            mine = grads[i][part].double().cpu()
            yield name, slope, float((mine * d).sum()), float(mine.norm() * d.norm())


# (differences in 64 bits: the loss, below 1e4, is off by 1e4 * 2^-53 * 1000 roundings, over 2e-6; a third derivative of 1e3 |d|^3 gives 1e-6)
DIFFERENCE = 1e-3


def plain_params():
    g = torch.Generator().manual_seed(1)
    return [torch.randn(s, generator=g) * k for s, k in (((V, D), 1.0), ((D, 3 * D), D ** -0.5), ((D, 2 * H), D ** -0.5), ((2 * D, V), (2 * D) ** -0.5))]


def test_the_reference_by_differences():
    """And that a block whose gradient is left at 0 is seen."""
    params, rest = plain_params(), case()
    grads = derivatives(params, *rest)
    for name, slope, mine, size in slopes(params, grads, *rest):
        assert abs(slope - mine) <= DIFFERENCE + 1e-6 * size, name
    planted = [g.clone() for g in grads]
    for name, (i, part) in blocks().items():
        planted[i][part] = 0.0
        if name in ("row 22", "row 28"):     # (the tokens that are not named)
            assert (grads[i][part] == 0).all()
        else:
            assert not (planted[i][part] - grads[i][part]).norm() <= LIMIT * grads[i][part].norm(), name


@pytest.mark.gpu
def test_gradients_block_by_block(example):  # noqa: F811
    model = example.MatrixModel(V, D, H, seed=1)
    for p, w in zip(model.parameters(), plain_params()):
        p.copy_(w)
        p.requires_grad_(True)
    token, length, state, up, up_state = case()
    loss = loss_of(model, up.cuda(), up_state.cuda(), token.cuda(), state.cuda(), length.cuda())
    grads = torch.autograd.grad(loss, model.parameters())
    want = derivatives(plain_params(), token, length, state, up, up_state)
    for name, (i, part) in blocks().items():
        off, size = float((grads[i][part].double().cpu() - want[i][part]).norm()), float(want[i][part].norm())
        assert off <= LIMIT * size, "%s: %.3g of %.3g off" % (name, off, size)
    for name, slope, mine, size in slopes(plain_params(), grads, token, length, state, up, up_state):
        assert abs(slope - mine) <= DIFFERENCE + LIMIT * size, (name, slope, mine)
