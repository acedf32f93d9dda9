"""A draft model that learns from a prioritized memory what its target answers.

Actors draft G tokens ahead with a small recurrent model and have the target verify them.  Every verification becomes a row of
the replay memory: the tokens that stood, the draft's state in front of them, and the target's largest logits at each of them.
The learner samples rows by priority, runs the draft over them from the stored states, distils the stored logits, weighted by
importance, and writes each row's loss back as its priority.  The better the draft, the more tokens stand per verification.

    python examples/draft_distillation.py [rounds]

Both models are one gated recurrence between an embedding and a head: matrix products by PyTorch, everything between and behind
them by the library (gated_scan, verify_draft, distill_topk, and the memory's verbs).  A random target stands for a trained one.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1803_00933_amd import apex  # noqa: E402

DEVICE = "cuda:0"


def done(rc):
    if rc != apex.OK:
        raise RuntimeError(apex.STATUS_NAMES[rc])


class Scan(torch.autograd.Function):
    """gated_scan over the halves of one projection [S,T,2D], from h0 [S,D]; steps past `length` are no steps."""

    @staticmethod
    def forward(ctx, both, h0, length):
        D = both.shape[2] // 2
        rc, out = apex.gated_scan(both[:, :, :D], both[:, :, D:], h0=h0, length=length, carry=True)
        done(rc)
        ctx.save_for_backward(both, out["carry"])
        ctx.length = length
        return out["h"], out["h_last"]

    @staticmethod
    def backward(ctx, dh, dh_last):
        both, carry = ctx.saved_tensors
        D = both.shape[2] // 2
        grad = torch.empty_like(both)
        rc, back = apex.gated_scan_backward(both[:, :, :D], both[:, :, D:], dh.contiguous(), carry, length=ctx.length,
                                            dh_last=dh_last.contiguous(), out=dict(dg=grad[:, :, :D], dx=grad[:, :, D:]))
        done(rc)
        return grad, None, None


class Model:
    def __init__(self, V, D, gain, seed):
        g = torch.Generator(DEVICE)
        g.manual_seed(seed)
        made = [torch.randn(s, generator=g, device=DEVICE) * k for s, k in (((V, D), 1.0), ((D, 2 * D), gain / D ** 0.5), ((D, V), gain / D ** 0.5))]
        self.embedding, self.projection, self.head = made
        self.D = D

    def parameters(self):
        return [self.embedding, self.projection, self.head]

    def __call__(self, token, state, length=None):
        """Logits [S,T,V] behind each of the tokens [S,T], and the state [S,D] behind the last (or `length`-th) one."""
        h, last = Scan.apply(self.embedding[token.long()] @ self.projection, state, length)
        return h @ self.head, last


def uniforms(*shape):
    return torch.randint(-(1 << 63), (1 << 63) - 1, shape, device=DEVICE, dtype=torch.int64)


class Rows:
    """Layout of a row of the memory, in words of 32 bits."""

    def __init__(self, places, K, D):
        self.parts = [("token", places, torch.int32), ("index", places * K, torch.int32), ("value", places * K, torch.float32),
                      ("lse", places, torch.float32), ("state", D, torch.float32), ("length", 1, torch.int32)]
        self.words = sum(n for _, n, _ in self.parts)

    def pack(self, **what):
        return torch.cat([what[name].reshape(-1, n).view(torch.int32) for name, n, _ in self.parts], 1)

    def unpack(self, rows):
        out, at = {}, 0
        for name, n, dtype in self.parts:
            out[name] = rows[:, at:at + n].contiguous().view(dtype)
            at += n
        return out


def main(rounds=60, B=64, G=15, V=256, K=16, batch=128, learner_steps=8, lr=1e-2, seed=0, say=print):
    torch.manual_seed(seed)
    target, draft = Model(V, 32, 2.0, seed + 1), Model(V, 128, 1.0, seed + 2)
    for p in draft.parameters():
        p.requires_grad_(True)
    adam = torch.optim.Adam(draft.parameters(), lr=lr)
    rows = Rows(G + 1, K, draft.D)
    memory = apex.Replay(20_000, 32_768, 4 * rows.words, 4)
    batch_out = memory.alloc_sample_outputs(1, batch)
    verify_space = apex.verify_draft_workspace(B, V)
    state_d, state_t = torch.zeros(B, draft.D, device=DEVICE), torch.zeros(B, target.D, device=DEVICE)
    last = torch.randint(V, (B,), device=DEVICE, dtype=torch.int32)
    history = []
    for r in range(rounds):
        with torch.no_grad():
            # the actor: G tokens by the draft, one step of the recurrence at a time
            token, q, state = [last], [], state_d
            for _ in range(G):
                logits, state = draft(token[-1][:, None], state)
                q.append(torch.softmax(logits[:, 0], 1))
                token.append(torch.multinomial(q[-1], 1)[:, 0].int())
            token, q = torch.stack(token, 1), torch.stack(q, 1)
            answers, _ = target(token, state_t)
            rc, verdict = apex.verify_draft(torch.softmax(answers, 2), q, token[:, 1:].contiguous(), uniforms(B, G + 1), workspace=verify_space)
            done(rc)
            length = verdict["accepted"] + 1                      # the token they began with, and those that stood
            # what is learned from: the target's largest logits behind each of them
            value, index = answers.topk(K, dim=2)
            lse = torch.logsumexp(answers, 2)
            obs = rows.pack(token=token, index=index.int(), value=value, lse=lse, state=state_d, length=length)
            rc, _ = memory.add(torch.full((B,), 10.0, device=DEVICE), obs=obs.view(torch.uint8))   # new ones soon
            done(rc)
            _, state_d = draft(token, state_d, length)
            _, state_t = target(token, state_t, length)
            last = verdict["token"].gather(1, verdict["accepted"].long()[:, None])[:, 0]
        # the learner
        losses = []
        for _ in range(learner_steps):
            rc, out = memory.sample(1, batch, 0.4, uniforms(batch), out=batch_out)
            done(rc)
            row = rows.unpack(out["obs"].view(torch.int32))
            length = row["length"][:, 0].contiguous()
            inside = torch.arange(G + 1, device=DEVICE) < length[:, None]
            logits, _ = draft(row["token"], row["state"], length)
            weight = (out["weight"][:, None] * inside / inside.sum()).reshape(-1)
            rc, distilled = apex.distill_topk(logits.detach().reshape(-1, V), row["index"].reshape(-1, K), row["value"].reshape(-1, K),
                                              weight=weight, top_lse=row["lse"].reshape(-1))
            done(rc)
            adam.zero_grad(set_to_none=True)
            logits.backward(distilled["grad"].view_as(logits))
            adam.step()
            loss = (distilled["loss"].view(batch, G + 1) * inside).sum(1) / length
            done(memory.update_priorities(out["key"], loss))
            losses.append(loss.mean())
        rc, _ = memory.evict()
        done(rc)
        history.append((float(verdict["accepted"].float().mean()), float(torch.stack(losses).mean())))
        if r % 10 == 0 or r == rounds - 1:
            say("round %3d: %.2f of %d drafted tokens stand, loss %.3f" % (r, history[-1][0], G, history[-1][1]))
    return history


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:2]))
