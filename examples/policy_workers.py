"""Asynchronous workers that improve a policy: the operators and the commits together.

The model is an embedding, a short causal convolution, a selective state space scan with a gate, and an
output matrix.  A worker answers prompts with its snapshot of the parameters, token after token from
states kept in place (gem_embed_forward, gem_conv_forward, gem_ssm_forward, gem_token_scores); what it
answered is rewarded, and by the time it takes the gradient of the clipped policy loss
(gem_policy_grad, gem_ssm_backward, gem_conv_backward, gem_embed_backward) its answers are an older
policy's, whose ratio the loss clips.  It commits its stale update to the master (gem_commit).

    python examples/policy_workers.py [--steps N] [--workers n]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_1805_08469_amd import gem as G   # noqa: E402

WIDTH, STATE = 4, 8          # taps of the convolution, states of a channel
F32 = G.GEM_F32


class Model:
    """Parameters in one flat vector (what a commit updates), and views of it by name."""

    def __init__(self, vocab: int, dim: int, theta: torch.Tensor | None = None):
        self.vocab, self.dim = vocab, dim
        shapes = dict(embed=(vocab, dim), conv=(dim, WIDTH), conv_bias=(dim,), wdt=(dim, dim), wb=(dim, STATE), wc=(dim, STATE),
                      wz=(dim, dim), rate=(dim, STATE), skip=(dim,), dt_bias=(dim,), out=(dim, vocab))
        self.size = sum(math.prod(s) for s in shapes.values())
        self.theta = torch.zeros(self.size, device="cuda") if theta is None else theta
        self.views, at = {}, 0
        for name, s in shapes.items():
            self.views[name] = self.theta[at:at + math.prod(s)].view(s)
            at += math.prod(s)

    def init(self, seed: int) -> "Model":
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.theta.copy_(torch.randn(self.size, device="cuda", generator=g))
        for name in ("wdt", "wb", "wc", "wz", "out"):
            self.views[name].div_(math.sqrt(self.dim))
        self.views["conv"].mul_(0.5)
        self.views["conv_bias"].zero_()
        self.views["rate"].copy_(torch.arange(1, STATE + 1, device="cuda").float().log().expand(self.dim, STATE))
        self.views["skip"].fill_(1.0)
        self.views["dt_bias"].fill_(-2.0)
        return self

    def decay(self) -> torch.Tensor:
        """The scan's a: decays whose rates stay positive."""
        return -self.views["rate"].exp()


class Runner:
    """The model on `sequences` sequences of `length` tokens, forward and backward."""

    def __init__(self, sequences: int, length: int, m: Model, stream: int | None = None):
        self.b, self.n, self.d, self.v = sequences, sequences * length, m.dim, m.vocab
        scratch = max(G.gem_embed_scratch(self.n, m.vocab, m.dim), G.gem_conv_scratch(self.n, m.dim),
                      G.gem_ssm_scratch(self.n, m.dim, STATE))
        self.ops = G.Ops(scratch, stream)
        self.states = torch.empty(G.gem_ssm_state_rows(self.n), m.dim, STATE, device="cuda")

    def layer(self, m: Model, tokens: torch.Tensor, count: int, before=None, last=None, h0=None, h_last=None, states=None):
        """What the model makes of `count` tokens ahead of the output matrix, and all that leads there."""
        p, t = m.views, tokens.data_ptr()
        rows = [torch.empty(count, self.d, device="cuda") for _ in range(3)]
        e, u, y = rows
        self.ops.embed_forward(p["embed"].data_ptr(), t, count, self.v, self.d, F32, out=e.data_ptr(), out_dtype=F32)
        self.ops.conv_forward(e.data_ptr(), p["conv"].data_ptr(), count, self.d, self.b, WIDTH, F32, y=u.data_ptr(),
                              bias=p["conv_bias"].data_ptr(), before=before, last=last, act=1)
        a = m.decay()
        dt, b, c, z = u @ p["wdt"], u @ p["wb"], u @ p["wc"], e @ p["wz"]
        self.ops.ssm_forward(u.data_ptr(), dt.data_ptr(), b.data_ptr(), c.data_ptr(), a.data_ptr(), count, self.d, STATE, self.b, F32,
                             y=y.data_ptr(), z=z.data_ptr(), d=p["skip"].data_ptr(), dt_bias=p["dt_bias"].data_ptr(), h0=h0,
                             h_last=h_last, states=states)
        return e, u, dt, b, c, z, a, y

    def scores(self, z: torch.Tensor, tokens: torch.Tensor) -> torch.Tensor:
        """Log probabilities of one token of each row of logits."""
        lp = torch.empty(z.shape[0], device="cuda")
        self.ops.token_scores(z.data_ptr(), z.shape[0], self.v, F32, tokens=tokens.data_ptr(), n_tokens=1, logprob=lp.data_ptr())
        return lp

    def answer(self, m: Model, first: torch.Tensor, count: int, generator: torch.Generator):
        """`count` tokens drawn after each of `first` ([sequences, count + 1] with it), and the log
        probabilities under the policy that drew them."""
        before = torch.zeros(self.b, WIDTH - 1, self.d, device="cuda")
        h = torch.zeros(self.b, self.d, STATE, device="cuda")
        tokens, scores = [first.to(torch.int32)], []
        for _ in range(count):
            y = self.layer(m, tokens[-1], self.b, before.data_ptr(), before.data_ptr(), h.data_ptr(), h.data_ptr())[-1]
            z = y @ m.views["out"]
            noise = torch.rand(z.shape, device="cuda", generator=generator).clamp_(1e-20).log_().neg_().log_().neg_()
            tokens.append((z + noise).argmax(1).to(torch.int32))
            scores.append(self.scores(z, tokens[-1]))
        return torch.stack(tokens, 1), torch.stack(scores, 1)

    def logits(self, m: Model, tokens: torch.Tensor):
        saved = self.layer(m, tokens, self.n, states=self.states.data_ptr())
        return saved[-1] @ m.views["out"], saved

    def gradient(self, m: Model, tokens, action, old, advantage, ref, kl: float):
        """The mean loss of the actions and its gradient as one flat vector."""
        p, n, d = m.views, self.n, self.d
        z, (e, u, dt, b, c, gate, a, y) = self.logits(m, tokens)
        loss, w = torch.empty(n, device="cuda"), torch.full((n,), 1.0 / n, device="cuda")
        self.ops.policy_grad(z.data_ptr(), n, self.v, F32, action=action.data_ptr(), old_logprob=old.data_ptr(),
                             advantage=advantage.data_ptr(), ref_logprob=ref.data_ptr(), kl_coef=kl, weight=w.data_ptr(),
                             loss=loss.data_ptr(), grad=z.data_ptr())
        g = Model(m.vocab, m.dim)
        q = g.views
        q["out"].copy_(y.t() @ z)
        dy = z @ p["out"].t()
        du, ddt, dgate = (torch.empty_like(u) for _ in range(3))
        db, dc, da = torch.empty_like(b), torch.empty_like(c), torch.empty_like(a)
        self.ops.ssm_backward(u.data_ptr(), dt.data_ptr(), b.data_ptr(), c.data_ptr(), a.data_ptr(), n, d, STATE, self.b, F32,
                              states=self.states.data_ptr(), dy=dy.data_ptr(), dx=du.data_ptr(), ddt=ddt.data_ptr(), db=db.data_ptr(),
                              dc=dc.data_ptr(), z=gate.data_ptr(), dz=dgate.data_ptr(), d=p["skip"].data_ptr(),
                              dt_bias=p["dt_bias"].data_ptr(), da=da.data_ptr(), dd=q["skip"].data_ptr(),
                              ddt_bias=q["dt_bias"].data_ptr())
        q["rate"].copy_(da * a)
        for name, x, dx in (("wdt", u, ddt), ("wb", u, db), ("wc", u, dc), ("wz", e, dgate)):
            q[name].copy_(x.t() @ dx)
        du += ddt @ p["wdt"].t() + db @ p["wb"].t() + dc @ p["wc"].t()
        de = torch.empty_like(e)
        self.ops.conv_backward(e.data_ptr(), p["conv"].data_ptr(), n, d, self.b, WIDTH, F32, dy=du.data_ptr(), dx=de.data_ptr(),
                               dweight=q["conv"].data_ptr(), bias=p["conv_bias"].data_ptr(), dbias=q["conv_bias"].data_ptr(), act=1)
        de += dgate @ p["wz"].t()
        self.ops.embed_backward(tokens.data_ptr(), n, self.v, d, F32, dout=de.data_ptr(), dout_dtype=F32, grad=q["embed"].data_ptr())
        return loss.mean(), g.theta


def reward(tokens: torch.Tensor, vocab: int) -> torch.Tensor:
    """1 for an answer that follows the token before it, which is what the workers are to learn."""
    return (tokens[:, 1:] == (tokens[:, :-1] + 1) % vocab).float()


def train(steps=60, workers=4, vocab=16, dim=64, sequences=32, length=16, kl=0.0, lr=0.1, seed=0):
    """Mean rewards of the answers behind each commit, and the last policy."""
    stream = torch.cuda.current_stream().cuda_stream
    g = torch.Generator(device="cuda").manual_seed(seed)
    start = Model(vocab, dim).init(seed + 1)
    policy, snapshot = Model(vocab, dim, start.theta.clone()), Model(vocab, dim)
    runner = Runner(sequences, length, start, stream)
    order, _ = G.gem_schedule_make(workers, steps, G.GEM_LAW_EXP, seed=seed)
    waiting, rewards = {}, []

    def read(w: int):
        rc = G.lib().gem_read_state(master.h, w, G.GEM_SNAPSHOT, snapshot.theta.data_ptr(), 1)
        if rc != G.GEM_OK:
            raise G.GemError(rc, "gem_read_state")

    with G.Gem(policy.size, workers, stream=stream) as master:
        G.gem_set_theta(master.h, policy.theta.data_ptr(), True)
        for w in (int(v) for v in order):
            read(w)
            if w not in waiting:
                first = torch.randint(vocab, (sequences,), device="cuda", generator=g)
                waiting[w] = runner.answer(snapshot, first, length, g)
            drawn, old = waiting.pop(w)
            tokens, action = (t.reshape(-1).contiguous() for t in (drawn[:, :-1], drawn[:, 1:]))
            r = reward(drawn, vocab)
            advantage = (r - r.mean()).reshape(-1).contiguous()
            ref = runner.scores(runner.logits(start, tokens)[0], action)
            _, grad = runner.gradient(snapshot, tokens, action, old.reshape(-1).contiguous(), advantage, ref, kl)
            grad.mul_(-lr)
            # The next answers come from the policy that this commit has not reached yet.
            first = torch.randint(vocab, (sequences,), device="cuda", generator=g)
            waiting[w] = runner.answer(snapshot, first, length, g)
            master.commit(grad.data_ptr(), w)
            rewards.append(r.mean())
        policy.theta.copy_(torch.from_numpy(master.theta()))
    return torch.stack(rewards).tolist(), policy


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--workers", type=int, default=4)
    a = p.parse_args()
    rewards, _ = train(a.steps, a.workers)
    part = max(1, len(rewards) // 6)
    for i in range(0, len(rewards), part):
        some = rewards[i:i + part]
        print(f"commits {i} to {i + len(some) - 1}: mean reward {sum(some) / len(some):.3f}")


if __name__ == "__main__":
    main()
