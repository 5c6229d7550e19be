"""Asynchronous workers that distil a language model into a smaller one: the operators and the
commits together.

The model is an embedding, one gated recurrence and an output matrix.  A teacher's logits are
recorded as the likeliest tokens of each place (gem_token_scores); every worker holds its
snapshot of the student's parameters, takes the loss against that record and its gradient
(gem_distill_grad, gem_scan_backward), and commits its stale update to the master (gem_commit).
At the end the student answers token after token from a state kept in place.

    python examples/distill_workers.py [--steps N] [--workers n]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_1805_08469_amd import gem as G   # noqa: E402

GATE_BIAS = 2.0          # a state lives some eight tokens to begin with


class Model:
    """Parameters in one flat vector (what a commit updates), and the matrices as views of it."""

    def __init__(self, vocab: int, width: int, theta: torch.Tensor | None = None):
        self.vocab, self.width = vocab, width
        shapes = dict(embed=(vocab, width), wx=(width, width), wg=(width, width), out=(width, vocab))
        self.size = sum(a * b for a, b in shapes.values())
        self.theta = torch.zeros(self.size, device="cuda") if theta is None else theta
        at = 0
        self.views = {}
        for name, (a, b) in shapes.items():
            self.views[name] = self.theta[at:at + a * b].view(a, b)
            at += a * b

    def init(self, seed: int, gain: float = 1.0) -> "Model":
        """Random parameters; gain sets how sharp the output's distributions are."""
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.theta.copy_(torch.randn(self.size, device="cuda", generator=g))
        for name, scale in dict(wx=1.0, wg=1.0, out=gain).items():
            self.views[name].mul_(scale / math.sqrt(self.width))
        return self


class Runner:
    """Forward and backward of a model on `sequences` sequences of `length` tokens."""

    def __init__(self, sequences: int, length: int, width: int, stream: int | None = None):
        self.b, self.n, self.d = sequences, sequences * length, width
        self.ops = G.Ops(G.gem_scan_scratch(self.n, width), stream)
        self.states = torch.empty(G.gem_scan_state_rows(self.n), width, device="cuda")

    def logits(self, m: Model, tokens: torch.Tensor):
        """The logits of every place, and what the backward pass needs."""
        e = m.views["embed"][tokens.reshape(-1)]
        x, gate = e @ m.views["wx"], e @ m.views["wg"] + GATE_BIAS
        y = torch.empty_like(x)
        self.ops.scan_forward(x.data_ptr(), gate.data_ptr(), self.n, self.d, self.b, G.GEM_F32, y=y.data_ptr(),
                              states=self.states.data_ptr())
        return y @ m.views["out"], (e, x, gate, y)

    def record(self, z: torch.Tensor, k: int, temperature: float):
        """The k likeliest tokens of each place and their log probabilities."""
        ids = torch.empty(self.n, k, device="cuda", dtype=torch.int32)
        lp = torch.empty(self.n, k, device="cuda")
        self.ops.token_scores(z.data_ptr(), self.n, z.shape[1], G.GEM_F32, temperature=temperature, top_k=k,
                              top_ids=ids.data_ptr(), top_logprob=lp.data_ptr())
        return ids, lp

    def gradient(self, m: Model, tokens: torch.Tensor, record, temperature: float):
        """The mean loss of the places, and its gradient as one flat vector."""
        ids, lp = record
        z, (e, x, gate, y) = self.logits(m, tokens)
        loss = torch.empty(self.n, device="cuda")
        self.ops.distill_grad(z.data_ptr(), self.n, m.vocab, G.GEM_F32, ids=ids.data_ptr(), teacher=lp.data_ptr(),
                              k=ids.shape[1], tail=1, temperature=temperature, loss=loss.data_ptr(), grad=z.data_ptr())
        dz = z.div_(self.n)
        dy = dz @ m.views["out"].t()
        dx, dgate = torch.empty_like(x), torch.empty_like(x)
        self.ops.scan_backward(x.data_ptr(), gate.data_ptr(), self.n, self.d, self.b, G.GEM_F32,
                               states=self.states.data_ptr(), dy=dy.data_ptr(), dx=dx.data_ptr(), dgate=dgate.data_ptr())
        grad = Model(m.vocab, m.width)
        grad.views["out"].copy_(y.t() @ dz)
        grad.views["wx"].copy_(e.t() @ dx)
        grad.views["wg"].copy_(e.t() @ dgate)
        de = dx @ m.views["wx"].t() + dgate @ m.views["wg"].t()
        grad.views["embed"].index_add_(0, tokens.reshape(-1), de)
        return loss.mean(), grad.theta


def answer(m: Model, first: torch.Tensor, count: int):
    """`count` tokens after each of `first`, the likeliest one at a time, with their log
    probabilities: the recurrence's state is kept in place."""
    b, d = first.numel(), m.width
    h, y = torch.zeros(b, d, device="cuda"), torch.empty(b, d, device="cuda")
    ids = torch.empty(b, 1, device="cuda", dtype=torch.int32)
    lp = torch.empty(b, 1, device="cuda")
    token, out, scores = first, [], []
    with G.Ops(0, torch.cuda.current_stream().cuda_stream) as ops:
        for _ in range(count):
            e = m.views["embed"][token]
            x, gate = e @ m.views["wx"], e @ m.views["wg"] + GATE_BIAS
            ops.scan_forward(x.data_ptr(), gate.data_ptr(), b, d, b, G.GEM_F32, y=y.data_ptr(), h0=h.data_ptr(),
                             h_last=h.data_ptr())
            z = y @ m.views["out"]
            ops.token_scores(z.data_ptr(), b, m.vocab, G.GEM_F32, top_k=1, top_ids=ids.data_ptr(),
                             top_logprob=lp.data_ptr())
            token = ids[:, 0].long()
            out.append(token)
            scores.append(lp[:, 0].clone())
    return torch.stack(out, 1), torch.stack(scores, 1)


def train(steps=120, workers=4, vocab=500, width=64, sequences=4, length=64, k=32, temperature=1.0, lr=0.3, seed=0):
    """Losses of the committed updates, and the student."""
    stream = torch.cuda.current_stream().cuda_stream
    teacher = Model(vocab, 2 * width).init(seed + 1, gain=4.0)
    student = Model(vocab, width).init(seed + 2)
    tr, sr = Runner(sequences, length, 2 * width, stream), Runner(sequences, length, width, stream)
    g = torch.Generator(device="cuda").manual_seed(seed)
    order, _ = G.gem_schedule_make(workers, steps, G.GEM_LAW_EXP, seed=seed)
    data = [torch.randint(vocab, (sequences, length), device="cuda", generator=g) for _ in range(8)]
    records = [tr.record(tr.logits(teacher, t)[0], k, temperature) for t in data]
    losses = []
    snapshot = Model(vocab, width)
    with G.Gem(student.size, workers, stream=stream) as master:
        G.gem_set_theta(master.h, student.theta.data_ptr(), True)
        for step, w in enumerate(order):
            rc = G.lib().gem_read_state(master.h, int(w), G.GEM_SNAPSHOT, snapshot.theta.data_ptr(), 1)
            if rc != G.GEM_OK:
                raise G.GemError(rc, "gem_read_state")
            batch = step % len(data)
            loss, grad = sr.gradient(snapshot, data[batch], records[batch], temperature)
            grad.mul_(-lr)
            master.commit(grad.data_ptr(), int(w))
            losses.append(loss)
        student.theta.copy_(torch.from_numpy(master.theta()))
    return torch.stack(losses).tolist(), student


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=120)
    p.add_argument("--workers", type=int, default=4)
    a = p.parse_args()
    losses, student = train(a.steps, a.workers, lr=1.0)
    for i in range(0, len(losses), max(1, len(losses) // 6)):
        print(f"commit {i}: divergence from the teacher {losses[i]:.4f}")
    print(f"commit {len(losses) - 1}: {losses[-1]:.4f}")
    ids, lp = answer(student, torch.arange(2, device="cuda"), 8)
    for row, s in zip(ids.tolist(), lp.tolist()):
        print("answer", row, "log probability", round(sum(s), 3))


if __name__ == "__main__":
    main()
