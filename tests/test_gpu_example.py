"""examples/distill_workers.py: the operators and the commits used together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "distill_workers.py")


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


@pytest.fixture(scope="module")
def example(torch):
    spec = importlib.util.spec_from_file_location("distill_workers", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _loss(torch, theta, vocab, width, tokens, ids, lp, T):
    """The mean distillation loss in 64 bits on the CPU, token after token, for autograd."""
    at, parts = 0, []
    for a, b in ((vocab, width), (width, width), (width, width), (width, vocab)):
        parts.append(theta[at:at + a * b].view(a, b))
        at += a * b
    embed, wx, wg, out = parts
    e = embed[tokens]
    x, a = e @ wx, torch.sigmoid(e @ wg + 2.0)
    h, ys = torch.zeros(tokens.shape[0], width, dtype=theta.dtype), []
    for t in range(tokens.shape[1]):
        h = a[:, t] * h + (1 - a[:, t]) * x[:, t]
        ys.append(h)
    z = torch.stack(ys, 1).reshape(-1, width) @ out
    logq = torch.log_softmax(z / T, 1)
    p = lp.exp()
    listed = torch.zeros_like(logq, dtype=torch.bool).scatter_(1, ids, True)
    pt = 1 - p.sum(1)
    qt = logq.exp().masked_fill(listed, 0).sum(1)
    return ((p * (lp - logq.gather(1, ids))).sum(1) + pt * (pt.log() - qt.log())).mean()


def test_a_workers_gradient_is_the_losss(torch, example):
    """Through the embedding, the recurrence and the loss, against autograd in 64 bits."""
    vocab, width, b, n, k, T = 90, 24, 3, 37, 8, 1.3
    m = example.Model(vocab, width).init(3)
    teacher = example.Model(vocab, width).init(4)
    tokens = torch.randint(vocab, (b, n), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    r = example.Runner(b, n, width, torch.cuda.current_stream().cuda_stream)
    record = r.record(r.logits(teacher, tokens)[0], k, T)
    loss, grad = r.gradient(m, tokens, record, T)
    theta = m.theta.double().cpu().requires_grad_()
    want = _loss(torch, theta, vocab, width, tokens.cpu(), record[0].long().cpu(), record[1].double().cpu(), T)
    want.backward()
    # Products and sums of at most 111 terms in 32 bits, five of them in a row, and exponentials
    # of logits below 16: a few thousand units of the largest gradient's last place at most.
    assert abs(float(loss) - want.item()) < 2e-5 * max(1.0, abs(want.item()))
    off = (grad.double().cpu() - theta.grad).abs().max()
    assert float(off) < 2e-4 * float(theta.grad.abs().max())


def test_workers_learn_from_the_record(torch, example):
    losses, student = example.train(steps=48, workers=3, vocab=200, width=32, sequences=2, length=32, k=16)
    assert all(l == l for l in losses)
    assert sum(losses[-8:]) < 0.9 * sum(losses[:8])
    ids, lp = example.answer(student, torch.arange(5, device="cuda"), 6)
    assert ids.shape == (5, 6) and bool((lp <= 0).all()) and bool(((ids >= 0) & (ids < 200)).all())
