"""The operators of a policy's workers run together, as the example has them: its gradients against
differentiation of the plain formulas in 64 bits, and its answers against the whole sequences' call."""
import importlib.util
import os

import pytest
import torch
import torch.nn.functional as F

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "policy_workers.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("policy_workers", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain(E, theta, tokens, sequences):
    """Logits in 64 bits, from torch's own functions."""
    m = E.Model(*E_SIZES, theta=theta)
    p, n = m.views, tokens.numel() // sequences
    e = p["embed"][tokens.long()].view(sequences, n, -1)
    x = F.pad(e.transpose(1, 2), (E.WIDTH - 1, 0))
    u = F.silu(sum(x[:, :, j:j + n] * p["conv"][:, j, None] for j in range(E.WIDTH)) + p["conv_bias"][:, None]).transpose(1, 2)
    step = F.softplus(u @ p["wdt"] + p["dt_bias"])
    b, c, z = u @ p["wb"], u @ p["wc"], e @ p["wz"]
    a, h, ys = -p["rate"].exp(), 0.0, []
    for t in range(n):
        h = torch.exp(step[:, t, :, None] * a) * h + (step[:, t] * u[:, t])[:, :, None] * b[:, t, None]
        ys.append((h * c[:, t, None]).sum(2) + p["skip"] * u[:, t])
    y = torch.stack(ys, 1) * F.silu(z)
    return (y @ p["out"]).reshape(tokens.numel(), -1)


E_SIZES = (11, 20)


@pytest.mark.gpu
def test_gradient(example):
    E, S, n = example, 3, 37
    g = torch.Generator(device="cuda").manual_seed(0)
    m = E.Model(*E_SIZES).init(1)
    r = E.Runner(S, n, m, torch.cuda.current_stream().cuda_stream)
    tokens, action = (torch.randint(11, (S * n,), device="cuda", generator=g).to(torch.int32) for _ in range(2))
    theta = m.theta.double().cpu().requires_grad_()
    lp = torch.log_softmax(plain(E, theta, tokens.cpu(), S), 1).gather(1, action.cpu().long()[:, None])[:, 0]
    shift = torch.randn(S * n, generator=torch.Generator().manual_seed(3), dtype=torch.float64) * 0.1
    shift = shift.clamp(-0.17, 0.17)                  # inside the clip, away from its borders
    old, ref = (lp.detach() - shift).float(), (lp.detach() + 0.2).float()
    adv = torch.randn(S * n, generator=torch.Generator().manual_seed(4))
    d = ref.double() - lp
    loss = (-(lp - old.double()).exp() * adv.double() + 0.1 * (torch.expm1(d) - d)).mean()
    loss.backward()
    got, grad = r.gradient(m, tokens, action, old.cuda(), adv.cuda(), ref.cuda(), 0.1)
    assert abs(got.item() - loss.item()) < 1e-5
    want = E.Model(*E_SIZES, theta=theta.grad)
    for name, v in E.Model(*E_SIZES, theta=grad).views.items():
        w = want.views[name]
        # binary32 through the layers' products (sums of up to 111 terms) and a scan of 37 tokens: some 1e3
        # roundings of 2^-24 of the gradient's size.
        assert (v.double().cpu() - w).norm() <= 1e3 * 2.0 ** -24 * w.norm(), name


@pytest.mark.gpu
def test_answers_are_the_whole_sequences(example):
    E, S, n = example, 5, 12
    m = E.Model(*E_SIZES).init(2)
    r = E.Runner(S, n, m, torch.cuda.current_stream().cuda_stream)
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens, scores = r.answer(m, torch.arange(S, device="cuda"), n, g)
    z, _ = r.logits(m, tokens[:, :-1].reshape(-1).contiguous())
    again = r.scores(z, tokens[:, 1:].reshape(-1).contiguous()).view(S, n)
    # The matrix products of one token and of many may add in other orders: sums of 20 terms, four deep.
    assert (scores - again).abs().max() <= 2.0 ** -24 * 400 * (1 + scores.abs().max())


@pytest.mark.gpu
def test_runs(example):
    rewards, policy = example.train(steps=6, workers=3, vocab=8, dim=16, sequences=4, length=6)
    assert len(rewards) == 6 and all(0 <= v <= 1 for v in rewards)
    assert policy.theta.isfinite().all()
