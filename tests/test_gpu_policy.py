"""The clipped policy loss and its gradient against the formula in 64 bits."""
import math

import pytest
import torch

from paper_1805_08469_amd import gem as G

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
KIND = {torch.float32: G.GEM_F32, torch.bfloat16: G.GEM_BF16}
TERMS = ("loss", "logprob", "ratio", "kl")


def formula(z, T, action, old, adv, ref, low, high, beta, weight):
    """Terms and gradient in 64 bits, and a bound of each: the log probability is off by eps (four
    roundings of terms no larger than |lp| and 28, since a reference lies at most 20 octaves below the
    largest logit, and V/256 additions a thread, joined in a few steps), all else by what that does."""
    z = z.double() / T
    rows, V = z.shape
    w = torch.ones(rows, dtype=torch.float64, device=z.device) if weight is None else weight.double()
    live = (w != 0) & (action >= 0) & (action < V)
    at = torch.where(live, action, 0).long()[:, None]
    logq = torch.log_softmax(z, 1)
    lp = logq.gather(1, at)[:, 0]
    eps = U * (4 * lp.abs() + V / 256 + 144)
    old, adv = old.double(), adv.double()
    ratio = (lp - old).exp()
    ratio_e = ratio * (eps + U * ((lp - old).abs() + 4))
    free, held = ratio * adv, ratio.clamp(1 - low, 1 + high) * adv
    gain = torch.where(adv == 0, 0.0, torch.minimum(free, held))
    slope = torch.where((adv != 0) & (free <= held), -free, 0.0)
    loss, loss_e = -gain, adv.abs() * ratio_e + 4 * U * gain.abs()
    slope_e = torch.where(slope != 0, adv.abs() * ratio_e + 4 * U * free.abs(), 0.0)
    kl = kl_e = torch.zeros_like(lp)
    if ref is not None:
        d = ref.double() - lp
        d_e = eps + U * d.abs()
        kl = torch.expm1(d) - d
        # A difference of e^d - 1 and d outside the series, which is |d| < 1/4.
        kl_e = torch.expm1(d).abs() * d_e + d_e ** 2 + 8 * U * (kl + torch.where(d.abs() > 0.2, d.abs() + torch.expm1(d).abs(), 0.0))
        if beta:
            loss, loss_e = loss + beta * kl, loss_e + beta * kl_e + 4 * U * beta * kl
            slope, slope_e = slope - beta * torch.expm1(d), slope_e + beta * (d.exp() * d_e + 8 * U * torch.expm1(d).abs())
    f, f_e = w / T * slope, w.abs() / T * (slope_e + 8 * U * slope.abs())
    q = logq.exp()
    q_e = q * U * ((z.amax(1, keepdim=True) - z).clamp(max=1e4) * 4 + V / 256 + 200)
    hit = torch.zeros_like(q).scatter_(1, at, 1.0)
    g = f[:, None] * (hit - q)
    g_e = f_e[:, None] * (hit - q).abs() + f.abs()[:, None] * (q_e + 4 * U * hit)
    zero = torch.zeros_like(lp)
    terms = {n: (torch.where(live, v, zero), torch.where(live, e, zero) + 4 * U * v.abs().nan_to_num())
             for n, v, e in (("loss", loss, loss_e), ("logprob", lp, eps), ("ratio", ratio, ratio_e), ("kl", kl, kl_e))}
    return terms, torch.where(live[:, None], g, 0.0), torch.where(live[:, None], g_e, 0.0), live


def inputs(rows, vocab, dtype, pad=0, T=1.0, seed=0, low=0.2, high=0.3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.zeros(rows, vocab + pad, device="cuda", dtype=dtype)[:, :vocab]
    z.copy_(torch.randn(rows, vocab, device="cuda", generator=g) * 3)
    action = torch.randint(vocab, (rows,), device="cuda", generator=g)
    lp = torch.log_softmax(z.double() / T, 1).gather(1, action[:, None])[:, 0]
    shift = torch.randn(rows, device="cuda", generator=g, dtype=torch.float64) * 0.3
    for border in (math.log1p(-low), math.log1p(high)):        # where the gradient jumps
        shift = torch.where((shift - border).abs() < 1e-2, border + 3e-2, shift)
    ref = lp + torch.randn(rows, device="cuda", generator=g, dtype=torch.float64) * 0.4
    adv = torch.randn(rows, device="cuda", generator=g)
    if rows > 4:
        adv[3] = 0.0
        action[4] = -1
    w = torch.rand(rows, device="cuda", generator=g) + 0.5
    if rows > 2:
        w[2] = 0.0
    return z, action.to(torch.int32), (lp - shift).float(), adv, ref.float(), w


def ptr(t):
    return None if t is None else t.data_ptr()


def call(ops, z, action, old, adv, ref, w, T=1.0, low=0.2, high=0.3, beta=0.1, grad=None, terms=None):
    rows, vocab = z.shape
    if terms is None:
        terms = {n: torch.full((rows,), 7.0, device="cuda") for n in TERMS}
    args = dict(action=ptr(action), old_logprob=ptr(old), advantage=ptr(adv), ref_logprob=ptr(ref), clip_low=low,
                clip_high=high, kl_coef=beta, stride=z.stride(0), temperature=T, weight=ptr(w), **{n: ptr(t) for n, t in terms.items()})
    if grad is None:
        ops.policy_loss(z.data_ptr(), rows, vocab, KIND[z.dtype], **args)
    else:
        ops.policy_grad(z.data_ptr(), rows, vocab, KIND[z.dtype], grad=grad.data_ptr(), grad_stride=grad.stride(0), **args)
    return terms


@pytest.fixture
def ops():
    with G.Ops(0, torch.cuda.current_stream().cuda_stream) as o:
        yield o


def check(terms, want, dz=None, g=None, g_e=None):
    for n in TERMS:
        v, e = want[n]
        off = (terms[n].double() - v).abs() - e
        assert (off <= 0).all(), (n, off.max().item())
    if dz is not None:
        off = (dz.double() - g).abs() - g_e - g.abs() * HALF[dz.dtype] - 1e-37
        assert (off <= 0).all(), off.max().item()


SIZES = [(1, 1), (1, 7), (1, 50021), (3, 8200), (5, 2), (37, 20011), (256, 4096), (300, 1000), (300, 8), (261, 5001),
         (257, 32768), (260, 65000), (259, 131072), (258, 140003)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_loss_and_gradient(ops, rows, vocab, dtype):
    """Rows in parts, in one block, in registers, and beyond them; aligned, and not."""
    for pad, T, kl in ((0, 1.0, True), (5, 0.7, False)):
        z, action, old, adv, ref, w = inputs(rows, vocab, dtype, pad, T)
        if not kl:
            ref = w = None
        want, g, g_e, _ = formula(z, T, action, old, adv, ref, 0.2, 0.3, 0.1, w)
        check(call(ops, z, action, old, adv, ref, w, T), want)
        dz = torch.full((rows, vocab + pad), 7.0, device="cuda", dtype=dtype)
        terms = call(ops, z, action, old, adv, ref, w, T, grad=dz[:, :vocab])
        check(terms, want, dz[:, :vocab], g, g_e)
        assert (dz[:, vocab:] == 7).all()
        keep = {n: t.clone() for n, t in terms.items()}
        call(ops, z, action, old, adv, ref, w, T, grad=z, terms=terms)       # over the logits
        assert torch.equal(z, dz[:, :vocab])
        assert all(torch.equal(keep[n], terms[n]) for n in TERMS)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(3, 40), (9, 20011), (300, 515), (258, 140003)])
def test_rows_out_of_the_ordinary(ops, rows, vocab):
    """Rows without weight or token are not read; impossible tokens, masks and no numbers."""
    z, action, old, adv, ref, w = inputs(rows, vocab, torch.float32)
    w[:] = 0.5
    adv[:] = 1.5
    action[:] = 7
    dz = torch.empty_like(z)
    z[0], w[0] = math.nan, 0.0
    z[1], action[1] = math.nan, vocab
    z[2, 7] = -math.inf                      # the token that was taken cannot occur
    terms = call(ops, z, action, old, adv, ref, w, beta=0.0, grad=dz)
    for n in TERMS:
        assert terms[n][0] == 0 and terms[n][1] == 0
    assert (dz[:2] == 0).all() and (dz[2] == 0).all()
    assert terms["logprob"][2] == -math.inf and terms["ratio"][2] == 0 and terms["loss"][2] == 0
    assert terms["kl"][2] == math.inf
    assert call(ops, z, action, old, adv, ref, w, beta=0.1)["loss"][2] == math.inf
    adv[2] = -2.0                            # a ratio held at 0.8
    terms = call(ops, z, action, old, adv, ref, w, beta=0.0, grad=dz)
    assert abs(terms["loss"][2].item() - 1.6) < 1e-6 and (dz[2] == 0).all()
    z, action, old, adv, ref, w = inputs(rows, vocab, torch.float32, seed=3)
    action[:], w[:] = 7, 1.0
    z[0] = -math.inf
    z[1, 5] = math.nan
    z[2, 5] = math.inf
    terms = call(ops, z, action, old, adv, ref, w, grad=dz)
    assert terms["logprob"][0] == -math.inf
    assert all(terms[n][1:3].isnan().all() for n in TERMS)
    assert dz[1:3].isnan().all()
    # Masks by -inf and by the type's lowest value.
    for mask in (-math.inf, torch.finfo(torch.float32).min):
        z, action, old, adv, ref, w = inputs(rows, vocab, torch.float32, seed=4)
        action[:] = 3
        z[:, 8:] = mask
        old = torch.log_softmax(z.double(), 1)[:, 3].float() - 0.05
        ref = old + 0.2
        want, g, g_e, _ = formula(z, 1.0, action, old, adv, ref, 0.2, 0.3, 0.1, w)
        check(call(ops, z, action, old, adv, ref, w, grad=dz), want, dz, g, g_e)
        assert (dz[:, 8:] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(3, 30), (7, 20011), (300, 4099), (259, 131071)])
def test_rows_that_start_anywhere(ops, rows, vocab, dtype):
    """Logits and gradient of other alignments and strides, and what lies around them."""
    z, action, old, adv, ref, w = inputs(rows, vocab, dtype)
    want, g, g_e, _ = formula(z, 1.0, action, old, adv, ref, 0.2, 0.3, 0.1, w)
    for a, b in ((1, 3), (3, 0), (2, 5)):
        zs = torch.full((rows * (vocab + 3) + 8,), math.nan, device="cuda", dtype=dtype)
        gs = torch.full((rows * (vocab + 7) + 8,), 7.0, device="cuda", dtype=dtype)
        zv = zs[a:a + rows * (vocab + 3)].view(rows, vocab + 3)[:, :vocab]
        gv = gs[b:b + rows * (vocab + 7)].view(rows, vocab + 7)[:, :vocab]
        zv.copy_(z)
        check(call(ops, zv, action, old, adv, ref, w, grad=gv), want, gv, g, g_e)
        gv.fill_(7)
        assert (gs == 7).all()


@pytest.mark.gpu
def test_gradient_is_that_of_differences(ops):
    """Central differences of the loss in its logits, away from the clip's borders: the formula's are
    those of 64 bits, the kernel's gradient stands for it."""
    z, action, old, adv, ref, w = inputs(6, 23, torch.float32, seed=1)
    w[:], adv[3] = 1.0, -0.5
    action[4] = 2
    dz = torch.empty_like(z)
    call(ops, z, action, old, adv, ref, w, T=1.3, beta=0.2, grad=dz)

    def loss(v):
        return formula(v, 1.3, action, old, adv, ref, 0.2, 0.3, 0.2, w)[0]["loss"][0]

    h = 1e-5
    for v in range(23):
        up, down = z.double(), z.double()
        up[:, v] += h
        down[:, v] -= h
        # Terms of the third order: the third derivatives are below 10 here, and 64 bits' rounding / h.
        assert ((loss(up) - loss(down)) / (2 * h) - dz[:, v].double()).abs().max() < 1e-8 + 2e-5 * dz.abs().max()


@pytest.mark.gpu
def test_same_bits_on_a_stream_and_in_a_graph():
    s = torch.cuda.Stream()
    z, action, old, adv, ref, w = inputs(40, 50021, torch.bfloat16)
    dz = torch.zeros_like(z)
    terms = {n: torch.zeros(40, device="cuda") for n in TERMS}
    torch.cuda.synchronize()
    with G.Ops(0, s.cuda_stream) as ops:
        call(ops, z, action, old, adv, ref, w, grad=dz, terms=terms)
        s.synchronize()
        want, want_g = {n: t.clone() for n, t in terms.items()}, dz.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call(ops, z, action, old, adv, ref, w, grad=dz, terms=terms)
        for _ in range(3):
            dz.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(dz, want_g) and all(torch.equal(terms[n], want[n]) for n in TERMS)
        del graph


@pytest.mark.gpu
def test_more_elements_than_32_bits_count(ops):
    rows, vocab = 16500, 131072
    z = torch.zeros(rows, vocab, device="cuda", dtype=torch.bfloat16)
    z[-1, 1::2] = 1.0
    action = torch.full((rows,), vocab - 1, device="cuda", dtype=torch.int32)
    old = torch.full((rows,), -math.log(vocab), device="cuda")
    adv = torch.ones(rows, device="cuda")
    args = (action, old, adv, None, None)
    want, g, g_e, _ = formula(z[-3:], 1.0, *(t[-3:] for t in args[:3]), None, 0.2, 0.3, 0.0, None)
    call(ops, z, *args, beta=0.0, grad=z)
    off = (z[-3:].double() - g).abs() - g_e - g.abs() * 2.0 ** -8
    assert (off <= 0).all()
    assert (z[:-1] == z[0]).all()


def test_refusals():
    """On the host, before any work is queued."""
    L, C = G.lib(), G.C
    z = G.gem_logits(64, 2, 0, 10, G.GEM_F32, 1.0, 0)
    p = G.gem_policy(64, 64, None, 64, 0.2, 0.2, 0.0, 0)
    out = G.gem_policy_terms(64, None, None, None)
    fake = 1 << 20       # never reached

    def grad(z=z, p=p, weight=None, out=out, to=64, stride=0, ops=fake):
        return L.gem_policy_grad(ops, C.byref(z) if z else None, C.byref(p) if p else None, weight,
                                 C.byref(out) if out else None, to, stride)

    assert grad(ops=None) == grad(z=None) == grad(p=None) == grad(to=None) == G.GEM_EINVAL
    assert grad(stride=9) == G.GEM_EINVAL and grad(stride=11) == G.GEM_EINVAL      # over the logits, another stride
    assert grad(to=66) == grad(weight=65) == grad(out=G.gem_policy_terms(64, 65)) == G.GEM_EALIGN
    for k, v in dict(action=None, old_logprob=None, advantage=None, clip_low=1.5, clip_high=math.inf, kl=-1.0).items():
        bad = G.gem_policy(64, 64, None, 64, 0.2, 0.2, 0.0, 0)
        setattr(bad, k, v)
        assert grad(p=bad) == G.GEM_EINVAL, k
        bad = G.gem_policy(64, 64, None, 64, 0.2, 0.2, 0.0, 0)
        setattr(bad, k, math.nan if isinstance(v, float) else 66)
        assert grad(p=bad) == (G.GEM_EINVAL if isinstance(v, float) else G.GEM_EALIGN), k
    assert L.gem_policy_loss(fake, C.byref(z), C.byref(p), None, None) == G.GEM_EINVAL
    assert grad(z=G.gem_logits(64, 2, 0, 10, 5, 1.0, 0)) == G.GEM_EDTYPE
    empty = G.gem_logits(None, 0, 0, 10, G.GEM_F32, 1.0, 0)
    none = G.gem_policy(None, None, None, None, 0.2, 0.2, 0.0, 0)
    assert L.gem_policy_loss(fake, C.byref(empty), C.byref(none), None, C.byref(out)) == G.GEM_OK


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(3, 40), (9, 20011), (300, 515), (258, 140003)])
def test_rows_of_no_numbers_without_advantage(ops, rows, vocab):
    """Their loss is no number, as their gradient is: an advantage of 0 leaves it out of ratios alone."""
    for kl in (True, False):
        for beta in (0.1, 0.0):
            z, action, old, adv, ref, w = inputs(rows, vocab, torch.float32, seed=5)
            action[:], w[:], adv[:] = 7, 1.0, 0.0
            z[0, 5], z[1, 5] = math.nan, math.inf
            dz = torch.empty_like(z)
            for terms in (call(ops, z, action, old, adv, ref if kl else None, w, beta=beta, grad=dz),
                          call(ops, z, action, old, adv, ref if kl else None, w, beta=beta)):
                assert all(terms[n][:2].isnan().all() for n in TERMS if kl or n != "kl")
                assert not any(terms[n][2:].isnan().any() for n in TERMS)
                if not kl or beta == 0:
                    assert (terms["loss"][2:] == 0).all()
            assert dz[:2].isnan().all() and not dz[2:].isnan().any()


def two_tokens(rows, vocab, T, seed=0):
    """Rows of two tokens that can occur: 0 at the last place, and the one that was taken far below it.
    A sum of exponentials is then 1 + p, so that its logarithm is off by little (see near_formula)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.full((rows, vocab), -math.inf, device="cuda")
    z[:, -1] = 0.0
    action = torch.randint(vocab - 1, (rows,), device="cuda", generator=g)
    x = -3.0 - 77.0 * torch.rand(rows, device="cuda", generator=g)
    z.scatter_(1, action[:, None], x[:, None])
    lp = torch.log_softmax(z.double() / T, 1).gather(1, action[:, None])[:, 0]
    old = (lp - 0.1 * torch.randn(rows, device="cuda", generator=g, dtype=torch.float64).clamp(-1.2, 1.2)).float()
    ref = (lp + 0.02 * torch.randn(rows, device="cuda", generator=g, dtype=torch.float64)).float()
    return z, action.to(torch.int32), old, torch.randn(rows, device="cuda", generator=g), ref


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1.0, 0.7, 3.0])
@pytest.mark.parametrize("rows,vocab", [(3, 40), (41, 20011), (300, 515), (258, 140003)])
def test_terms_are_differences_of_64_bits(ops, rows, vocab, T):
    """Ratios and the KL term are differences of logarithms of up to 115 here, whose 32 bits would leave
    errors of 64 units of 2^-24.  The sum is 1 + p: p is off by (8 |x| / T + 16) units (its exponent's
    roundings and the exponentials'), the sum by one more rounding and a half that is its neighbour's;
    differences are those of 64 bits, and each output has up to four roundings of its own.  The temperature is
    the binary32 number that is passed: 0.7 itself is 1.7e-8 of it away, 2e-6 of such a logarithm."""
    T = torch.tensor(T).item()
    z, action, old, adv, ref = two_tokens(rows, vocab, T)
    beta, zd = 0.5, z.double() / T
    at = action.long()[:, None]
    logq = torch.log_softmax(zd, 1)
    lp = logq.gather(1, at)[:, 0]
    p = lp.exp()
    eps = U * (2 + p * (8 * zd.gather(1, at)[:, 0].abs() + 16))
    ratio, gain = (lp - old.double()).exp(), adv.double()
    ratio_e = ratio * (eps + 4 * U)
    d = ref.double() - lp
    kl, grown = torch.expm1(d) - d, torch.expm1(d)
    kl_e = grown.abs() * eps + eps ** 2 + 4 * U * kl
    free, held = ratio * gain, ratio.clamp(0.8, 1.3) * gain
    loss = beta * kl - torch.minimum(free, held)
    loss_e = gain.abs() * ratio_e + beta * kl_e + 4 * U * loss.abs()
    slope = torch.where(free <= held, -free, 0.0) - beta * grown
    slope_e = gain.abs() * ratio_e + beta * (d.exp() * eps + 4 * U * grown.abs()) + 4 * U * slope.abs()
    dz = torch.empty_like(z)
    for terms in (call(ops, z, action, old, adv, ref, None, T, beta=beta),
                  call(ops, z, action, old, adv, ref, None, T, beta=beta, grad=dz)):
        for n, v, e in (("logprob", lp, eps + U * lp.abs()), ("ratio", ratio, ratio_e), ("kl", kl, kl_e), ("loss", loss, loss_e)):
            off = ((terms[n].double() - v).abs() - e).max().item()
            assert off <= 0, (n, off)
    got = dz.gather(1, at)[:, 0].double()
    want = slope / T * (1 - p)
    off = ((got - want).abs() - slope_e / T - want.abs() * 4 * U - (slope / T).abs() * p * U * (8 * zd.gather(1, at)[:, 0].abs() + 16)).max().item()
    assert off <= 0, off
