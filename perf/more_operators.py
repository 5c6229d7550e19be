"""Performance cases of further operators of a language model's workers, through the binding of the
C ABI (``paper_1805_08469_amd.gem``): the way into a model, a layer along its tokens and the loss of
workers that act with a policy that has aged, each with its gradient.

A case is a dict of plain values.  ``op`` says what a pass calls:

  lookup  rows of an embedding for tokens, scaled
  egrad   the embedding's gradient: rows of the same token summed
  ploss   the clipped policy loss with its KL term, of the tokens that were taken
  pgrad   the same with the gradient of the logits
  conv    the short causal convolution of each channel, with its activation
  ctrain  the convolution and its backward pass
  ssm     the selective state space scan, over packed or equal sequences or single tokens
  strain  the scan and its backward pass
"""
from __future__ import annotations

import math
import random

import torch

own = False

F32, BF16 = "f32", "bf16"
_TYPES = {F32: torch.float32, BF16: torch.bfloat16}


def _embed(name, op, count, vocab, dim, dtype, master, pad=0):
    """dtype: of the rows; master: of the table and its gradient; pad: elements between rows."""
    c = dict(op=op, count=count, vocab=vocab, dim=dim, dtype=dtype, master=master, pad=pad)
    if name:
        c["name"] = name
    return c


def _policy(name, op, rows, vocab, dtype, kl=0.05, T=1.0, pad=0, dead=0):
    """dead: columns at the end that are -inf (a vocabulary filled up to a round size)."""
    c = dict(op=op, rows=rows, vocab=vocab, dtype=dtype, kl=kl, T=T, pad=pad, dead=dead)
    if name:
        c["name"] = name
    return c


def _conv(name, op, tokens, seqs, channels, dtype, width=4, ragged=False, pad=0):
    c = dict(op=op, tokens=tokens, seqs=seqs, channels=channels, dtype=dtype, width=width, ragged=ragged, pad=pad)
    if name:
        c["name"] = name
    return c


def _ssm(name, op, tokens, seqs, channels, dtype, state=16, gated=True, ragged=False, pad=0):
    c = dict(op=op, tokens=tokens, seqs=seqs, channels=channels, dtype=dtype, state=state, gated=gated,
             ragged=ragged, pad=pad)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # The rows of 64 answered tokens: latency.
        _embed("lookup-answer", "lookup", 64, 65536, 4096, BF16, F32),
        # A worker's batch on its way into the model, from the parameters' own binary32.
        _embed("lookup-batch", "lookup", 32768, 65536, 2048, BF16, F32),
        # The same batch's gradient, in the type that a commit takes.
        _embed("embed-grad", "egrad", 32768, 65536, 2048, BF16, F32),
        # A small batch, everything in float, odd sizes.
        _embed("embed-grad-few", "egrad", 2047, 50021, 1001, F32, F32),
        # The loss and gradient of a batch of answers, with a KL term to the policy they began from.
        _policy("policy-step", "pgrad", 4096, 32768, BF16),
        # A worker's few answers in float over an odd vocabulary, at the temperature they were drawn at.
        _policy("policy-few", "pgrad", 37, 100003, F32, T=0.7),
        # The convolution of a training step.
        _conv("conv-train", "ctrain", 32768, 8, 2048, BF16),
        # One token for each of 64 sequences.
        _conv("conv-answer", "conv", 64, 64, 4096, BF16),
        # The scan's single token, from states of 16 values a channel.
        _ssm("ssm-answer", "ssm", 64, 64, 4096, BF16),
        # Prompts of unequal lengths, packed.
        _ssm("ssm-prompts", "ssm", 16384, 24, 2048, BF16, ragged=True),
        # A worker's batch: eight sequences of 4096 tokens, forward and backward.
        _ssm("ssm-train", "strain", 32768, 8, 2048, BF16),
        # One long sequence in float, an odd number of channels.
        _ssm("ssm-train-long", "strain", 65537, 1, 1001, F32),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _odd(rng, v):
    return int(v) | 1 if rng.random() < 0.5 else (int(v) + 7) // 8 * 8


MOST_TABLE = 1.4e8       # elements of a drawn case's table, and of its rows
MOST_LOGITS = 1.4e8      # of its logits
MOST_STEPS = 6.5e7       # token-channels


def draw(rng: random.Random):
    op = rng.choice(["lookup", "egrad", "egrad", "ploss", "pgrad", "pgrad", "conv", "ctrain", "ssm", "ssm", "strain",
                     "strain"])
    dtype = rng.choice([BF16, BF16, F32])
    pad = rng.choice([0, 0, 0, 8, 43])
    if op in ("lookup", "egrad"):
        dim = _odd(rng, _log(rng, 64, 8192))
        vocab = int(_log(rng, 500, min(160000.0, MOST_TABLE / dim)))
        count = int(_log(rng, 1, min(131072.0, MOST_STEPS / dim)))
        return _embed("", op, count, vocab, dim, dtype, F32 if dtype == F32 else rng.choice([F32, F32, BF16]), pad=pad)
    if op in ("ploss", "pgrad"):
        vocab = _odd(rng, _log(rng, 2000, 160000))
        rows = int(_log(rng, 1, min(8192.0, MOST_LOGITS / vocab)))
        return _policy("", op, rows, vocab, dtype, kl=rng.choice([0.0, 0.02, 0.1]), T=rng.choice([1.0, 1.0, 0.7, 2.0]),
                       pad=pad, dead=rng.choice([0, 0, 41]))
    channels = _odd(rng, _log(rng, 64, 8192))
    if op in ("conv", "ssm") and rng.random() < 0.4:
        tokens = seqs = int(_log(rng, 1, 512.999))
        ragged = False
    else:
        tokens = int(_log(rng, 16, min(131072.0, MOST_STEPS / channels)))
        seqs = max(1, min(int(_log(rng, 1, 64)), tokens // 8))
        ragged = rng.random() < 0.5
        if not ragged:
            tokens = tokens // seqs * seqs
    if op in ("conv", "ctrain"):
        return _conv("", op, tokens, seqs, channels, dtype, width=rng.choice([2, 3, 4, 4]), ragged=ragged, pad=pad)
    return _ssm("", op, tokens, seqs, channels, dtype, state=rng.choice([16, 16, 16, 8, rng.randint(1, 16)]),
                gated=rng.random() < 0.7, ragged=ragged, pad=pad)


# ---- inputs --------------------------------------------------------------------
def _generator(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + part)
    return g


def _wide(rows, cols, pad, dtype):
    """A [rows, cols] view of rows that are pad elements longer."""
    return torch.zeros(rows, cols + pad, device="cuda", dtype=dtype)[:, :cols]


def _filled(rows, cols, pad, dtype, g, mean=0.0, scale=1.0):
    t = _wide(rows, cols, pad, dtype)
    for at in range(0, rows, 8192):        # a part at a time, so that no float copy of all rows is held
        n = min(8192, rows - at)
        t[at:at + n] = torch.randn(n, cols, device="cuda", generator=g).mul_(scale).add_(mean)
    return t


def _make_embed(case, seed):
    g = _generator(seed, 1)
    count, vocab, dim = case["count"], case["vocab"], case["dim"]
    row, master = _TYPES[case["dtype"]], _TYPES[case["master"]]
    # Frequencies of language: the r-th likeliest token about 1/r times as often as the first.
    rank = torch.rand(count, device="cuda", generator=g, dtype=torch.float64).mul_(math.log(vocab + 1.0)).exp_()
    rank = rank.long().sub_(1).clamp_(0, vocab - 1)
    tok = torch.randperm(vocab, device="cuda", generator=g)[rank]
    tok[13::29] = -1                       # padding
    s = dict(tokens=tok.to(torch.int32), scale=math.sqrt(dim))
    if case["op"] == "lookup":
        s["table"] = _filled(vocab, dim, case["pad"], master, g, scale=0.02)
        s["out"] = _wide(count, dim, case["pad"], row)
    else:
        s["dout"] = _filled(count, dim, case["pad"], row, g, scale=0.01)
        s["grad"] = _wide(vocab, dim, case["pad"], master)
    return s


CLIP_LOW, CLIP_HIGH = 0.2, 0.28


def _make_policy(case, seed):
    g = _generator(seed, 2)
    rows, vocab = case["rows"], case["vocab"]
    z = _wide(rows, vocab, case["pad"], _TYPES[case["dtype"]])
    rank = torch.randperm(vocab, device="cuda", generator=g).float().add_(1.0)
    prior = rank.log_().neg_()
    alive = vocab - case["dead"]
    action = torch.zeros(rows, device="cuda", dtype=torch.int64)
    lp = torch.zeros(rows, device="cuda", dtype=torch.float64)
    for at in range(0, rows, 512):
        n = min(512, rows - at)
        part = z[at:at + n]
        part.copy_(torch.randn(n, vocab, device="cuda", generator=g).mul_(1.8).add_(prior))
        part[:, alive:] = -math.inf
        v = part.float() / case["T"]
        noise = torch.rand(n, vocab, device="cuda", generator=g).clamp_(1e-20).log_().neg_().log_().neg_()
        a = (v + noise).argmax(1)          # drawn from the policy
        action[at:at + n] = a
        lp[at:at + n] = v.gather(1, a[:, None])[:, 0].double() - v.double().logsumexp(1)
    # The behaviour policy is an older one: ratios about 1, some outside what is left unclipped;
    # none within the rounding of a border, where the gradient jumps.
    shift = torch.randn(rows, device="cuda", generator=g, dtype=torch.float64).mul_(0.2)
    for border in (math.log(1.0 - CLIP_LOW), math.log(1.0 + CLIP_HIGH)):
        near = (shift - border).abs() < 2e-3
        shift = torch.where(near, border + 4e-3, shift)
    s = dict(z=z, old=(lp - shift).float())
    s["ref"] = (lp + torch.randn(rows, device="cuda", generator=g, dtype=torch.float64).mul_(0.3)).float()
    s["advantage"] = torch.randn(rows, device="cuda", generator=g)
    w = torch.full((rows,), 1.0 / rows, device="cuda")
    w[7::8] = 0.0                          # prompts carry no loss
    action[11::16] = -1                    # padding
    s["w"], s["action"] = w, action.to(torch.int32)
    for n in ("loss", "logprob", "ratio", "klterm"):
        s[n] = torch.zeros(rows, device="cuda")
    if case["op"] == "pgrad":
        s["dz"] = _wide(rows, vocab, case["pad"], _TYPES[case["dtype"]])
    return s


def _lengths(case, seed):
    """Offsets of the sequences: equal lengths, or cuts at random places with an empty sequence
    and one of a single token among them."""
    tokens, seqs = case["tokens"], case["seqs"]
    if not case["ragged"]:
        return [tokens // seqs * i for i in range(seqs + 1)]
    r = random.Random(1000003 * int(seed) + 3)
    cuts = sorted(r.randint(0, tokens) for _ in range(seqs - 1))
    if seqs >= 4:
        cuts[1] = cuts[0]
        cuts[-1] = tokens - 1
        cuts.sort()
    return [0] + cuts + [tokens]


def _make_conv(case, seed):
    g = _generator(seed, 4)
    n, S, D, W, pad, dt = (case["tokens"], case["seqs"], case["channels"], case["width"], case["pad"],
                           _TYPES[case["dtype"]])
    off = _lengths(case, seed)
    s = dict(x=_filled(n, D, pad, dt, g), before=torch.randn(S, W - 1, D, device="cuda", generator=g).to(dt))
    s["weight"] = torch.randn(D, W, device="cuda", generator=g).mul_(0.5)
    s["bias"] = torch.randn(D, device="cuda", generator=g).mul_(0.1)
    s["off"] = torch.tensor(off, device="cuda", dtype=torch.int64)
    s["y"], s["last"] = _wide(n, D, pad, dt), torch.zeros(S, W - 1, D, device="cuda", dtype=dt)
    if case["op"] == "ctrain":
        s["dy"] = _filled(n, D, pad, dt, g, scale=0.01)
        s["dx"] = _wide(n, D, pad, dt)
        s["dweight"], s["dbias"] = torch.zeros(D, W, device="cuda"), torch.zeros(D, device="cuda")
    return s


def _make_ssm(case, seed):
    g = _generator(seed, 5)
    n, S, D, N, pad, dt = (case["tokens"], case["seqs"], case["channels"], case["state"], case["pad"],
                           _TYPES[case["dtype"]])
    off = _lengths(case, seed)
    s = dict(x=_filled(n, D, pad, dt, g), dt=_filled(n, D, pad, dt, g, scale=0.7), b=_filled(n, N, pad, dt, g),
             c=_filled(n, N, pad, dt, g), z=_filled(n, D, pad, dt, g) if case["gated"] else None)
    # Steps from a thousandth to a tenth, decays of 1 to N a unit of them.
    step = torch.rand(D, device="cuda", generator=g).mul_(math.log(100.0)).add_(math.log(1e-3)).exp_()
    s["dt_bias"] = step + torch.log(-torch.expm1(-step))
    rate = torch.arange(1, N + 1, device="cuda", dtype=torch.float32).repeat(D, 1)
    s["a"] = -rate * torch.randn(D, N, device="cuda", generator=g).mul_(0.1).exp_()
    s["d"] = torch.randn(D, device="cuda", generator=g).mul_(0.1).add_(1.0)
    s["h0"] = torch.randn(S, D, N, device="cuda", generator=g).mul_(0.3)
    s["off"] = torch.tensor(off, device="cuda", dtype=torch.int64)
    s["longest"] = max(q - p for p, q in zip(off, off[1:]))
    s["y"], s["h_last"] = _wide(n, D, pad, dt), torch.zeros(S, D, N, device="cuda")
    if case["op"] == "strain":
        s["dy"] = _filled(n, D, pad, dt, g, scale=0.01)
        s["dh_last"] = torch.randn(S, D, N, device="cuda", generator=g).mul_(0.01)
        for name in ("dx", "ddt") + (("dz",) if case["gated"] else ()):
            s[name] = _wide(n, D, pad, dt)
        s["db"], s["dc"] = _wide(n, N, pad, dt), _wide(n, N, pad, dt)
        s["da"], s["dh0"] = torch.zeros(D, N, device="cuda"), torch.zeros(S, D, N, device="cuda")
        s["dd"], s["ddt_bias"] = torch.zeros(D, device="cuda"), torch.zeros(D, device="cuda")
    return s


def prepare(case, seed):
    op = case["op"]
    make = {"lookup": _make_embed, "egrad": _make_embed, "ploss": _make_policy, "pgrad": _make_policy,
            "conv": _make_conv, "ctrain": _make_conv, "ssm": _make_ssm, "strain": _make_ssm}[op]
    s = make(case, seed)
    s["case"] = case
    if own:                                # the handle such a program keeps, and its scratch
        from paper_1805_08469_amd import gem as G
        scratch = 0
        if op == "egrad":
            scratch = G.gem_embed_scratch(case["count"], case["vocab"], case["dim"])
        elif op == "ctrain":
            scratch = G.gem_conv_scratch(case["tokens"], case["channels"])
        elif op in ("ssm", "strain"):
            scratch = G.gem_ssm_scratch(case["tokens"], case["channels"], case["state"])
        s["ops"] = G.Ops(scratch, torch.cuda.current_stream().cuda_stream)
        if op == "strain":
            s["states"] = torch.zeros(G.gem_ssm_state_rows(case["tokens"]), case["channels"], case["state"],
                                      device="cuda")
    return s


# ---- the plain forms -------------------------------------------------------------
def _plain_lookup(s):
    tok = s["tokens"].long()
    have = tok >= 0
    r = s["table"][torch.where(have, tok, torch.zeros_like(tok))].float() * s["scale"]
    return dict(out=torch.where(have[:, None], r, torch.zeros_like(r)).to(_TYPES[s["case"]["dtype"]]))


def _plain_egrad(s):
    case = s["case"]
    tok = s["tokens"].long()
    r = s["dout"].float() * s["scale"]
    # Padding goes to a row of its own.
    total = torch.zeros(case["vocab"] + 1, case["dim"], device=r.device)
    total.index_add_(0, torch.where(tok >= 0, tok, case["vocab"]), r)
    return dict(grad=total[:-1].to(_TYPES[case["master"]]))


def _plain_policy(s):
    case, T = s["case"], s["case"]["T"]
    z = s["z"].float() / T
    e = z - z.amax(1, keepdim=True)
    at = s["action"].long()
    live = (at >= 0) & (s["w"] != 0)
    at = torch.where(at >= 0, at, torch.zeros_like(at))[:, None]
    picked = e.gather(1, at)[:, 0].double()
    e = e.exp_()
    total = e.sum(1, keepdim=True)
    # Ratios and the KL term are differences of logarithms: in 64 bits.
    lp = picked - total[:, 0].double().log()
    ratio = (lp - s["old"]).exp()
    adv = s["advantage"].double()
    free, held = ratio * adv, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * adv
    gap = s["ref"].double() - lp
    kl = torch.expm1(gap) - gap
    loss = case["kl"] * kl - torch.minimum(free, held)
    zero = torch.zeros_like(loss)
    r = {n: torch.where(live, v, zero).float() for n, v in (("loss", loss), ("logprob", lp), ("ratio", ratio), ("kl", kl))}
    if case["op"] == "pgrad":
        slope = torch.where(free <= held, -free, zero) - case["kl"] * torch.expm1(gap)
        slope = torch.where(live, slope * s["w"] / T, zero).float()[:, None]
        g = e.mul_(-slope / total)
        g.scatter_add_(1, at, slope)
        r["dz"] = torch.where(live[:, None], g, torch.zeros_like(g)).to(s["z"].dtype)
    return r


def _places(s, W):
    """Rows of [x; before] that the taps of each token read, and those that stay behind a sequence."""
    off, n = s["off"], s["case"]["tokens"]
    S = off.numel() - 1
    t = torch.arange(n, device=off.device)
    q = torch.searchsorted(off[1:], t, right=True)
    begin = off[:-1][q]
    taps = []
    for j in range(W):
        src = t - (W - 1) + j
        taps.append(torch.where(src >= begin, src, n + q * (W - 1) + src - begin + (W - 1)))
    i = torch.arange(W - 1, device=off.device)[None]
    ext = (off[1:] - off[:-1])[:, None] + i                  # of the W - 1 earlier inputs and the sequence
    seq = torch.arange(S, device=off.device)[:, None]
    keep = torch.where(ext >= W - 1, off[:-1][:, None] + ext - (W - 1), n + seq * (W - 1) + ext)
    return taps, keep


def _plain_conv(s):
    case, W, D = s["case"], s["case"]["width"], s["case"]["channels"]
    taps, keep = _places(s, W)
    e = torch.cat([s["x"].float(), s["before"].float().reshape(-1, D)])
    c = s["bias"].expand(case["tokens"], D)
    for j in range(W):
        c = c + e[taps[j]] * s["weight"][:, j]
    gate = 1.0 / (1.0 + (-c).exp())
    r = dict(y=(c * gate).to(s["x"].dtype), last=e[keep].to(s["x"].dtype))
    if case["op"] == "ctrain":
        g = s["dy"].float() * gate * (1.0 + c * (1.0 - gate))
        de = torch.zeros_like(e)
        dw = []
        for j in range(W):
            de.index_add_(0, taps[j], g * s["weight"][:, j])  # no row twice
            dw.append((g * e[taps[j]]).sum(0))
        r.update(dx=de[:case["tokens"]].to(s["x"].dtype), dweight=torch.stack(dw, 1), dbias=g.sum(0))
    return r


def _scanned(a, b, longest):
    """h_t = a_t h_{t-1} + b_t down the rows, by doubling."""
    step = 1
    while step < longest:
        b[step:] = b[step:] + a[step:] * b[:-step]
        a[step:] = a[step:] * a[:-step]
        step *= 2
    return b


def _plain_ssm(s):
    case, off = s["case"], s["off"]
    x, B, C = s["x"].float(), s["b"].float(), s["c"].float()
    v = s["dt"].float() + s["dt_bias"]
    delta = v.clamp(min=0) + torch.log1p((-v.abs()).exp())
    full = off[1:] > off[:-1]
    first, last, of = off[:-1][full], off[1:][full] - 1, full.nonzero()[:, 0]
    a = (delta[:, :, None] * s["a"]).exp()
    h = (delta * x)[:, :, None] * B[:, None, :]
    h[first] += a[first] * s["h0"][of]
    w = a.clone()
    w[first] = 0.0
    h = _scanned(w, h, s["longest"])
    h_last = s["h0"].clone()
    h_last[of] = h[last]
    bare = (h * C[:, None, :]).sum(2) + s["d"] * x
    if case["gated"]:
        z = s["z"].float()
        gate = 1.0 / (1.0 + (-z).exp())
        r = dict(y=(bare * z * gate).to(s["x"].dtype), h_last=h_last)
    else:
        r = dict(y=bare.to(s["x"].dtype), h_last=h_last)
    if case["op"] != "strain":
        return r
    dy = s["dy"].float()
    if case["gated"]:
        r["dz"] = (dy * bare * gate * (1.0 + z * (1.0 - gate))).to(s["x"].dtype)
        dy = dy * z * gate
    # dh_t = C_t dy_t + a_{t+1} dh_{t+1}: the same recurrence from the right.
    g = dy[:, :, None] * C[:, None, :]
    g[last] += s["dh_last"][of]
    w = torch.cat([a[1:], torch.zeros_like(a[:1])])
    w[last] = 0.0
    g = _scanned(w.flip(0), g.flip(0), s["longest"]).flip(0)
    del w
    r["dc"] = (dy[:, :, None] * h).sum(1).to(s["x"].dtype)
    r["db"] = ((delta * x)[:, :, None] * g).sum(1).to(s["x"].dtype)
    p = (g * B[:, None, :]).sum(2)
    r["dx"] = (s["d"] * dy + delta * p).to(s["x"].dtype)
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    before[first] = s["h0"][of]
    r["dh0"] = s["dh_last"].clone()
    r["dh0"][of] = a[first] * g[first]
    q = a.mul_(g).mul_(before)
    ddelta = p * x + (q * s["a"]).sum(2)
    ddt = ddelta / (1.0 + (-v).exp())
    r.update(ddt=ddt.to(s["x"].dtype), da=(q * delta[:, :, None]).sum(0), dd=(dy * x).sum(0), ddt_bias=ddt.sum(0))
    return r


# ---- one pass --------------------------------------------------------------------
def _at(t):
    return t.data_ptr() if t is not None else None


def run(s):
    case, op = s["case"], s["case"]["op"]
    if not own:
        return {"lookup": _plain_lookup, "egrad": _plain_egrad, "ploss": _plain_policy, "pgrad": _plain_policy,
                "conv": _plain_conv, "ctrain": _plain_conv, "ssm": _plain_ssm, "strain": _plain_ssm}[op](s)
    ops, kind = s["ops"], 1 if case["dtype"] == BF16 else 0
    if op in ("lookup", "egrad"):
        master = 1 if case["master"] == BF16 else 0
        tok = s["tokens"].data_ptr()
        if op == "lookup":
            ops.embed_forward(s["table"].data_ptr(), tok, case["count"], case["vocab"], case["dim"], master,
                              out=s["out"].data_ptr(), out_dtype=kind, scale=s["scale"], stride=s["table"].stride(0),
                              out_stride=s["out"].stride(0))
            return dict(out=s["out"])
        ops.embed_backward(tok, case["count"], case["vocab"], case["dim"], master, dout=s["dout"].data_ptr(),
                           dout_dtype=kind, grad=s["grad"].data_ptr(), scale=s["scale"],
                           dout_stride=s["dout"].stride(0), grad_stride=s["grad"].stride(0))
        return dict(grad=s["grad"])
    if op in ("ploss", "pgrad"):
        z = s["z"]
        args = dict(action=s["action"].data_ptr(), old_logprob=s["old"].data_ptr(),
                    advantage=s["advantage"].data_ptr(), ref_logprob=s["ref"].data_ptr(), clip_low=CLIP_LOW,
                    clip_high=CLIP_HIGH, kl_coef=case["kl"], stride=z.stride(0), temperature=case["T"],
                    weight=s["w"].data_ptr(), loss=s["loss"].data_ptr(), logprob=s["logprob"].data_ptr(),
                    ratio=s["ratio"].data_ptr(), kl=s["klterm"].data_ptr())
        r = dict(loss=s["loss"], logprob=s["logprob"], ratio=s["ratio"], kl=s["klterm"])
        if op == "ploss":
            ops.policy_loss(z.data_ptr(), case["rows"], case["vocab"], kind, **args)
            return r
        ops.policy_grad(z.data_ptr(), case["rows"], case["vocab"], kind, grad=s["dz"].data_ptr(),
                        grad_stride=s["dz"].stride(0), **args)
        return dict(r, dz=s["dz"])
    row, off = s["x"].stride(0), s["off"].data_ptr() if case["ragged"] else None
    if op in ("conv", "ctrain"):
        args = dict(bias=s["bias"].data_ptr(), before=s["before"].data_ptr(), offsets=off, act=1, x_stride=row)
        sizes = case["tokens"], case["channels"], case["seqs"], case["width"], kind
        x, w = s["x"].data_ptr(), s["weight"].data_ptr()
        ops.conv_forward(x, w, *sizes, y=s["y"].data_ptr(), last=s["last"].data_ptr(), y_stride=row, **args)
        r = dict(y=s["y"], last=s["last"])
        if op == "ctrain":
            ops.conv_backward(x, w, *sizes, dy=s["dy"].data_ptr(), dx=s["dx"].data_ptr(),
                              dweight=s["dweight"].data_ptr(), dbias=s["dbias"].data_ptr(), dy_stride=row,
                              dx_stride=row, **args)
            r.update(dx=s["dx"], dweight=s["dweight"], dbias=s["dbias"])
        return r
    inputs = [s[n].data_ptr() for n in ("x", "dt", "b", "c", "a")]
    sizes = case["tokens"], case["channels"], case["state"], case["seqs"], kind
    short = s["b"].stride(0)
    args = dict(z=_at(s["z"]), d=s["d"].data_ptr(), dt_bias=s["dt_bias"].data_ptr(), h0=s["h0"].data_ptr(), offsets=off,
                x_stride=row, dt_stride=row, z_stride=row, b_stride=short, c_stride=short)
    states = s["states"].data_ptr() if op == "strain" else None
    ops.ssm_forward(*inputs, *sizes, y=s["y"].data_ptr(), h_last=s["h_last"].data_ptr(), states=states, y_stride=row,
                    **args)
    r = dict(y=s["y"], h_last=s["h_last"])
    if op == "strain":
        names = ("dx", "ddt", "db", "dc", "da", "dd", "ddt_bias", "dh0") + (("dz",) if case["gated"] else ())
        ops.ssm_backward(*inputs, *sizes, states=states, dy=s["dy"].data_ptr(), dh_last=s["dh_last"].data_ptr(),
                         dy_stride=row, dx_stride=row, ddt_stride=row, dz_stride=row, db_stride=short, dc_stride=short,
                         **{n: s[n].data_ptr() for n in names}, **args)
        r.update({n: s[n] for n in names})
    return r


def work(case):
    op, size = case["op"], 2 if case["dtype"] == BF16 else 4
    if op in ("lookup", "egrad"):
        n, master = case["count"] * case["dim"], 2 if case["master"] == BF16 else 4
        if op == "lookup":
            # Rows that are looked up often are read once: by frequencies of 1/r, the distinct ones.
            V = case["vocab"]
            h = math.log(V + 1.0)
            distinct = sum(1.0 - (1.0 - math.log1p(1.0 / r) / h) ** case["count"] for r in range(1, V + 1))
            return dict(bytes=n * size + distinct * case["dim"] * master + 4 * case["count"], flops=n)
        return dict(bytes=n * size + case["vocab"] * case["dim"] * master + 4 * case["count"], flops=n)
    if op in ("ploss", "pgrad"):
        n, rows = case["rows"] * case["vocab"], case["rows"]
        read = sum(1 for r in range(rows) if r % 8 != 7 and r % 16 != 11)
        by = read * case["vocab"] * size + 36 * rows
        return dict(bytes=by + (n * size if op == "pgrad" else 0), flops=(7 if op == "pgrad" else 4) * n)
    n, D, S = case["tokens"] * case["channels"], case["channels"], case["seqs"]
    if op in ("conv", "ctrain"):
        W = case["width"]
        ends, weights = 2 * S * (W - 1) * D * size, 4 * D * (W + 1)
        if op == "conv":
            return dict(bytes=2 * n * size + ends + weights, flops=(2 * W + 5) * n)
        return dict(bytes=5 * n * size + ends + 3 * weights, flops=(8 * W + 16) * n)
    N, wide = case["state"], 4 if case["gated"] else 3
    ends, short, weights = 8 * S * D * N, 2 * case["tokens"] * N * size, 4 * D * (N + 2)
    # A step of one state: its decay, an exponential, what comes in, and its part of the output.
    if op == "ssm":
        return dict(bytes=wide * n * size + short + ends + weights, flops=(7 * N + 20) * n)
    # Backward reads the inputs and dy, and writes a gradient for each; a step of one state takes its
    # gradient on (3), its parts of the four sums over channels and states (8) and that of A (3).
    back = (2 * wide - 1) * n * size + 2 * short + ends + 2 * weights
    return dict(bytes=wide * n * size + short + ends + weights + back, flops=(21 * N + 60) * n)


# ---- the definitions in 64 bits -----------------------------------------------------
def _exact_embed(case, s):
    tok = s["tokens"].tolist()
    if case["op"] == "lookup":
        out = torch.zeros(case["count"], case["dim"], device="cuda", dtype=torch.float64)
        at = [i for i, v in enumerate(tok) if v >= 0]
        if at:
            rows = torch.tensor([tok[i] for i in at], device="cuda")
            out[torch.tensor(at, device="cuda")] = s["table"].double()[rows] * s["scale"]
        return dict(out=out)
    # Rows of one token stand together, and each group is summed by itself.
    groups = {}
    for i, v in enumerate(tok):
        if v >= 0:
            groups.setdefault(v, []).append(i)
    grad = torch.zeros(case["vocab"], case["dim"], device="cuda", dtype=torch.float64)
    alone = [(v, m[0]) for v, m in groups.items() if len(m) == 1]
    if alone:
        grad[torch.tensor([v for v, _ in alone], device="cuda")] = \
            s["dout"][torch.tensor([i for _, i in alone], device="cuda")].double()
    for v, m in groups.items():
        if len(m) > 1:
            grad[v] = s["dout"][torch.tensor(m, device="cuda")].double().sum(0)
    return dict(grad=grad.mul_(s["scale"]))


def _exact_policy(case, s):
    rows, vocab, T = case["rows"], case["vocab"], case["T"]
    r = {n: torch.zeros(rows, device="cuda", dtype=torch.float64) for n in ("loss", "logprob", "ratio", "kl")}
    if case["op"] == "pgrad":
        r["dz"] = torch.zeros(rows, vocab, device="cuda", dtype=torch.float64)
    action, weight = s["action"].tolist(), s["w"].tolist()
    rest = [v.double() for v in (s["old"], s["ref"], s["advantage"], s["w"])]
    live = [i for i in range(rows) if weight[i] != 0.0 and 0 <= action[i] < vocab]
    for k in range(0, len(live), 256):
        at = torch.tensor(live[k:k + 256], device="cuda")
        old, ref, adv, w = (v[at] for v in rest)
        logits = s["z"][at].double().requires_grad_()
        logp = torch.log_softmax(logits / T, dim=1)
        lp = logp[torch.arange(at.numel(), device="cuda"), s["action"][at].long()]
        ratio = torch.exp(lp - old)
        kl = torch.exp(ref - lp) - 1.0 - (ref - lp)
        # What a clipped ratio gives does not depend on the logits.
        up, down = ratio > 1.0 + CLIP_HIGH, ratio < 1.0 - CLIP_LOW
        held = torch.where(adv >= 0, up, down)
        edge = torch.where(adv >= 0, 1.0 + CLIP_HIGH, 1.0 - CLIP_LOW)
        gain = adv * torch.where(held, edge, ratio)
        loss = case["kl"] * kl - gain
        for n, v in (("loss", loss), ("logprob", lp), ("ratio", ratio), ("kl", kl)):
            r[n][at] = v.detach()
        if "dz" in r:
            (loss * w).sum().backward()
            r["dz"][at] = logits.grad
    return r


def _exact_conv(case, s):
    W, train = case["width"], case["op"] == "ctrain"
    w = s["weight"].double().requires_grad_()
    bias = s["bias"].double().requires_grad_()
    x = s["x"].double().requires_grad_()
    off = s["off"].tolist()
    ys, last = [], []
    for q, (lo, hi) in enumerate(zip(off, off[1:])):
        e = torch.cat([s["before"][q].double(), x[lo:hi]])
        last.append(e.detach()[hi - lo:])
        if hi > lo:
            c = torch.stack([e[j:j + hi - lo] * w[:, j] for j in range(W)]).sum(0) + bias
            ys.append(torch.nn.functional.silu(c))
    y = torch.cat(ys)
    r = dict(y=y.detach(), last=torch.stack(last))
    if train:
        r["dx"], r["dweight"], r["dbias"] = torch.autograd.grad((y * s["dy"].double()).sum(), [x, w, bias])
    return r


def _exact_ssm(case, s):
    """Token after token, in each sequence by itself."""
    n, D, N, train = case["tokens"], case["channels"], case["state"], case["op"] == "strain"
    x, B, C, A, skip = (s[k].double() for k in ("x", "b", "c", "a", "d"))
    v = s["dt"].double() + s["dt_bias"].double()
    delta = torch.logaddexp(v, torch.zeros_like(v))
    keep = torch.exp(delta.unsqueeze(2) * A)
    H = (delta * x).unsqueeze(2) * B.unsqueeze(1)            # the states take its place
    before = torch.empty_like(H) if train else None
    off = s["off"].tolist()
    if case["ragged"]:
        groups = [(slice(q, q + 1), slice(lo, hi), (1, hi - lo)) for q, (lo, hi) in enumerate(zip(off, off[1:])) if hi > lo]
    else:
        groups = [(slice(0, case["seqs"]), slice(0, n), (case["seqs"], n // case["seqs"]))]
    h_last = s["h0"].double()
    for which, rows, lead in groups:
        k, hh = keep[rows].view(*lead, D, N), H[rows].view(*lead, D, N)
        h = h_last[which].clone()
        if train:
            before[rows].view(*lead, D, N)[:, 0] = h
        for t in range(lead[1]):
            h = torch.addcmul(hh[:, t], k[:, t], h, out=hh[:, t])
        h_last[which] = h
        if train:
            before[rows].view(*lead, D, N)[:, 1:] = hh[:, :-1]
    bare = torch.matmul(H, C.unsqueeze(2)).squeeze(2) + skip * x
    z = s["z"].double() if case["gated"] else None
    r = dict(y=bare * torch.nn.functional.silu(z) if case["gated"] else bare, h_last=h_last)
    if not train:
        return r
    dy = s["dy"].double()
    if case["gated"]:
        sig = torch.sigmoid(z)
        r["dz"] = dy * bare * (sig + z * sig * (1.0 - sig))
        dy = dy * (z * sig)
    r["dc"] = torch.matmul(dy.unsqueeze(1), H).squeeze(1)
    G = H
    torch.mul(dy.unsqueeze(2), C.unsqueeze(1), out=G)        # and now their gradients'
    dh0 = s["dh_last"].double()
    for which, rows, lead in groups:
        k, g = keep[rows].view(*lead, D, N), G[rows].view(*lead, D, N)
        e = dh0[which].clone()
        for t in range(lead[1] - 1, -1, -1):
            now = g[:, t].add_(e)
            e = torch.mul(k[:, t], now, out=e)
        dh0[which] = e
    r["dh0"] = dh0
    r["db"] = torch.matmul((delta * x).unsqueeze(1), G).squeeze(1)
    into = torch.matmul(G, B.unsqueeze(2)).squeeze(2)
    r["dx"] = skip * dy + delta * into
    r["dd"] = (dy * x).sum(0)
    flow = before.mul_(keep).mul_(G)
    ddt = (x * into + (flow * A).sum(2)) * torch.sigmoid(v)
    r.update(ddt=ddt, ddt_bias=ddt.sum(0), da=flow.mul_(delta.unsqueeze(2)).sum(0))
    return r


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("lookup", "egrad"):
        return _exact_embed(case, s)
    if op in ("ploss", "pgrad"):
        return _exact_policy(case, s)
    return _exact_conv(case, s) if op in ("conv", "ctrain") else _exact_ssm(case, s)
