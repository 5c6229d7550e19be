"""The worker's operators where values leave the ordinary: records without mass, tails far below
the listed tokens, masks of any size, NaN, and what every call has to leave behind."""
import math

import numpy as np
import pytest

import ops_reference as R
from test_gpu_ops import DT, G, INF, _check_distill, _check_scores, _host, _matrix, _same, _score, _teacher, torch  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- masks -----------------------------------------------------------------------
MASKS = [-1e9, -3e9, -1e10, -7e12, -1e30, -3e35]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 20001, 150001])
def test_scores_of_rows_masked_by_any_finite_value(torch, G, V, dt):
    """Whole threads, parts and rows of logits far below the others, where no multiple of a
    logit is exact any more."""
    rng = np.random.default_rng(V)
    for T in (1.0, 0.5):
        z = rng.normal(size=(4 * len(MASKS), V)) * 2
        for i, m in enumerate(MASKS):
            z[4 * i, :V // 2] = m
            z[4 * i + 1, V // 3:] = m
            z[4 * i + 2, np.arange(V) != V - 2] = m
            z[4 * i + 3, :] = m
        _check_scores(torch, G, z, dt, T=T, k=8, n=3, what=f"masked T={T}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(24, 700), (24, 20001), (24, 150001), (288, 5001), (264, 40001)])
def test_distill_of_rows_masked_by_any_finite_value(torch, G, rows, V, dt):
    rng = np.random.default_rng(V + rows)
    ids, lp = _teacher(rng, rows, V, 16)
    values = rng.normal(size=(rows, V)) * 2
    free = np.ones((rows, V), bool)
    for i in range(rows):
        if i % 4 == 0:
            free[i, :V // 2] = False
        elif i % 4 == 1:
            free[i, V // 3:] = False
        elif i % 4 == 2:
            free[i, rng.random(V) < 0.9] = False
        free[i, ids[i]] = True
        values[i, ~free[i]] = MASKS[i // 4 % len(MASKS)]
        if i % 24 == 3:
            values[i, :] = MASKS[i // 24 % len(MASKS)]
    z, _ = _matrix(torch, values, dt)
    ti, tl = torch.from_numpy(ids).cuda(), torch.from_numpy(lp).cuda()
    loss, loss2 = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    g = torch.zeros(rows, V, device="cuda", dtype=z.dtype)
    print(f"[distill] masked rows={rows} V={V} {dt}", flush=True)
    args = dict(ids=ti.data_ptr(), teacher=tl.data_ptr(), k=16, tail=0, temperature=0.5)
    with G.Ops() as ops:
        ops.distill_loss(z.data_ptr(), rows, V, DT[dt], loss=loss.data_ptr(), **args)
        ops.distill_grad(z.data_ptr(), rows, V, DT[dt], loss=loss2.data_ptr(), grad=g.data_ptr(), **args)
        torch.cuda.synchronize()
    host, got, got2, grad = _host(z), _host(loss), _host(loss2), _host(g)
    for r in range(rows):
        lo, gr, q, p, pt, qt = R.distill_row(host[r], 0.5, ids[r], lp[r], 0)
        # A masked logit's distance from the others is a difference that rounds once and that
        # nothing is read from: the spread that enters the bounds is that of the free ones.
        level = np.where(free[r], host[r], -INF) if r % 24 != 3 else np.zeros(V)
        lt, gt = R.distill_tolerance(V, 16, 0.5, level, q, p, pt, qt, lo, gr, 1.0, dt == "bf16")
        _same(got[r:r + 1], np.array([lo]), lt, f"loss of row {r}")
        _same(got2[r:r + 1], np.array([lo]), lt, f"loss (with gradient) of row {r}")
        _same(grad[r], gr, gt, f"gradient of row {r}")


# ---- what a record holds ------------------------------------------------------------
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(6, 40), (3, 90001), (300, 3001)])
def test_distill_rows_without_entries_have_no_gradient(torch, G, rows, V, dt):
    """Their loss is 0 whatever the logits are."""
    rng = np.random.default_rng(21)
    ids, lp = _teacher(rng, rows, V, 7)
    ids[::3] = -1
    ids[1::3] = V
    lp[2::3] = -INF
    z, _ = _matrix(torch, rng.normal(size=(rows, V)), dt)
    ti, tl = torch.from_numpy(ids).cuda(), torch.from_numpy(lp).cuda()
    for tail in (0, 1):
        loss, g = torch.full((rows,), 55.0, device="cuda"), torch.full((rows, V), 33.0, device="cuda", dtype=z.dtype)
        with G.Ops() as ops:
            ops.distill_grad(z.data_ptr(), rows, V, DT[dt], ids=ti.data_ptr(), teacher=tl.data_ptr(), k=7, tail=tail,
                             loss=loss.data_ptr(), grad=g.data_ptr())
            torch.cuda.synchronize()
        empty = slice(None) if tail == 0 else [r for r in range(rows) if r % 3 != 2]
        # with a tail all mass is the tail's, and its gradient is q (1 - 1 / 1)
        assert float(loss[empty].abs().max()) <= (0 if tail == 0 else 4 * R.U)
        assert float(g[empty].float().abs().max()) <= (0 if tail == 0 else 8 * R.U)


@pytest.mark.parametrize("over", [1.05, 1.5])
def test_distill_gradient_of_records_of_any_mass_against_differences(torch, G, over):
    """Probabilities that sum to more than 1, against central differences of the loss in 64 bits."""
    rng = np.random.default_rng(22)
    V, step = 29, 1e-5
    ids, lp = _teacher(rng, 1, V, 6, mass=over)
    z = (rng.normal(size=(1, V))).astype(np.float32).astype(np.float64)
    zt, _ = _matrix(torch, z, "f32")
    g = torch.zeros(1, V, device="cuda")
    ti, tl = torch.from_numpy(ids).cuda(), torch.from_numpy(lp).cuda()
    with G.Ops() as ops:
        ops.distill_grad(zt.data_ptr(), 1, V, 0, ids=ti.data_ptr(), teacher=tl.data_ptr(), k=6, tail=1, grad=g.data_ptr())
        torch.cuda.synchronize()

    def loss(z):
        e = np.exp(z - z.max())
        logq = np.log(e / e.sum())[ids[0]]
        return float((np.exp(lp[0].astype(np.float64)) * (lp[0] - logq)).sum())

    for v in range(V):
        hi, lo = z[0].copy(), z[0].copy()
        hi[v] += step
        lo[v] -= step
        d = (loss(hi) - loss(lo)) / (2 * step)
        assert abs(d - float(g[0, v])) < 2e-5 * max(abs(d), 0.05), v


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("rows,V", [(5, 60), (2, 90001), (300, 3001)])
def test_distill_of_records_with_a_nan_is_nan(torch, G, rows, V, tail):
    """A broken record shows in its row's loss and gradient, and in no other's."""
    rng = np.random.default_rng(23)
    ids, lp = _teacher(rng, rows, V, 5)
    lp[1, 2] = np.nan
    z, _ = _matrix(torch, rng.normal(size=(rows, V)), "f32")
    ti, tl = torch.from_numpy(ids).cuda(), torch.from_numpy(lp).cuda()
    loss, loss2 = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    g = torch.zeros(rows, V, device="cuda")
    args = dict(ids=ti.data_ptr(), teacher=tl.data_ptr(), k=5, tail=tail)
    with G.Ops() as ops:
        ops.distill_loss(z.data_ptr(), rows, V, 0, loss=loss.data_ptr(), **args)
        ops.distill_grad(z.data_ptr(), rows, V, 0, loss=loss2.data_ptr(), grad=g.data_ptr(), **args)
        torch.cuda.synchronize()
    for out in (loss, loss2, g[:, 0], g[:, V - 1]):
        assert torch.isnan(out).tolist() == [r == 1 for r in range(rows)]
    assert bool(torch.isnan(g[1]).all())


# ---- the tail -----------------------------------------------------------------------
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(8, 50), (8, 9001), (3, 90001), (280, 3001), (264, 40001), (258, 70001)])
@pytest.mark.parametrize("gap,T", [(60.0, 1.0), (80.0, 1.0), (90.0, 1.0), (100.0, 1.0), (200.0, 1.0), (10.0, 0.05),
                                   (600.0, 1.0)])
def test_distill_tail_far_below_the_listed_tokens(torch, G, rows, V, gap, T, dt):
    """Unlisted logits so far down that their exponentials, taken about the listed ones, are
    nothing in 32 bits."""
    rng = np.random.default_rng(int(gap) + V)
    ids, lp = _teacher(rng, rows, V, 6)
    z = rng.normal(size=(rows, V))
    for r in range(rows):
        z[r, ids[r, :1 + r % 6]] += gap
    _check_distill(torch, G, z, ids, lp, dt, T=T, tail=1, what=f"gap {gap}")
    if rows < 9:
        _check_distill(torch, G, z, ids, lp, dt, T=T, tail=1, in_place=True, what=f"gap {gap}, in place")


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(12, 60), (12, 9001), (4, 90001), (1300, 3001), (520, 40001), (520, 70001)])
def test_distill_of_logits_that_are_no_numbers(torch, G, rows, V, dt, tail):
    """NaN and +inf, listed or not: NaN in the row's loss and all of its gradient, and nothing in
    any other row, the next one of the same block among them."""
    rng = np.random.default_rng(28)
    ids, lp = _teacher(rng, rows, V, 6)
    z = torch.randn(rows, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(28)).to(
        torch.float32 if dt == "f32" else torch.bfloat16)
    bad = np.arange(1, rows, 3)
    for r in bad:
        other = next(v for v in rng.permutation(V) if v not in ids[r])
        z[r, int(ids[r, 2] if r % 2 else other)] = math.nan if r % 4 < 2 else INF
    ti, tl = torch.from_numpy(ids).cuda(), torch.from_numpy(lp).cuda()
    loss, loss2 = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    g = torch.zeros_like(z)
    args = dict(ids=ti.data_ptr(), teacher=tl.data_ptr(), k=6, tail=tail)
    with G.Ops() as ops:
        ops.distill_loss(z.data_ptr(), rows, V, DT[dt], loss=loss.data_ptr(), **args)
        ops.distill_grad(z.data_ptr(), rows, V, DT[dt], loss=loss2.data_ptr(), grad=g.data_ptr(), **args)
        torch.cuda.synchronize()
    want = np.zeros(rows, bool)
    want[bad] = True
    for out in (loss, loss2, g.float().sum(1)):
        assert np.array_equal(np.isnan(_host(out)), want)
    assert bool(torch.isnan(g[torch.from_numpy(bad).cuda()]).all())
    assert bool(torch.isfinite(g[torch.from_numpy(~want).cuda()]).all())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,possible", [(4, 12, 12), (3, 4000, 20), (2, 90001, 20), (300, 3001, 20)])
def test_a_record_of_all_possible_tokens_distils_into_itself(torch, G, rows, V, possible, dt):
    """Where every token that can occur is listed nothing is left for the tail but the record's
    rounding."""
    rng = np.random.default_rng(24)
    k = 24
    values = np.full((rows, V), -INF)
    for r in range(rows):
        values[r, rng.permutation(V)[:possible]] = rng.normal(size=possible) * 3
    z, _ = _matrix(torch, values, dt)
    ids = torch.zeros(rows, k, device="cuda", dtype=torch.int32)
    lp, loss = torch.zeros(rows, k, device="cuda"), torch.zeros(rows, device="cuda")
    g = torch.zeros(rows, V, device="cuda", dtype=z.dtype)
    with G.Ops() as ops:
        for T in (1.0, 0.7, 1.9):
            ops.token_scores(z.data_ptr(), rows, V, DT[dt], temperature=T, top_k=k, top_ids=ids.data_ptr(),
                             top_logprob=lp.data_ptr())
            ops.distill_grad(z.data_ptr(), rows, V, DT[dt], temperature=T, ids=ids.data_ptr(), teacher=lp.data_ptr(), k=k,
                             tail=1, loss=loss.data_ptr(), grad=g.data_ptr())
            torch.cuda.synchronize()
            # both sides carry the bounds of their log probabilities (of at most 30 nats)
            tol = 4 * R.U * (V / 256 + 64 + 4 * 30)
            assert float(loss.abs().max()) < tol and float(g.float().abs().max()) < tol / T


# ---- scores --------------------------------------------------------------------------
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(64, 30), (64, 3001), (2, 90001)])
def test_scores_are_those_of_probabilities(torch, G, rows, V, dt):
    """Near a single outcome: no probability above 1, no entropy below 0."""
    rng = np.random.default_rng(25)
    z = rng.normal(size=(rows, V)) * 0.3
    z[np.arange(rows), rng.integers(0, V, rows)] += rng.uniform(2, 40, rows) + math.log(V)
    z += rng.normal(size=(rows, 1)) * 5
    zt, _ = _matrix(torch, z, dt)
    for T in (1.0, 0.9, 0.37):
        got = _score(torch, G, zt, T, None, 3, dt)
        assert float(got["top_logprob"].max()) <= 0 and float(got["entropy"].min()) >= 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(6, 9), (6, 700), (6, 20001), (2, 90001)])
def test_scores_alternatives_beside_a_signalling_nan(torch, G, rows, V, dt):
    """Every NaN is left out of the alternatives, whatever its bits."""
    rng = np.random.default_rng(26)
    z = rng.normal(size=(rows, V)) * 3
    z, buf = _matrix(torch, z, dt)
    bits = z.view(torch.int32 if dt == "f32" else torch.int16)
    codes = (0x7FA00001, -0x005FFFFF) if dt == "f32" else (0x7FA1, -0x005F)
    best = z.float().argsort(dim=1, descending=True)[:, :4].cpu().numpy()
    for r in range(rows):
        for i, b in enumerate(best[r]):
            # beside the row's largest, on one side or the other
            at = min(V - 1, b + 1) if (r + i) % 2 else max(0, b - 1)
            if at not in best[r]:
                bits[r, int(at)] = codes[i % 2]
    with np.errstate(invalid="ignore"):
        host = z.float().cpu().numpy().astype(np.float64)
    broken = np.isnan(host).any(axis=1)
    assert broken.any()
    k = min(8, V)
    got = _score(torch, G, z, 1.0, None, k, dt)
    want = R.scores(host, 1.0, np.zeros((rows, 0), int), k)
    assert np.array_equal(got["top_ids"].cpu().numpy(), want["top_ids"])
    for name in ("lse", "entropy"):
        assert np.array_equal(np.isnan(_host(got[name])), broken)


# ---- the recurrence -------------------------------------------------------------------
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("B,D", [(1, 3), (8, 64), (21, 137), (64, 520)])
def test_single_tokens_leave_their_states(torch, G, B, D, dt):
    """A training call of one token a sequence keeps its states as any other does."""
    rng = np.random.default_rng(27)
    x, _ = _matrix(torch, rng.normal(size=(B, D)), dt)
    g, _ = _matrix(torch, rng.normal(size=(B, D)), dt)
    h0 = torch.from_numpy(rng.normal(size=(B, D)).astype(np.float32)).cuda()
    rows = G.gem_scan_state_rows(B)
    states = torch.full((rows * D + 4,), math.nan, device="cuda")
    y, dx, dg = (torch.zeros(B, D, device="cuda", dtype=x.dtype) for _ in range(3))
    d0 = torch.zeros(B, D, device="cuda")
    dy, _ = _matrix(torch, rng.normal(size=(B, D)), dt)
    args = (x.data_ptr(), g.data_ptr(), B, D, B, DT[dt])
    with G.Ops(G.gem_scan_scratch(B, D)) as ops:
        ops.scan_forward(*args, y=y.data_ptr(), h0=h0.data_ptr(), states=states.data_ptr())
        torch.cuda.synchronize()
        assert bool(torch.isfinite(states[:rows * D]).all()) and bool(torch.isnan(states[rows * D:]).all())
        ops.scan_backward(*args, h0=h0.data_ptr(), states=states.data_ptr(), dy=dy.data_ptr(), dx=dx.data_ptr(),
                          dgate=dg.data_ptr(), dh0=d0.data_ptr())
        torch.cuda.synchronize()
    u = R.BF16_U if dt == "bf16" else 0.0
    for b in range(B):
        w = R.scan(_host(x)[b:b + 1], _host(g)[b:b + 1], _host(h0)[b], _host(dy)[b:b + 1], np.zeros(D))
        _same(_host(dx)[b:b + 1], w["dx"], w["dxe"] + u * np.abs(w["dx"]) + 1e-37, "dx")
        _same(_host(dg)[b:b + 1], w["dg"], w["dge"] + u * np.abs(w["dg"]) + 1e-37, "dgate")
        _same(_host(d0)[b], w["dh0"], w["dh0e"] + 1e-37, "dh0")


@pytest.mark.parametrize("most,tokens,channels", [(32768, 32640, 2048), (4097, 4096, 130), (70000, 65535, 513)])
def test_a_handle_for_the_longest_batch_takes_shorter_ones(torch, G, most, tokens, channels):
    x = torch.randn(tokens, channels, device="cuda", dtype=torch.bfloat16)
    y, y2 = torch.zeros_like(x), torch.zeros_like(x)
    with G.Ops(G.gem_scan_scratch(most, channels)) as ops, G.Ops(G.gem_scan_scratch(tokens, channels)) as own:
        ops.scan_forward(x.data_ptr(), x.data_ptr(), tokens, channels, 1, G.GEM_BF16, y=y.data_ptr())
        own.scan_forward(x.data_ptr(), x.data_ptr(), tokens, channels, 1, G.GEM_BF16, y=y2.data_ptr())
        torch.cuda.synchronize()
    assert torch.equal(y, y2)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_nothing_passes_from_one_sequence_to_another(torch, G, dt):
    """NaN and infinities in one sequence of a pack, in both directions."""
    lengths, D = [300, 40, 700, 5, 333], 72
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    N, B = int(off[-1]), len(lengths)
    rng = np.random.default_rng(29)
    x, g, dy = (_matrix(torch, rng.normal(size=(N, D)) + m, dt)[0] for m in (0, 2, 0))
    h0, dl = (torch.from_numpy(rng.normal(size=(B, D)).astype(np.float32)).cuda() for _ in range(2))
    offs = torch.from_numpy(off).cuda()

    def go():
        y, dx, dg = (torch.zeros_like(x) for _ in range(3))
        last, d0 = torch.zeros_like(h0), torch.zeros_like(h0)
        states = torch.zeros(G.gem_scan_state_rows(N), D, device="cuda")
        args = dict(x=x.data_ptr(), gate=g.data_ptr(), tokens=N, channels=D, sequences=B, dtype=DT[dt], offsets=offs.data_ptr(),
                    h0=h0.data_ptr())
        with G.Ops(G.gem_scan_scratch(N, D)) as ops:
            ops.scan_forward(y=y.data_ptr(), h_last=last.data_ptr(), states=states.data_ptr(), **args)
            ops.scan_backward(states=states.data_ptr(), dy=dy.data_ptr(), dx=dx.data_ptr(), dgate=dg.data_ptr(),
                              dh_last=dl.data_ptr(), dh0=d0.data_ptr(), **args)
            torch.cuda.synchronize()
        return (y, dx, dg), (last, d0)

    whole, ends = go()
    for broken in (1, 2, 4):
        for value in (math.nan, INF):
            kept = [a.clone() for a in (x, dy, h0, dl)]
            lo, hi = int(off[broken]), int(off[broken + 1])
            x[lo:hi:7], dy[lo:hi:5], h0[broken], dl[broken] = value, value, value, value
            rows, rest = go()
            for a, b in zip(kept, (x, dy, h0, dl)):
                b.copy_(a)
            for a, b in zip(rows, whole):
                assert torch.equal(a[:lo], b[:lo]) and torch.equal(a[hi:], b[hi:])
                assert not bool(torch.isfinite(a[hi - 1]).any())
            for a, b in zip(rest, ends):
                assert torch.equal(a[:broken], b[:broken]) and torch.equal(a[broken + 1:], b[broken + 1:])
