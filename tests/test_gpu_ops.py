"""The worker's operators on the GPU against their formulas in 64 bits (ops_reference.py): sizes
from one up, odd ones, strides, addresses off every alignment, masks, ties, infinities and NaN,
and what each call refuses."""
import ctypes as C
import math

import numpy as np
import pytest

import ops_reference as R

pytestmark = pytest.mark.gpu

INF = math.inf


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


@pytest.fixture(scope="module")
def G():
    from paper_1805_08469_amd import gem
    return gem


DT = {"f32": 0, "bf16": 1}


def _type(torch, dt):
    return torch.float32 if dt == "f32" else torch.bfloat16


def _matrix(torch, values, dt, pad=0, shift=0, fill=77.0):
    """The values on the GPU in rows `pad` longer, the first `shift` elements off the
    allocation's start; the view, and the whole buffer whose other elements hold `fill`."""
    rows, cols = values.shape
    buf = torch.full((shift + rows * (cols + pad) + 8,), fill, device="cuda", dtype=_type(torch, dt))
    view = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.from_numpy(np.ascontiguousarray(values, dtype=np.float32)))
    return view, buf


def _kept(torch, buf, view, fill=77.0):
    """Every element of buf outside view still holds fill."""
    other = buf.clone()
    o = view.storage_offset() - buf.storage_offset()
    rows, cols = view.shape
    other[o:o + rows * view.stride(0)].view(rows, view.stride(0))[:, :cols] = fill
    return bool((other == fill).all())


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _same(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what + ": NaN places"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what + ": infinities"
    assert not np.isinf(got[~inf]).any(), what + ": infinities"
    fin = np.isfinite(want)
    off = np.abs(got[fin] - want[fin]) - np.broadcast_to(tol, want.shape)[fin]
    assert off.size == 0 or off.max() <= 0, f"{what}: {off.max():.3g} beyond the bound"


# ---- scores ----------------------------------------------------------------------
def _score(torch, G, z, T=1.0, tokens=None, k=0, dt="f32", stream=None):
    rows, V = z.shape
    n = 0 if tokens is None else tokens.shape[1]
    tok = torch.from_numpy(np.ascontiguousarray(tokens, np.int32)).cuda() if n else None
    lse, ent = (torch.full((rows,), 55.0, device="cuda") for _ in range(2))
    given = torch.full((rows, n), 55.0, device="cuda")
    ids = torch.full((rows, k), 55, device="cuda", dtype=torch.int32)
    top = torch.full((rows, k), 55.0, device="cuda")
    with G.Ops(0, stream) as ops:
        ops.token_scores(z.data_ptr(), rows, V, DT[dt], stride=z.stride(0), temperature=T,
                         tokens=tok.data_ptr() if n else None, n_tokens=n, top_k=k,
                         logprob=given.data_ptr() if n else None, entropy=ent.data_ptr(),
                         lse=lse.data_ptr(), top_ids=ids.data_ptr() if k else None,
                         top_logprob=top.data_ptr() if k else None)
        torch.cuda.synchronize()
    return dict(lse=lse, entropy=ent, logprob=given, top_ids=ids, top_logprob=top)


def _check_scores(torch, G, values, dt, T=1.0, k=4, n=2, pad=0, shift=0, what=""):
    z, buf = _matrix(torch, values, dt, pad, shift)
    rows, V = z.shape
    rng = np.random.default_rng(rows * 7919 + V)
    tokens = rng.integers(-1, V + 1, size=(rows, n))
    print(f"[scores] {what} rows={rows} V={V} {dt} T={T} k={k} n={n} pad={pad} shift={shift}", flush=True)
    got = _score(torch, G, z, T, tokens, k, dt)
    want = R.scores(_host(z), T, tokens, k)
    assert np.array_equal(got["top_ids"].cpu().numpy(), want["top_ids"]), what
    for name in ("lse", "logprob", "top_logprob"):
        _same(_host(got[name]), want[name], R.score_tolerance(V, want[name]), f"{what} {name}")
    _same(_host(got["entropy"]), want["entropy"], R.entropy_tolerance(V, want["entropy"]), f"{what} entropy")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 63, 64, 65, 255, 257, 1000, 2049, 8191, 20001])
def test_scores_of_any_vocabulary(torch, G, V, dt):
    rng = np.random.default_rng(V)
    z = rng.normal(size=(5, V)) * 3
    _check_scores(torch, G, z, dt, k=min(V + 2, 64))
    _check_scores(torch, G, z, dt, T=0.7, k=1, n=5)


@pytest.mark.parametrize("rows,V", [(1, 130001), (2, 70000), (3, 33333), (17, 40000), (700, 5001), (1500, 300)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_scores_of_few_and_many_rows(torch, G, rows, V, dt):
    rng = np.random.default_rng(rows)
    _check_scores(torch, G, rng.normal(size=(rows, V)) * 2.5, dt, k=20, n=1)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (0, 1), (1, 0), (3, 5), (8, 0), (8, 3), (43, 7)])
def test_scores_of_strided_rows_at_any_address(torch, G, pad, shift, dt):
    rng = np.random.default_rng(pad * 10 + shift)
    _check_scores(torch, G, rng.normal(size=(9, 3001)) * 3, dt, k=17, pad=pad, shift=shift)
    _check_scores(torch, G, rng.normal(size=(2, 30011)) * 3, dt, k=17, pad=pad, shift=shift)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("k", [0, 1, 2, 31, 64, 127, 128])
def test_scores_any_number_of_alternatives(torch, G, k, dt):
    rng = np.random.default_rng(k)
    _check_scores(torch, G, rng.normal(size=(6, 9001)) * 3, dt, k=k, n=1)
    _check_scores(torch, G, rng.normal(size=(300, 1501)) * 3, dt, k=k, n=0)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 12000, 50000])
@pytest.mark.parametrize("kind", ["equal", "zeros of both signs", "rising", "falling", "few levels", "one high",
                                  "rising in steps", "two halves"])
def test_scores_ties_and_orders(torch, G, V, kind, dt):
    i = np.arange(V)
    rng = np.random.default_rng(V)
    z = {"equal": np.full(V, 1.5), "zeros of both signs": np.where(i % 3 == 0, -0.0, 0.0),
         "rising": i * (20.0 / V), "falling": -i * (20.0 / V), "few levels": rng.integers(0, 5, V) * 0.5,
         "one high": np.where(i == V - 1, 30.0, 0.0), "rising in steps": i // 700 * 0.25,
         "two halves": np.where(i < V // 2, 0.0, 1.0 + i % 2)}[kind]
    _check_scores(torch, G, np.stack([z, z + 0.25, rng.permutation(z)]), dt, k=64, what=kind)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [9, 3000, 40001])
def test_scores_of_masked_and_unusual_logits(torch, G, V, dt):
    rng = np.random.default_rng(V + 1)
    z = rng.normal(size=(12, V)) * 2
    low = -3.3895313892515355e38                 # bfloat16's lowest value
    z[0, :] = -INF                               # nothing can occur
    z[1, 1:] = -INF                              # one token left
    z[2, ::2] = -INF
    z[3, :] = low                                # everything masked by the lowest value: equal
    z[4, V // 2:] = low
    z[5, V - 1] = np.nan
    z[6, 0] = INF
    z[7, :-1] = -INF
    z[8, :] = low
    z[8, V // 3] = -INF
    z[9] *= 1e4                                  # a spread of thousands
    z[10, 2] = np.nan
    z[10, 4] = INF
    z[11, :] = np.nan
    _check_scores(torch, G, z, dt, k=8, n=3, what="unusual")
    _check_scores(torch, G, z, dt, k=8, n=3, T=2.0, what="unusual")


def test_scores_of_large_logits_keep_their_differences(torch, G):
    rng = np.random.default_rng(0)
    z = rng.normal(size=(4, 5000)) + 1e4         # binary32 holds them to 5e-4; differences count
    _check_scores(torch, G, z.astype(np.float32), "f32", k=5)


def test_scores_outputs_may_be_left_out(torch, G):
    z, _ = _matrix(torch, np.random.default_rng(1).normal(size=(3, 500)), "f32")
    ent = torch.zeros(3, device="cuda")
    ids = torch.zeros(3, 7, device="cuda", dtype=torch.int32)
    with G.Ops() as ops:
        ops.token_scores(z.data_ptr(), 3, 500, 0, entropy=ent.data_ptr())
        ops.token_scores(z.data_ptr(), 3, 500, 0, top_k=7, top_ids=ids.data_ptr())
        ops.token_scores(z.data_ptr(), 0, 500, 0, entropy=ent.data_ptr())      # no rows
        ops.token_scores(z.data_ptr(), 3, 500, 0, top_k=7)                     # nothing asked
        torch.cuda.synchronize()
    want = R.scores(_host(z), 1.0, np.zeros((3, 0), int), 7)
    assert np.array_equal(ids.cpu().numpy(), want["top_ids"])
    _same(_host(ent), want["entropy"], R.entropy_tolerance(500, want["entropy"]), "entropy")


# ---- distillation -----------------------------------------------------------------
def _teacher(rng, rows, V, k, mass=0.9):
    ids = np.full((rows, k), -1, np.int32)
    lp = np.full((rows, k), -INF, np.float32)
    for r in range(rows):
        m = min(k, V)
        pick = rng.permutation(V)[:m] if V < 100000 else np.unique(rng.integers(0, V, 2 * m))[:m]
        p = rng.gamma(0.5, size=len(pick)) + 1e-6
        ids[r, :len(pick)] = pick
        lp[r, :len(pick)] = np.log(p / p.sum() * mass)
    return ids, lp


def _check_distill(torch, G, values, ids, lp, dt, T=1.0, tail=0, w=None, pad=0, shift=0, gpad=0, gshift=0,
                   in_place=False, what=""):
    z, buf = _matrix(torch, values, dt, pad, shift)
    rows, V = z.shape
    k = ids.shape[1]
    print(f"[distill] {what} rows={rows} V={V} {dt} T={T} k={k} tail={tail} pad={pad},{gpad} shift={shift},{gshift}",
          flush=True)
    host = _host(z)
    ti, tl = torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(lp.astype(np.float32)).cuda()
    wt = None if w is None else torch.from_numpy(np.asarray(w, np.float32)).cuda()
    loss, loss2 = (torch.full((rows,), 55.0, device="cuda") for _ in range(2))
    if in_place:
        g, gbuf = z, buf
    else:
        g, gbuf = _matrix(torch, np.full((rows, V), 33.0), dt, gpad, gshift)
    args = dict(stride=z.stride(0), temperature=T, ids=ti.data_ptr(), teacher=tl.data_ptr(), k=k, tail=tail,
                weight=None if wt is None else wt.data_ptr())
    with G.Ops() as ops:
        ops.distill_loss(z.data_ptr(), rows, V, DT[dt], loss=loss.data_ptr(), **args)
        ops.distill_grad(z.data_ptr(), rows, V, DT[dt], loss=loss2.data_ptr(), grad=g.data_ptr(),
                         grad_stride=g.stride(0), **args)
        torch.cuda.synchronize()
    assert _kept(torch, gbuf, g), f"{what}: a write beside the gradient"
    got, got2, grad = _host(loss), _host(loss2), _host(g)
    for r in range(rows):
        wr = 1.0 if w is None else float(np.float32(w[r]))
        if wr == 0.0:
            assert got[r] == 0 and got2[r] == 0 and not grad[r].any(), f"{what}: row {r} has no weight"
            continue
        lo, gr, q, p, pt, qt = R.distill_row(host[r], T, ids[r], lp[r], tail)
        lt, gt = R.distill_tolerance(V, k, T, host[r], q, p, pt, qt, lo if np.isfinite(lo) else 0.0, gr, wr, dt == "bf16")
        _same(got[r:r + 1], np.array([lo]), lt, f"{what} loss of row {r}")
        _same(got2[r:r + 1], np.array([lo]), lt, f"{what} loss (with gradient) of row {r}")
        _same(grad[r], gr * wr, gt, f"{what} gradient of row {r}")


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 257, 1000, 8193, 40003])
def test_distill_of_any_vocabulary(torch, G, V, dt, tail):
    rng = np.random.default_rng(V)
    ids, lp = _teacher(rng, 4, V, min(V, 16))
    _check_distill(torch, G, rng.normal(size=(4, V)) * 2, ids, lp, dt, tail=tail, w=[1.0, 0.5, -0.25, 0.0])


@pytest.mark.parametrize("rows,V,k", [(1, 150001, 64), (3, 70001, 1), (33, 20011, 128), (600, 3001, 32)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_distill_of_few_and_many_rows(torch, G, rows, V, k, dt):
    rng = np.random.default_rng(rows)
    ids, lp = _teacher(rng, rows, V, k)
    w = np.where(np.arange(rows) % 4 == 3, 0.0, 1.0 / rows)
    _check_distill(torch, G, rng.normal(size=(rows, V)) * 2, ids, lp, dt, T=2.0, tail=1, w=w)
    _check_distill(torch, G, rng.normal(size=(rows, V)) * 2, ids, lp, dt, T=0.7, tail=0, w=w)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift,gpad,gshift", [(0, 1, 0, 0), (0, 0, 0, 1), (1, 0, 3, 5), (8, 3, 0, 2), (43, 7, 43, 7)])
@pytest.mark.parametrize("V", [1001, 30011])
def test_distill_of_strided_rows_at_any_address(torch, G, V, pad, shift, gpad, gshift, dt):
    rng = np.random.default_rng(pad + shift)
    ids, lp = _teacher(rng, 5, V, 20)
    _check_distill(torch, G, rng.normal(size=(5, V)) * 2, ids, lp, dt, tail=1, pad=pad, shift=shift, gpad=gpad,
                   gshift=gshift)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [901, 50021, 140003])
@pytest.mark.parametrize("rows", [2, 300])
def test_distill_gradient_in_the_logits_memory(torch, G, rows, V, dt):
    if rows * V > 2e7:
        rows = 140
    rng = np.random.default_rng(5)
    ids, lp = _teacher(rng, rows, V, 9)
    _check_distill(torch, G, rng.normal(size=(rows, V)) * 2, ids, lp, dt, tail=1, pad=3, in_place=True)


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [50, 20000])
def test_distill_entries_that_do_not_count(torch, G, V, dt, tail):
    rng = np.random.default_rng(6)
    ids, lp = _teacher(rng, 8, V, 12)
    ids[0, :] = -1                              # no entries
    ids[1, 3:] = -1
    ids[2, 5] = ids[2, 1]                       # a token twice: the first counts
    ids[2, 9] = ids[2, 1]
    ids[3, 4] = V                               # beyond the vocabulary
    ids[3, 5] = 2**31 - 1
    ids[3, 6] = -2**31
    lp[4, 2] = -INF                             # a listed token of probability 0
    lp[5, :] = -INF                             # all of them
    lp[6, :] += 0.5                             # more than the whole mass: nothing left for the tail
    ids[7, :] = ids[7, 0]
    _check_distill(torch, G, rng.normal(size=(8, V)) * 2, ids, lp, dt, tail=tail, what="entries")


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 20000])
def test_distill_of_masked_logits(torch, G, V, dt, tail):
    rng = np.random.default_rng(7)
    ids, lp = _teacher(rng, 6, V, 8, mass=0.95)
    z = rng.normal(size=(6, V)) * 2
    listed = np.zeros((6, V), bool)
    listed[np.arange(6)[:, None], ids] = True
    z[0, ~listed[0]] = -INF                     # only listed tokens can occur
    z[1, ids[1, 0]] = -INF                      # a listed one cannot: infinite loss
    z[2, :] = -INF
    z[3, ~listed[3]] = -3.3895313892515355e38
    z[4, ::2] = np.where(listed[4, ::2], z[4, ::2], -INF)
    z[5, :] += 60.0
    _check_distill(torch, G, z, ids, lp, dt, tail=tail, what="masked")


def test_distill_weightless_rows_are_not_read(torch, G):
    rng = np.random.default_rng(8)
    ids, lp = _teacher(rng, 3, 3000, 8)
    z = rng.normal(size=(3, 3000))
    z[1] = np.nan
    ids[1], lp[1] = 7, np.nan
    _check_distill(torch, G, z, ids, lp, "f32", tail=1, w=[1.0, 0.0, 2.0])


def test_distill_gradient_against_differences_of_the_loss(torch, G):
    """The gradient the kernel gives, against central differences of the loss in 64 bits."""
    rng = np.random.default_rng(9)
    V = 31
    ids, lp = _teacher(rng, 1, V, 6, mass=0.8)
    z = rng.normal(size=(1, V)).astype(np.float32).astype(np.float64)
    for tail in (0, 1):
        zt, _ = _matrix(torch, z, "f32")
        g = torch.zeros(1, V, device="cuda")
        ti, tl = torch.from_numpy(ids).cuda(), torch.from_numpy(lp).cuda()
        with G.Ops() as ops:
            ops.distill_grad(zt.data_ptr(), 1, V, 0, ids=ti.data_ptr(), teacher=tl.data_ptr(), k=6, tail=tail,
                             grad=g.data_ptr(), temperature=1.5)
            torch.cuda.synchronize()
        for v in range(V):
            hi, lo = z[0].copy(), z[0].copy()
            hi[v] += 1e-5
            lo[v] -= 1e-5
            d = (R.distill_row(hi, 1.5, ids[0], lp[0], tail)[0] - R.distill_row(lo, 1.5, ids[0], lp[0], tail)[0]) / 2e-5
            assert abs(d - float(g[0, v])) < 2e-5 * max(abs(d), 0.05)


def test_a_record_of_scores_distils_into_itself(torch, G):
    """The alternatives that gem_token_scores records, read by the loss at the same
    temperature against the same logits: no divergence, no gradient."""
    rows, V, k, T = 6, 9000, 48, 1.7
    z, _ = _matrix(torch, np.random.default_rng(10).normal(size=(rows, V)) * 3, "f32")
    ids = torch.zeros(rows, k, device="cuda", dtype=torch.int32)
    lp, loss, g = torch.zeros(rows, k, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros(rows, V, device="cuda")
    with G.Ops() as ops:
        ops.token_scores(z.data_ptr(), rows, V, 0, temperature=T, top_k=k, top_ids=ids.data_ptr(), top_logprob=lp.data_ptr())
        ops.distill_grad(z.data_ptr(), rows, V, 0, temperature=T, ids=ids.data_ptr(), teacher=lp.data_ptr(), k=k, tail=1,
                         loss=loss.data_ptr(), grad=g.data_ptr())
        torch.cuda.synchronize()
    # both sides carry the bounds of their log probabilities
    tol = 4 * R.U * (V / 256 + 64 + 40)
    assert float(loss.abs().max()) < tol and float(g.abs().max()) < tol


# ---- the recurrence ---------------------------------------------------------------
def _check_scan(torch, G, lengths, D, dt, ragged=True, pad=0, shift=0, h0=True, train=True, gate=(1.0, 2.0), what=""):
    rng = np.random.default_rng(len(lengths) * 31 + D + sum(lengths))
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    N, B = int(off[-1]), len(lengths)
    print(f"[scan] {what} lengths={lengths[:6]}.. N={N} B={B} D={D} {dt} pad={pad} shift={shift} ragged={ragged}", flush=True)
    x, _ = _matrix(torch, rng.normal(size=(N, D)), dt, pad, shift)
    g, _ = _matrix(torch, rng.normal(size=(N, D)) * gate[1] + gate[0], dt, pad, shift)
    dy, _ = _matrix(torch, rng.normal(size=(N, D)), dt, pad, shift)
    y, ybuf = _matrix(torch, np.full((N, D), 33.0), dt, pad, shift)
    dx, dxbuf = _matrix(torch, np.full((N, D), 33.0), dt, pad, shift)
    dg, dgbuf = _matrix(torch, np.full((N, D), 33.0), dt, pad, shift)
    start = torch.from_numpy(rng.normal(size=(B, D)).astype(np.float32)).cuda()
    last = torch.full((B, D), 55.0, device="cuda")
    dl = torch.from_numpy(rng.normal(size=(B, D)).astype(np.float32)).cuda()
    d0 = torch.full((B, D), 55.0, device="cuda")
    offs = torch.from_numpy(off).cuda()
    states = torch.full((G.gem_scan_state_rows(N) * D + 4,), 55.0, device="cuda")
    row = D + pad
    args = dict(x=x.data_ptr(), gate=g.data_ptr(), tokens=N, channels=D, sequences=B, dtype=DT[dt],
                offsets=offs.data_ptr() if ragged else None, h0=start.data_ptr() if h0 else None, x_stride=row,
                gate_stride=row)
    with G.Ops(G.gem_scan_scratch(N, D)) as ops:
        ops.scan_forward(y=y.data_ptr(), y_stride=row, h_last=last.data_ptr(), states=states.data_ptr() if train else None, **args)
        if train:
            ops.scan_backward(states=states.data_ptr(), dy=dy.data_ptr(), dy_stride=row, dx=dx.data_ptr(), dx_stride=row,
                              dgate=dg.data_ptr(), dgate_stride=row, dh_last=dl.data_ptr() if h0 else None,
                              dh0=d0.data_ptr(), **args)
        torch.cuda.synchronize()
    for buf, view in ((ybuf, y), (dxbuf, dx), (dgbuf, dg)):
        assert _kept(torch, buf, view), f"{what}: a write beside an output"
    assert bool((states[-4:] == 55.0).all())
    X, Gt, DY = _host(x), _host(g), _host(dy)
    H0 = _host(start) if h0 else np.zeros((B, D))
    DL = _host(dl) if h0 else np.zeros((B, D))
    u = R.BF16_U if dt == "bf16" else 0.0
    for b in range(B):
        lo, hi = off[b], off[b + 1]
        w = R.scan(X[lo:hi], Gt[lo:hi], H0[b], DY[lo:hi] if train else None, DL[b])
        _same(_host(y[lo:hi]), w["y"], w["yerr"] + u * np.abs(w["y"]), f"{what} y of sequence {b}")
        _same(_host(last[b]), w["h_last"], w["h_err"], f"{what} h_last of {b}")
        if train:
            _same(_host(dx[lo:hi]), w["dx"], w["dxe"] + u * np.abs(w["dx"]) + 1e-37, f"{what} dx of {b}")
            _same(_host(dg[lo:hi]), w["dg"], w["dge"] + u * np.abs(w["dg"]) + 1e-37, f"{what} dgate of {b}")
            _same(_host(d0[b]), w["dh0"], w["dh0e"] + 1e-37, f"{what} dh0 of {b}")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 2, 3, 7, 16, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 513, 1100])
def test_scan_of_any_length(torch, G, N, dt):
    _check_scan(torch, G, [N], 72, dt)
    _check_scan(torch, G, [N, N, N], 33, dt, ragged=False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", [1, 2, 3, 4, 7, 8, 31, 63, 64, 65, 127, 129, 257, 520])
def test_scan_of_any_number_of_channels(torch, G, D, dt):
    _check_scan(torch, G, [5, 140, 1, 60], D, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", [[0], [0, 0, 0], [0, 5, 0, 0, 9, 0], [1] * 300, [0] * 200 + [1] * 3 + [0] * 100,
                                     [128, 128, 0, 128], [127, 1, 128, 129, 0, 255], [300, 0, 1, 700, 2, 0],
                                     [3] * 90 + [0] * 5 + [400], [1, 0] * 150])
def test_scan_of_unequal_sequences(torch, G, lengths, dt):
    _check_scan(torch, G, lengths, 70, dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 0), (8, 8), (43, 2)])
def test_scan_of_strided_rows_at_any_address(torch, G, pad, shift, dt):
    _check_scan(torch, G, [200, 77, 0, 40], 96, dt, pad=pad, shift=shift)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_scan_without_states_or_starts(torch, G, dt):
    _check_scan(torch, G, [150, 20], 40, dt, h0=False)
    _check_scan(torch, G, [150, 20], 40, dt, train=False)
    _check_scan(torch, G, [1] * 64, 256, dt, ragged=False, train=False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("gate", [(9.0, 1.0), (-9.0, 1.0), (0.0, 30.0), (16.0, 0.5)])
def test_scan_gates_near_their_ends(torch, G, gate, dt):
    _check_scan(torch, G, [600, 33], 50, dt, gate=gate)


def test_scan_gates_that_are_infinite(torch, G):
    """A gate of -inf forgets at once, one of +inf keeps; a NaN stays in its channel."""
    N, D = 200, 8
    rng = np.random.default_rng(12)
    g = rng.normal(size=(N, D))
    g[50, 0], g[60:, 1], g[70, 2] = -INF, INF, np.nan
    X, x_ = _matrix(torch, rng.normal(size=(N, D)), "f32")
    gt, _ = _matrix(torch, g, "f32")
    y = torch.zeros(N, D, device="cuda")
    with G.Ops(G.gem_scan_scratch(N, D)) as ops:
        ops.scan_forward(X.data_ptr(), gt.data_ptr(), N, D, 1, 0, y=y.data_ptr())
        torch.cuda.synchronize()
    x, y = _host(X), _host(y)
    assert abs(y[50, 0] - x[50, 0]) < 1e-6
    assert np.all(np.abs(y[60:, 1] - y[59, 1]) < 1e-5 * 140)
    assert np.isnan(y[70:, 2]).all() and np.isfinite(y[:70, 2]).all()
    assert np.isfinite(np.delete(y, 2, axis=1)).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_scan_steps_in_place_are_the_whole(torch, G, dt):
    """Answering token after token from a state kept in place gives the sequence's values."""
    B, T, D = 5, 40, 136
    rng = np.random.default_rng(13)
    x, _ = _matrix(torch, rng.normal(size=(B * T, D)), dt)
    g, _ = _matrix(torch, rng.normal(size=(B * T, D)) + 1, dt)
    y, whole = torch.zeros(B * T, D, device="cuda", dtype=x.dtype), torch.zeros(B * T, D, device="cuda", dtype=x.dtype)
    h = torch.zeros(B, D, device="cuda")
    last = torch.zeros(B, D, device="cuda")
    with G.Ops(G.gem_scan_scratch(B * T, D)) as ops:
        ops.scan_forward(x.data_ptr(), g.data_ptr(), B * T, D, B, DT[dt], y=whole.data_ptr(), h_last=last.data_ptr())
        size = x.element_size()
        for t in range(T):
            ops.scan_forward(x.data_ptr() + t * D * size, g.data_ptr() + t * D * size, B, D, B, DT[dt],
                             y=y.data_ptr() + t * D * size, h0=h.data_ptr(), h_last=h.data_ptr(), x_stride=T * D,
                             gate_stride=T * D, y_stride=T * D)
        torch.cuda.synchronize()
    tol = 1e-5 if dt == "f32" else 2.02 * R.BF16_U      # bfloat16: neighbours where the roundings part
    assert float((y.float() - whole.float()).abs().max()) <= tol * float(whole.float().abs().max())
    assert float((h - last).abs().max()) < 1e-5


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("ragged,lengths", [(False, [40] * 3), (True, [300, 0, 1, 16, 40, 0, 7, 2000, 3]),
                                            (True, [0, 5000, 0]), (False, [4096] * 2), (True, [9000, 64, 20000])])
def test_scan_of_long_sequences_keeps_a_state_in_place(torch, G, ragged, lengths, dt):
    """h_last in h0's memory: the same bits as with a memory of its own, also where other blocks
    hold a sequence's first tokens and its last."""
    D, B = 137, len(lengths)
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    N = int(off[-1])
    rng = np.random.default_rng(16)
    x, _ = _matrix(torch, rng.normal(size=(N, D)), dt)
    g, _ = _matrix(torch, rng.normal(size=(N, D)) + 4, dt)
    start = torch.from_numpy(rng.normal(size=(B, D)).astype(np.float32)).cuda()
    offs = torch.from_numpy(off).cuda()
    y, y2 = (torch.zeros(N, D, device="cuda", dtype=x.dtype) for _ in range(2))
    last, state = torch.zeros(B, D, device="cuda"), start.clone()
    args = dict(x=x.data_ptr(), gate=g.data_ptr(), tokens=N, channels=D, sequences=B, dtype=DT[dt],
                offsets=offs.data_ptr() if ragged else None)
    with G.Ops(G.gem_scan_scratch(N, D)) as ops:
        ops.scan_forward(y=y.data_ptr(), h0=start.data_ptr(), h_last=last.data_ptr(), **args)
        ops.scan_forward(y=y2.data_ptr(), h0=state.data_ptr(), h_last=state.data_ptr(), **args)
        torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(state, last)


def test_scan_long_sequence(torch, G):
    """Long enough that thousands of parts of the sequence are joined."""
    _check_scan(torch, G, [40000, 3, 20001], 65, "bf16", gate=(5.0, 2.0))


@pytest.mark.parametrize("offsets", [[0, 10**9, 100], [-5, 40, 100], [0, 90, 20], [100, 50, 0], [7, 7, 7]])
def test_scan_offsets_of_any_content_stay_in_bounds(torch, G, offsets):
    """Offsets are not checked: a malformed table gives some values, within the arrays."""
    N, D = 100, 40
    rng = np.random.default_rng(14)
    x, _ = _matrix(torch, rng.normal(size=(N, D)), "f32")
    y, ybuf = _matrix(torch, np.zeros((N, D)), "f32")
    off = torch.tensor(offsets, device="cuda", dtype=torch.int64)
    h = torch.full((2 * D + 8,), 55.0, device="cuda")
    with G.Ops(G.gem_scan_scratch(N, D)) as ops:
        ops.scan_forward(x.data_ptr(), x.data_ptr(), N, D, 2, 0, y=y.data_ptr(), offsets=off.data_ptr(), h_last=h.data_ptr())
        torch.cuda.synchronize()
    assert _kept(torch, ybuf, y) and bool((h[2 * D:] == 55.0).all())


# ---- streams, graphs, repeats -------------------------------------------------------
def _everything(torch, G, ops, dt="bf16"):
    """A function that queues every operator, and its outputs."""
    rng = np.random.default_rng(15)
    rows, V, k, N, D = 5, 40003, 20, 1500, 200
    z, _ = _matrix(torch, rng.normal(size=(rows, V)) * 3, dt)
    x, _ = _matrix(torch, rng.normal(size=(N, D)), dt)
    g, _ = _matrix(torch, rng.normal(size=(N, D)) + 2, dt)
    dev = dict(device="cuda")
    o = dict(ids=torch.zeros(rows, k, dtype=torch.int32, **dev), lp=torch.zeros(rows, k, **dev),
             ent=torch.zeros(rows, **dev), loss=torch.zeros(rows, **dev), dz=torch.zeros(rows, V, dtype=z.dtype, **dev),
             y=torch.zeros(N, D, dtype=x.dtype, **dev), h=torch.zeros(3, D, **dev), dx=torch.zeros(N, D, dtype=x.dtype, **dev),
             dg=torch.zeros(N, D, dtype=x.dtype, **dev), d0=torch.zeros(3, D, **dev))
    states = torch.zeros(G.gem_scan_state_rows(N), D, **dev)

    def go():
        ops.token_scores(z.data_ptr(), rows, V, DT[dt], temperature=2.0, top_k=k, entropy=o["ent"].data_ptr(),
                         top_ids=o["ids"].data_ptr(), top_logprob=o["lp"].data_ptr())
        ops.distill_grad(z.data_ptr(), rows, V, DT[dt], ids=o["ids"].data_ptr(), teacher=o["lp"].data_ptr(), k=k, tail=1,
                         loss=o["loss"].data_ptr(), grad=o["dz"].data_ptr())
        ops.scan_forward(x.data_ptr(), g.data_ptr(), N, D, 3, DT[dt], y=o["y"].data_ptr(), h_last=o["h"].data_ptr(),
                         states=states.data_ptr())
        ops.scan_backward(x.data_ptr(), g.data_ptr(), N, D, 3, DT[dt], states=states.data_ptr(), dy=o["y"].data_ptr(),
                          dx=o["dx"].data_ptr(), dgate=o["dg"].data_ptr(), dh0=o["d0"].data_ptr())
    return go, o, (z, x, g, states)


def test_repeats_give_the_same_bits(torch, G):
    with G.Ops(G.gem_scan_scratch(1500, 200)) as ops:
        go, o, keep = _everything(torch, G, ops)
        go()
        torch.cuda.synchronize()
        first = {n: t.clone() for n, t in o.items()}
        for _ in range(5):
            for t in o.values():
                t.zero_()
            go()
            torch.cuda.synchronize()
            for n, t in o.items():
                assert torch.equal(t, first[n]), n


def test_work_is_queued_on_the_handles_stream(torch, G):
    """On a stream of its own, behind inputs that the same stream still has to write."""
    s = torch.cuda.Stream()
    with G.Ops(G.gem_scan_scratch(1500, 200), s.cuda_stream) as ops:
        go, o, (z, x, g, states) = _everything(torch, G, ops)
        torch.cuda.synchronize()
        go()
        torch.cuda.synchronize()
        first = {n: t.clone() for n, t in o.items()}
        real = z.clone()
        z.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            big = torch.randn(64 << 20, device="cuda").sort().values      # keeps the stream busy
            z.copy_(real)
        go()
        s.synchronize()
        for n, t in o.items():
            assert torch.equal(t, first[n]), n
        del big


def test_a_captured_graph_replays(torch, G):
    s = torch.cuda.Stream()
    with G.Ops(G.gem_scan_scratch(1500, 200), s.cuda_stream) as ops:
        go, o, (z, x, g, states) = _everything(torch, G, ops)
        torch.cuda.synchronize()
        go()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            go()
        for step in range(4):
            z.mul_(0.9)
            x.mul_(1.1)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = {n: t.clone() for n, t in o.items()}
            for t in o.values():
                t.zero_()
            torch.cuda.synchronize()
            go()
            torch.cuda.synchronize()
            for n, t in o.items():
                assert torch.equal(t, got[n]), (step, n)


# ---- the ends of the ranges ---------------------------------------------------------
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300007, 1 << 22])
def test_scores_of_the_largest_vocabularies(torch, G, V, dt):
    """Rows in as many parts as there are, with the most alternatives."""
    rng = np.random.default_rng(17)
    _check_scores(torch, G, rng.normal(size=(2, V)) * 2, dt, k=128, n=3)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_distill_of_the_largest_vocabulary(torch, G, dt):
    rng = np.random.default_rng(18)
    V = 1 << 22
    ids, lp = _teacher(rng, 2, V, 128, mass=0.9)
    _check_distill(torch, G, rng.normal(size=(2, V)) * 2, ids, lp, dt, tail=1)


# ---- refusals ----------------------------------------------------------------------
def test_refusals(torch, G):
    L = G.lib()
    buf = torch.zeros(4096, device="cuda")
    p = buf.data_ptr()
    out = C.c_void_p()
    assert L.gem_ops_create(1 << 60, None, C.byref(out)) == G.GEM_ENOMEM and out.value is None
    with G.Ops() as ops:
        h = ops.h

        def score(n=0, k=0, tok=None, scores=None, **kw):
            z = dict(data=p, rows=2, stride=0, vocab=10, dtype=0, temperature=1.0, reserved=0)
            z.update(kw)
            return L.gem_token_scores(h, C.byref(G.gem_logits(**z)), tok, n, k,
                                      C.byref(scores or G.gem_scores(entropy=p + 1024)))

        assert score() == G.GEM_OK
        for bad in (dict(data=None), dict(rows=-1), dict(vocab=0), dict(vocab=G.GEM_VOCAB_MAX + 1), dict(stride=9),
                    dict(stride=-10), dict(stride=2**40), dict(rows=2**40), dict(temperature=0.0), dict(temperature=-1.0),
                    dict(temperature=INF), dict(temperature=math.nan), dict(temperature=1e-40), dict(temperature=3e38),
                    dict(n=-1), dict(k=-1), dict(k=G.GEM_TOP_MAX + 1), dict(n=3)):
            assert score(**bad) == G.GEM_EINVAL, bad
        assert score(dtype=2) == G.GEM_EDTYPE and score(dtype=-1) == G.GEM_EDTYPE
        assert score(data=p + 2) == G.GEM_EALIGN and score(data=p + 1, dtype=1) == G.GEM_EALIGN
        assert score(data=p + 2, dtype=1) == G.GEM_OK
        assert score(scores=G.gem_scores(entropy=p + 1026)) == G.GEM_EALIGN
        assert score(n=1, tok=p + 2) == G.GEM_EALIGN
        assert L.gem_token_scores(h, None, None, 0, 0, C.byref(G.gem_scores())) == G.GEM_EINVAL
        assert L.gem_token_scores(None, C.byref(G.gem_logits(p, 2, 0, 10, 0, 1.0, 0)), None, 0, 0,
                                  C.byref(G.gem_scores())) == G.GEM_EINVAL

        ids = torch.full((16,), -1, device="cuda", dtype=torch.int32)

        def distill(grad=p + 2048, gs=0, loss=p + 1024, t=None, **kw):
            z = dict(data=p, rows=2, stride=0, vocab=10, dtype=0, temperature=1.0, reserved=0)
            z.update({n: kw[n] for n in kw if n in z})
            te = dict(ids=ids.data_ptr(), logprob=p + 512, k=4, tail=0)
            te.update({n: kw[n] for n in kw if n in te})
            return L.gem_distill_grad(h, C.byref(G.gem_logits(**z)), C.byref(G.gem_teacher(**te)), None, loss, grad, gs)

        assert distill() == G.GEM_OK and distill(loss=None) == G.GEM_OK
        for bad in (dict(k=0), dict(k=G.GEM_TOP_MAX + 1), dict(tail=2), dict(tail=-1), dict(ids=None), dict(logprob=None),
                    dict(grad=None), dict(gs=9), dict(rows=-1), dict(vocab=0), dict(temperature=0.0),
                    dict(grad=p, gs=12)):
            assert distill(**bad) == G.GEM_EINVAL, bad
        assert distill(dtype=3) == G.GEM_EDTYPE
        assert distill(grad=p + 2049) == G.GEM_EALIGN and distill(loss=p + 1) == G.GEM_EALIGN
        assert L.gem_distill_loss(h, C.byref(G.gem_logits(p, 2, 0, 10, 0, 1.0, 0)), None, None, p) == G.GEM_EINVAL
        assert L.gem_distill_loss(h, C.byref(G.gem_logits(p, 2, 0, 10, 0, 1.0, 0)),
                                  C.byref(G.gem_teacher(ids.data_ptr(), p, 4, 0)), None, None) == G.GEM_EINVAL

        def scan(y=p + 4096, ys=0, **kw):
            s = dict(x=p, gate=p, offsets=None, h0=None, tokens=8, x_stride=0, gate_stride=0, channels=4, sequences=2,
                     dtype=0, reserved=0)
            s.update(kw)
            return L.gem_scan_forward(h, C.byref(G.gem_scan(**s)), y, ys, None, None)

        assert scan() == G.GEM_OK
        for bad in (dict(x=None), dict(gate=None), dict(tokens=-1), dict(tokens=2**31), dict(channels=0), dict(sequences=0),
                    dict(sequences=3), dict(x_stride=3), dict(gate_stride=-1), dict(ys=2), dict(y=None)):
            assert scan(**bad) == G.GEM_EINVAL, bad
        assert scan(dtype=7) == G.GEM_EDTYPE
        for bad in (dict(x=p + 2), dict(gate=p + 1, dtype=1), dict(offsets=p + 4), dict(h0=p + 2), dict(y=p + 4097)):
            assert scan(**bad) == G.GEM_EALIGN, bad
        s = G.gem_scan(p, p, None, None, 8, 0, 0, 4, 2, 0, 0)
        assert L.gem_scan_backward(h, C.byref(s), None, p, 0, None, p, 0, p, 0, None) == G.GEM_EINVAL
        assert L.gem_scan_backward(h, C.byref(s), p, None, 0, None, p, 0, p, 0, None) == G.GEM_EINVAL
        assert L.gem_scan_backward(h, C.byref(s), p, p, 2, None, p, 0, p, 0, None) == G.GEM_EINVAL
        assert L.gem_scan_backward(h, None, p, p, 0, None, p, 0, p, 0, None) == G.GEM_EINVAL
        torch.cuda.synchronize()
