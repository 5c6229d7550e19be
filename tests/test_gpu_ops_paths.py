"""The worker's operators at the sizes that take their other paths: more rows of logits than
blocks, runs of every length, more rows than one launch takes, more elements than 32 bits count."""
import numpy as np
import pytest

import ops_reference as R
from test_gpu_ops import DT, G, _check_distill, _host, _same, _teacher, torch  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- more rows than blocks ---------------------------------------------------------------
def _weights(rows, seed):
    """Of any sign, with runs of rows that have none as long as several rounds of blocks, and
    single ones."""
    rng = np.random.default_rng(seed)
    w = rng.normal(size=rows)
    w[5::11] = 0.0
    w[rows // 3:rows // 3 + 40] = 0.0
    w[np.arange(rows) % 256 == 17] = 0.0       # all rows of a block of the larger grids
    w[-3:] = 0.0
    return w


@pytest.mark.parametrize("tail,k,pad,in_place,T", [(0, 32, 0, False, 1.0), (1, 128, 3, False, 0.7), (1, 9, 1, True, 1.0)])
@pytest.mark.parametrize("rows,V,dt", [(2500, 3001, "f32"), (2500, 3001, "bf16"), (1100, 20001, "bf16"), (1100, 12001, "f32"),
                                       (560, 50021, "bf16"), (560, 25001, "f32"), (530, 100003, "bf16"), (530, 50001, "f32")])
def test_distill_of_more_rows_than_blocks(torch, G, rows, V, dt, tail, k, pad, in_place, T):
    """Blocks that go from row to row, in every layout of a row over registers."""
    rng = np.random.default_rng(rows + V + k)
    ids, lp = _teacher(rng, rows, V, k)
    values = rng.standard_normal(size=(rows, V), dtype=np.float32) * 2
    _check_distill(torch, G, values, ids, lp, dt, T=T, tail=tail, w=_weights(rows, k), pad=pad, shift=pad, gpad=pad,
                   in_place=in_place, what="rows")


# ---- more rows than one launch takes ------------------------------------------------------
def test_scores_in_several_launches(torch, G):
    """Rows whose parts leave more than the handle's scratch holds at once."""
    rows, V, k = 4200, 66001, 128
    z = torch.randn(rows, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).mul_(2)
    lse, ids = torch.zeros(rows, device="cuda"), torch.zeros(rows, k, device="cuda", dtype=torch.int32)
    top = torch.zeros(rows, k, device="cuda")
    with G.Ops() as ops:
        ops.token_scores(z.data_ptr(), rows, V, 0, top_k=k, lse=lse.data_ptr(), top_ids=ids.data_ptr(), top_logprob=top.data_ptr())
        torch.cuda.synchronize()
    some = np.unique(np.concatenate([np.arange(0, rows, 400), np.arange(4020, 4050), [rows - 1]]))
    want = R.scores(_host(z[some]), 1.0, np.zeros((some.size, 0), int), k)
    assert np.array_equal(ids[some].cpu().numpy(), want["top_ids"])
    _same(_host(lse[some]), want["lse"], R.score_tolerance(V, want["lse"]), "lse")
    _same(_host(top[some]), want["top_logprob"], R.score_tolerance(V, want["top_logprob"]), "top_logprob")
    assert bool(((lse - z.logsumexp(1)).abs() < 1e-3).all())


def test_distill_in_several_launches(torch, G):
    rows, V, k = 15500, 65601, 128
    rng = np.random.default_rng(2)
    z = torch.randn(rows, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).mul_(2)
    some = np.unique(np.concatenate([np.arange(0, rows, 1500), np.arange(15410, 15432), [rows - 1]]))
    before = _host(z[some])
    one, onelp = _teacher(rng, 64, V, k)
    ids, lp = np.tile(one, (rows // 64 + 1, 1))[:rows], np.tile(onelp, (rows // 64 + 1, 1))[:rows]
    ti, tl = torch.from_numpy(ids).cuda(), torch.from_numpy(lp).cuda()
    loss, loss2 = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    args = dict(ids=ti.data_ptr(), teacher=tl.data_ptr(), k=k, tail=1)
    with G.Ops() as ops:
        ops.distill_loss(z.data_ptr(), rows, V, 0, loss=loss.data_ptr(), **args)
        ops.distill_grad(z.data_ptr(), rows, V, 0, loss=loss2.data_ptr(), grad=z.data_ptr(), **args)
        torch.cuda.synchronize()
    assert torch.equal(loss, loss2) and bool((z.sum(1).abs() < 1e-2).all())     # a gradient's elements sum to 0
    got, grad = _host(loss[some]), _host(z[some])
    for i, r in enumerate(some):
        lo, gr, q, p, pt, qt = R.distill_row(before[i], 1.0, ids[r], lp[r], 1)
        lt, gt = R.distill_tolerance(V, k, 1.0, before[i], q, p, pt, qt, lo, gr, 1.0, False)
        _same(got[i:i + 1], np.array([lo]), lt, f"loss of row {r}")
        _same(grad[i], gr, gt, f"gradient of row {r}")


# ---- runs of every length ------------------------------------------------------------------
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,ragged", [([1025] * 4, False), ([1300, 0, 1, 700, 16, 0, 2083], True), ([4100], False),
                                            ([31, 97, 64, 127, 129, 3, 0, 255, 3394], True)])
@pytest.mark.parametrize("D", [2050, 4100, 8100, 16001])
def test_scan_in_runs_of_every_length(torch, G, D, lengths, ragged, dt):
    """The more channels, the longer the runs of a row of lanes (16 to 128 tokens)."""
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    N, B = int(off[-1]), len(lengths)
    gen = torch.Generator(device="cuda").manual_seed(D + B)
    t = torch.float32 if dt == "f32" else torch.bfloat16

    def rand(rows, mean, scale, dtype):
        return torch.randn(rows, D, device="cuda", generator=gen).mul_(scale).add_(mean).to(dtype)

    x, g, dy = rand(N, 0, 1, t), rand(N, 2, 2, t), rand(N, 0, 1, t)
    h0, dl = rand(B, 0, 1, torch.float32), rand(B, 0, 1, torch.float32)
    y, dx, dg = (torch.zeros_like(x) for _ in range(3))
    last, d0, state = torch.zeros_like(h0), torch.zeros_like(h0), h0.clone()
    states = torch.zeros(G.gem_scan_state_rows(N), D, device="cuda")
    offs = torch.from_numpy(off).cuda()
    args = dict(x=x.data_ptr(), gate=g.data_ptr(), tokens=N, channels=D, sequences=B, dtype=DT[dt],
                offsets=offs.data_ptr() if ragged else None)
    print(f"[scan] runs N={N} B={B} D={D} {dt}", flush=True)
    with G.Ops(G.gem_scan_scratch(N, D)) as ops:
        ops.scan_forward(y=y.data_ptr(), h0=h0.data_ptr(), h_last=last.data_ptr(), states=states.data_ptr(), **args)
        ops.scan_backward(states=states.data_ptr(), h0=h0.data_ptr(), dy=dy.data_ptr(), dx=dx.data_ptr(), dgate=dg.data_ptr(),
                          dh_last=dl.data_ptr(), dh0=d0.data_ptr(), **args)
        y2 = torch.zeros_like(y)
        ops.scan_forward(y=y2.data_ptr(), h0=state.data_ptr(), h_last=state.data_ptr(), **args)
        torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(state, last)
    # Channels at the slices' ends and the last ones, moved-back slices among them, and some between.
    some = np.unique(np.concatenate([np.arange(6), np.arange(60, 68), np.arange(124, 132), np.arange(0, D, D // 40),
                                     np.arange(D - 132, D - 120), np.arange(D - 68, D - 60), np.arange(D - 6, D)]))
    X, Gt, DY, Y, DX, DG = (_host(a[:, some]) for a in (x, g, dy, y, dx, dg))
    H0, DL, HL, D0 = (_host(a[:, some]) for a in (h0, dl, last, d0))
    u = R.BF16_U if dt == "bf16" else 0.0
    for b in range(B):
        lo, hi = off[b], off[b + 1]
        w = R.scan(X[lo:hi], Gt[lo:hi], H0[b], DY[lo:hi], DL[b])
        _same(Y[lo:hi], w["y"], w["yerr"] + u * np.abs(w["y"]), f"y of sequence {b}")
        _same(HL[b], w["h_last"], w["h_err"], f"h_last of {b}")
        _same(DX[lo:hi], w["dx"], w["dxe"] + u * np.abs(w["dx"]) + 1e-37, f"dx of {b}")
        _same(DG[lo:hi], w["dg"], w["dge"] + u * np.abs(w["dg"]) + 1e-37, f"dgate of {b}")
        _same(D0[b], w["dh0"], w["dh0e"] + 1e-37, f"dh0 of {b}")


# ---- offsets past 32 bits --------------------------------------------------------------------
def test_scores_and_gradients_of_more_elements_than_32_bits_count(torch, G):
    rows, V, k = 69000, 32768, 8
    z = torch.randn(rows, V, device="cuda", dtype=torch.bfloat16, generator=torch.Generator(device="cuda").manual_seed(3))
    ids, top = torch.zeros(rows, k, device="cuda", dtype=torch.int32), torch.zeros(rows, k, device="cuda")
    loss = torch.zeros(rows, device="cuda")
    some = np.array([0, 1, 32767, 32768, 65534, 65535, 65536, rows - 2, rows - 1])
    before = _host(z[some])
    with G.Ops() as ops:
        ops.token_scores(z.data_ptr(), rows, V, 1, top_k=k, top_ids=ids.data_ptr(), top_logprob=top.data_ptr(), temperature=0.5)
        ops.distill_grad(z.data_ptr(), rows, V, 1, ids=ids.data_ptr(), teacher=top.data_ptr(), k=k, tail=1,
                         loss=loss.data_ptr(), grad=z.data_ptr())
        torch.cuda.synchronize()
    want = R.scores(before, 0.5, np.zeros((some.size, 0), int), k)
    at, lp = ids[some].cpu().numpy(), top[some].cpu().numpy()
    assert np.array_equal(at, want["top_ids"])
    _same(lp, want["top_logprob"], R.score_tolerance(V, want["top_logprob"]), "top_logprob")
    got, grad = _host(loss[some]), _host(z[some])
    for i in range(some.size):
        lo, gr, q, p, pt, qt = R.distill_row(before[i], 1.0, at[i], lp[i], 1)
        lt, gt = R.distill_tolerance(V, k, 1.0, before[i], q, p, pt, qt, lo, gr, 1.0, True)
        _same(got[i:i + 1], np.array([lo]), lt, f"loss of row {some[i]}")
        _same(grad[i], gr, gt, f"gradient of row {some[i]}")


def test_scan_of_more_elements_than_32_bits_count(torch, G):
    B, T, D = 1080, 1000, 2048
    N = B * T
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, g, dy = (torch.randn(N, D, device="cuda", dtype=torch.bfloat16, generator=gen) for _ in range(3))
    y, dx, dg = (torch.zeros_like(x) for _ in range(3))
    h0, dl = (torch.randn(B, D, device="cuda", generator=gen) for _ in range(2))
    last, d0 = torch.zeros_like(h0), torch.zeros_like(h0)
    states = torch.zeros(G.gem_scan_state_rows(N), D, device="cuda")
    args = (x.data_ptr(), g.data_ptr(), N, D, B, 1)
    with G.Ops(G.gem_scan_scratch(N, D)) as ops:
        ops.scan_forward(*args, y=y.data_ptr(), h0=h0.data_ptr(), h_last=last.data_ptr(), states=states.data_ptr())
        ops.scan_backward(*args, h0=h0.data_ptr(), states=states.data_ptr(), dy=dy.data_ptr(), dx=dx.data_ptr(),
                          dgate=dg.data_ptr(), dh_last=dl.data_ptr(), dh0=d0.data_ptr())
        torch.cuda.synchronize()
    for b in (0, 524, 1048, 1049, B - 1):          # 2^31 elements end in sequence 1048
        at = slice(b * T, (b + 1) * T)
        w = R.scan(_host(x[at]), _host(g[at]), _host(h0[b]), _host(dy[at]), _host(dl[b]))
        _same(_host(y[at]), w["y"], w["yerr"] + R.BF16_U * np.abs(w["y"]), f"y of sequence {b}")
        _same(_host(last[b]), w["h_last"], w["h_err"], f"h_last of {b}")
        _same(_host(dx[at]), w["dx"], w["dxe"] + R.BF16_U * np.abs(w["dx"]) + 1e-37, f"dx of {b}")
        _same(_host(dg[at]), w["dg"], w["dge"] + R.BF16_U * np.abs(w["dg"]) + 1e-37, f"dgate of {b}")
        _same(_host(d0[b]), w["dh0"], w["dh0e"] + 1e-37, f"dh0 of {b}")
