"""The worker's operators in numpy, in 64 bits and straight from their formulas, with bounds
on what 32-bit arithmetic may differ by (no kernel code)."""
import numpy as np

U = 2.0 ** -24          # half a unit in the last place of binary32
BF16_U = 2.0 ** -8      # of bfloat16


def scores(z, T, tokens, k):
    """lse, entropy, logprob of given tokens, alternatives, and the probabilities' logs."""
    z = np.asarray(z, np.float64)
    rows, V = z.shape
    lse, ent = np.empty(rows), np.empty(rows)
    logp = np.empty((rows, V))
    ids, top = np.full((rows, k), -1, np.int32), np.full((rows, k), -np.inf)
    for r in range(rows):
        x = z[r] / T
        if np.isnan(x).any() or (x == np.inf).any():
            lse[r] = ent[r] = np.nan
            logp[r] = np.where(x == -np.inf, -np.inf, np.nan)
        elif (x == -np.inf).all():
            lse[r], ent[r], logp[r] = -np.inf, 0.0, -np.inf
        else:
            m = x.max()
            ls = np.log(np.exp(x - m).sum())
            lse[r] = m + ls
            logp[r] = x - m - ls
            p = np.exp(logp[r])
            ent[r] = -(p[p > 0] * logp[r][p > 0]).sum()
        order = [v for v in np.argsort(np.where(np.isnan(z[r]), np.inf, -z[r]), kind="stable")
                 if z[r, v] > -np.inf][:k]
        ids[r, :len(order)] = order
        top[r, :len(order)] = logp[r, order]
    given = np.zeros(tokens.shape)
    for r in range(rows):
        for i, t in enumerate(tokens[r]):
            if 0 <= t < V:
                given[r, i] = logp[r, t]
    return dict(lse=lse, entropy=ent, logprob=given, top_ids=ids, top_logprob=top)


def score_tolerance(V, value):
    """Of a log probability or lse v: the scale log2(e)/T, the fused product and the conversion
    to nats round once each (4 |v| U, with the logarithm's last bit); a thread adds at most
    V/256 exponentials of one or two units, and the partial sums meet in a few more steps."""
    return U * (4 * np.abs(np.where(np.isfinite(value), value, 0.0)) + V / 256 + 32)


def entropy_tolerance(V, H):
    """H = log s - t/s, where t is taken about a reference at most 20 octaves from the row's
    largest: s and t each carry the sum's relative error, and |t/s| <= H + 20 ln 2 + ..."""
    return U * (V / 256 + 32) * (30 + np.abs(np.where(np.isfinite(H), H, 0.0)))


def first_entries(ids, V):
    """The entries that count: inside the vocabulary, the first of each token."""
    seen, keep = set(), np.zeros(len(ids), bool)
    for i, t in enumerate(ids):
        if 0 <= t < V and t not in seen:
            seen.add(int(t))
            keep[i] = True
    return keep


def distill_row(z, T, ids, lp, tail):
    """(loss, gradient without the weight, q, p by token, p_t, q_t) of one row."""
    z, lp = np.asarray(z, np.float64) / T, np.asarray(lp, np.float64)
    V = z.size
    keep = first_entries(ids, V)
    at, lp = np.asarray(ids)[keep], lp[keep]
    m = z.max()
    if m == -np.inf:
        q, logq = np.zeros(V), np.full(V, -np.inf)
    else:
        e = np.exp(z - m)
        q, logq = e / e.sum(), z - m - np.log(e.sum())
    p = np.exp(lp)
    if not tail and p.sum() > 0:
        lp = lp - np.log(p.sum())
        p = p / p.sum()
    with np.errstate(divide="ignore", invalid="ignore"):
        loss = float(np.where(p > 0, p * (lp - logq[at]), 0.0).sum())
        full = np.zeros(V)
        full[at] = p
        out = np.ones(V, bool)
        out[at] = False
        pt = max(0.0, 1.0 - p.sum()) if tail else 0.0
        qt = q[out].sum()
        mass = p.sum() + pt
        g = mass * q - full
        if pt > 0:
            loss += pt * (np.log(pt) - np.log(qt))
            if qt > 0:
                g[out] = q[out] * (mass - pt / qt)
    return loss, g / T, q, full, pt, qt


def distill_tolerance(V, k, T, z, q, p, pt, qt, loss, g, w, bf16):
    """Bounds of the loss and of the (weighted) gradient.  q carries the row sum's relative
    error, the rounding of its exponent (in octaves, at most the row's spread) and of the
    scale; p a few units; 1 - sum p the absolute error of a sum of k terms."""
    fin = z[np.isfinite(z)] / T
    spread = (fin.max() - fin.min()) if fin.size else 0.0
    rel = U * (V / 256 + 64 + 2 * spread)
    miss = U * (k + 8)                                   # of p_t
    lp_err = (q > 0) * 0.0 + U * (V / 256 + 64 + 4 * spread + 8)
    loss_tol = (p * lp_err).sum() + 8 * U * np.abs(p[p > 0] * np.log(p[p > 0])).sum() + U * (k + 8) * abs(loss)
    if pt > 0 and qt > 0:
        loss_tol += pt * rel + miss * (abs(np.log(pt / qt)) + 2) + miss
    tol = (q * (1 + (pt / qt if pt > 0 and qt > 0 else 0)) + p) * rel
    if pt > 0 and qt > 0:
        tol = tol + q / qt * miss
    tol = tol * abs(w) / T + np.abs(g * w) * (BF16_U if bf16 else 4 * U) + 1e-37
    return loss_tol + 4 * U, tol


def scan(x, g, h0, dy, dh_last):
    """One sequence [T, D]: the recurrence, its backward pass, and a bound of each, run
    through the same recurrences: every step adds a few units of what it handles."""
    x, g = np.asarray(x, np.float64), np.asarray(g, np.float64)
    T, D = x.shape
    a, b = 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
    h, y, before, err, yerr, berr = h0.astype(np.float64), np.empty((T, D)), np.empty((T, D)), np.zeros(D), np.empty((T, D)), np.empty((T, D))
    gu = (8 + 2 * np.abs(g)) * U        # relative error of a and b: exp of g, division, products
    for t in range(T):
        before[t], berr[t] = h, err
        err = a[t] * err + (a[t] * np.abs(h) * b[t] + b[t] * np.abs(x[t])) * gu[t] + 4 * U * (a[t] * np.abs(h) + b[t] * np.abs(x[t]))
        h = a[t] * h + b[t] * x[t]
        y[t], yerr[t] = h, err
    out = dict(y=y, h_last=h, yerr=2 * yerr, h_err=2 * err)
    if dy is None:
        return out
    e, eerr = dh_last.astype(np.float64), np.zeros(D)
    dx, dg, dxe, dge = (np.empty((T, D)) for _ in range(4))
    for t in range(T - 1, -1, -1):
        r, re = dy[t] + e, eerr + 2 * U * (np.abs(dy[t]) + np.abs(e))
        dx[t], dxe[t] = b[t] * r, b[t] * (re + (gu[t] + 2 * U) * np.abs(r))
        f = a[t] * b[t]
        dg[t] = f * (before[t] - x[t]) * r
        dge[t] = f * ((np.abs(before[t]) + np.abs(x[t])) * (re + (2 * gu[t] + 4 * U) * np.abs(r)) + berr[t] * np.abs(r))
        e, eerr = a[t] * r, a[t] * (re + (b[t] * gu[t] + 4 * U) * np.abs(r))
    out.update(dx=dx, dg=dg, dh0=e, dxe=2 * dxe, dge=2 * dge, dh0e=2 * eerr)
    return out
