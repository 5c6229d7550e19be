"""The selective scan and its backward pass in numpy, in 64 bits and token after token, with bounds on
what 32-bit arithmetic may differ by (no kernel code)."""
import numpy as np

U = 2.0 ** -24


def sigmoid(v):
    return np.exp(-np.logaddexp(0.0, -v))


def scan(s, off, backward=True):
    """s: x, dt [T, D], b, c [T, N], z [T, D] or None, a [D, N], d, dt_bias [D], h0 [S, D, N] and, for the
    backward pass, dy [T, D], dh_last [S, D, N].  A dict of (value, bound).

    Each bound follows its value: a product or a sum adds the roundings of what it handles, an exponential
    four and four times its exponent's size, a sigmoid 8 + 2 |v|.  A sum over N states has N + 4, over D
    channels D / 4 + 24 (four in a lane, then steps that double), over tokens 300 + T / 64 (a run's 128,
    then the runs' by fours).  All are doubled for terms of the second order and states that several
    runs' products reach."""
    s = {k: np.asarray(v, np.float64) if v is not None else None for k, v in s.items()}
    T, D = s["x"].shape
    N = s["a"].shape[1]
    A, x, z = s["a"], s["x"], s["z"]
    v = s["dt"] + s["dt_bias"]
    sig = sigmoid(v)
    u = np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))
    u_e = U * ((3 * np.abs(v) + 4) * sig + 4 * u)
    h_all, h_err = np.empty((T, D, N)), np.empty((T, D, N))
    prev, prev_e = np.empty((T, D, N)), np.empty((T, D, N))
    h_last, h_last_e = s["h0"].copy(), np.zeros_like(s["h0"])

    def decay(t):
        r = u[t][:, None] * A
        a = np.exp(r)
        return a, a * (np.abs(A) * u_e[t][:, None] + U * (4 * np.abs(r) + 4))

    for q, (lo, hi) in enumerate(zip(off, off[1:])):
        h, e = s["h0"][q], np.zeros((D, N))
        for t in range(lo, hi):
            prev[t], prev_e[t] = h, e
            a, a_e = decay(t)
            inp = (u[t] * x[t])[:, None] * s["b"][t]
            in_e = np.abs(x[t][:, None] * s["b"][t]) * u_e[t][:, None] + 4 * U * np.abs(inp)
            e = a * e + a_e * np.abs(h) + in_e + 2 * U * (a * np.abs(h) + np.abs(inp))
            h = a * h + inp
            h_all[t], h_err[t] = h, e
        h_last[q], h_last_e[q] = h, e
    C = s["c"][:, None, :]
    bare = (C * h_all).sum(2) + s["d"] * x
    bare_e = (np.abs(C) * h_err).sum(2) + U * (N + 4) * ((np.abs(C * h_all)).sum(2) + np.abs(s["d"] * x))
    if z is not None:
        sz = sigmoid(z)
        gate, gate_e = z * sz, np.abs(z) * sz * U * (10 + 2 * np.abs(z))
        y, y_e = bare * gate, bare_e * np.abs(gate) + np.abs(bare) * gate_e
    else:
        y, y_e = bare, bare_e
    r = dict(y=(y, y_e), h_last=(h_last, h_last_e))
    if backward:
        dy = s["dy"]
        g, g_e = (dy * gate, np.abs(dy) * gate_e) if z is not None else (dy, np.zeros_like(dy))
        if z is not None:
            slope = sz * (1 + z * (1 - sz))
            r["dz"] = (dy * bare * slope, np.abs(dy) * (bare_e * np.abs(slope) + np.abs(bare) * U * (12 + 3 * np.abs(z)) *
                                                       (sz + np.abs(z) * sz * (1 - sz))))
        dx, dx_e, ddt, ddt_e = (np.empty((T, D)) for _ in range(4))
        db, db_e, dc, dc_e = (np.empty((T, N)) for _ in range(4))
        da, da_e = np.zeros((D, N)), np.zeros((D, N))
        dh0, dh0_e = s["dh_last"].copy(), np.zeros_like(s["dh_last"])
        wide, longer = U * (D / 4 + 24), U * (300 + T / 64)
        for q, (lo, hi) in enumerate(zip(off, off[1:])):
            e, e_e = s["dh_last"][q], np.zeros((D, N))
            for t in range(hi - 1, lo - 1, -1):
                a, a_e = decay(t)
                ux, ux_e = u[t] * x[t], np.abs(x[t]) * u_e[t] + U * np.abs(u[t] * x[t])
                cg = g[t][:, None] * s["c"][t]
                dh = cg + e
                dh_e = e_e + np.abs(s["c"][t]) * g_e[t][:, None] + 2 * U * (np.abs(cg) + np.abs(e))
                term = ux[:, None] * dh
                db[t] = term.sum(0)
                db_e[t] = (np.abs(ux)[:, None] * dh_e + ux_e[:, None] * np.abs(dh) + wide * np.abs(term)).sum(0)
                term = g[t][:, None] * h_all[t]
                dc[t] = term.sum(0)
                dc_e[t] = (np.abs(g[t])[:, None] * h_err[t] + g_e[t][:, None] * np.abs(h_all[t]) + wide * np.abs(term)).sum(0)
                into = (dh * s["b"][t]).sum(1)
                into_e = (dh_e * np.abs(s["b"][t]) + U * (N + 4) * np.abs(dh * s["b"][t])).sum(1)
                e, e_e = a * dh, a * dh_e + a_e * np.abs(dh) + U * np.abs(a * dh)
                p = e * prev[t]
                p_e = e_e * np.abs(prev[t]) + np.abs(e) * prev_e[t] + 2 * U * np.abs(p)
                flow = (p * A).sum(1)
                flow_e = (p_e * np.abs(A) + U * (N + 6) * np.abs(p * A)).sum(1)
                da += u[t][:, None] * p
                da_e += u[t][:, None] * p_e + u_e[t][:, None] * np.abs(p) + longer * np.abs(u[t][:, None] * p)
                dx[t] = s["d"] * g[t] + u[t] * into
                dx_e[t] = np.abs(s["d"]) * g_e[t] + u[t] * into_e + u_e[t] * np.abs(into) + 3 * U * (np.abs(s["d"] * g[t]) + np.abs(u[t] * into))
                k = x[t] * into + flow
                ddt[t] = k * sig[t]
                ddt_e[t] = sig[t] * (np.abs(x[t]) * into_e + flow_e + (np.abs(x[t] * into) + np.abs(flow)) * U * (14 + 3 * np.abs(v[t])))
            dh0[q], dh0_e[q] = e, e_e
        r.update(dx=(dx, dx_e), ddt=(ddt, ddt_e), db=(db, db_e), dc=(dc, dc_e), da=(da, da_e), dh0=(dh0, dh0_e),
                 dd=((g * x).sum(0), (g_e * np.abs(x) + longer * np.abs(g * x)).sum(0)),
                 ddt_bias=(ddt.sum(0), (ddt_e + longer * np.abs(ddt)).sum(0)))
    return {k: (value, 2 * e + 1e-37) for k, (value, e) in r.items()}
