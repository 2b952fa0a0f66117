"""Inputs, the formulas in 64 bits and error bounds for the tests of the adapter calls (test-side only).

Bounds: every sum of K products in fp32 is off by at most K 2^-23 times the sum of the products' magnitudes (2^-24 a
rounding, and as much again for the order inside the matrix pipes), a stored bf16 by 2^-8 of its value (half a step); the
projections H feed the second product, where they may be held in two bf16 terms (2^-16).
"""
import numpy as np
import torch

U32 = 2.0 ** -23


def make(T, J, D, n, R, S, dtype, seed, single=False, first=0, behind=0, none=0.15):
    """Host tensors of a batch: rows first .. T - behind - 1 belong to S requests (some empty, some without a block)."""
    g = torch.Generator().manual_seed(seed)
    last = T - behind
    if single:
        assert S == last - first
        start = torch.arange(first, last + 1)
    else:
        cuts = torch.randint(first, last + 1, (S + 1,), generator=g).sort().values
        if S:
            cuts[0], cuts[S] = first, last
        start = cuts
    c = dict(T=T, J=J, D=D, n=n, R=R, S=S, dtype=dtype, start=start.to(torch.int64))
    c["adapter"] = torch.randint(0, max(n, 1), (S,), generator=g, dtype=torch.int32)
    c["adapter"][torch.rand(S, generator=g) < none] = -1
    rnd = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    c["W"] = (rnd(J, D) * D ** -0.5).to(dtype)
    c["X"] = rnd(T, D).to(dtype)
    c["dY"] = (rnd(T, J) * 0.1).to(dtype)
    c["U"] = (rnd(n, R, J) * 0.5).to(dtype)
    c["V"] = (rnd(n, R, D) * D ** -0.5).to(dtype)
    c["ranks"] = torch.randint(0, R + 1, (n,), generator=g, dtype=torch.int32)
    if n:
        c["ranks"][n // 2] = R
    c["scale"] = torch.rand(n, generator=g) * 2 - 0.5
    return c


def poison(c):
    """Not-a-numbers where the calls must not look: pairs that are not in use, rows of no request."""
    for a in range(c["n"]):
        for k in ("U", "V"):
            c[k][a, int(c["ranks"][a]):] = float("nan")
    inside = torch.zeros(c["T"], dtype=torch.bool)
    if c["S"]:
        inside[int(c["start"][0]):int(c["start"][-1])] = True
    c["X"][~inside] = float("nan")
    c["dY"][~inside] = float("inf")
    return c


def rows_of(c):
    """{block or None: rows}, and the rows that belong to a request."""
    by, every = {}, []
    for q in range(c["S"]):
        a = int(c["adapter"][q])
        t = list(range(int(c["start"][q]), int(c["start"][q + 1])))
        if not 0 <= a < c["n"] or min(max(int(c["ranks"][a]), 0), c["R"]) == 0:
            a = None
        by.setdefault(a, []).extend(t)
        every += t
    return by, every


def _f(t):
    return t.double().numpy()


def reference(c):
    """Y, H, dX, dU, dV in 64 bits and, under the same names with "_tol", how far fp32 sums may be off (before any rounding of
    the result to bf16)."""
    T, J, D, n, R = (c[k] for k in ("T", "J", "D", "n", "R"))
    by, every = rows_of(c)
    X, W, G = (_f(c[k]) for k in ("X", "W", "dY"))
    r = {k: np.zeros(s) for k, s in (("Y", (T, J)), ("H", (T, R)), ("dX", (T, D)), ("dU", (n, R, J)), ("dV", (n, R, D)))}
    r.update({k + "_tol": np.zeros(v.shape) for k, v in list(r.items())})
    if every:
        r["Y"][every] = X[every] @ W.T
        r["Y_tol"][every] = (D + 16) * U32 * (np.abs(X[every]) @ np.abs(W).T)
        r["dX"][every] = G[every] @ W
        r["dX_tol"][every] = (J + 16) * U32 * (np.abs(G[every]) @ np.abs(W))
    for a, t in by.items():
        if a is None or not t:
            continue
        k = min(max(int(c["ranks"][a]), 0), R)
        s = float(c["scale"][a])
        U, V = _f(c["U"][a, :k]), _f(c["V"][a, :k])
        h, dh = s * X[t] @ V.T, s * G[t] @ U.T
        h_abs, dh_abs = abs(s) * np.abs(X[t]) @ np.abs(V).T, abs(s) * np.abs(G[t]) @ np.abs(U).T
        h_tol, dh_tol = (D + 16) * U32 * h_abs, (J + 16) * U32 * dh_abs
        r["H"][t, :k] = h
        r["H_tol"][t, :k] = h_tol
        r["Y"][t] += h @ U
        r["Y_tol"][t] += (h_tol + (2.0 ** -16 + (k + 16) * U32) * np.abs(h)) @ np.abs(U)
        r["dX"][t] += dh @ V
        r["dX_tol"][t] += (dh_tol + (2.0 ** -16 + (k + 16) * U32) * np.abs(dh)) @ np.abs(V)
        L = len(t) + 16
        r["dU"][a, :k] = h.T @ G[t]
        r["dU_tol"][a, :k] = (h_tol + L * U32 * np.abs(h)).T @ np.abs(G[t])
        r["dV"][a, :k] = dh.T @ X[t]
        r["dV_tol"][a, :k] = (dh_tol + L * U32 * np.abs(dh)).T @ np.abs(X[t])
    return r, every


def check(name, got, ref, rows=None):
    g = got.detach().cpu()
    half_step = 2.0 ** -8 if g.dtype == torch.bfloat16 else 2.0 ** -24
    g, r, tol = g.double().numpy(), ref[name], ref[name + "_tol"]
    if rows is not None:
        g, r, tol = g[rows], r[rows], tol[rows]
    assert g.shape == r.shape
    if not g.size:
        return
    assert np.all(np.isfinite(g)), name
    off = np.abs(g - r) - (tol * (1 + half_step) + half_step * np.abs(r) + 1e-37)
    assert np.all(off <= 0), (name, float(off.max()), np.unravel_index(off.argmax(), off.shape), int((off > 0).sum()))
