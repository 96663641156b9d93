"""Plain 64-bit implementations of the operators between a network and the leaf weights, written from their definitions (numpy, on
the CPU), and bounds on the fp32 kernels' rounding errors that follow from the arithmetic.

u = 2^-24 is half a step of fp32.  A sum of V positive terms in which each term passes through at most V / 256 + 64 additions and
multiplications (a thread's run over a row, then trees; exponential and scaling included) is off by at most `terms(V)` relative.
"""
import numpy as np

U, LEAST = 2.0 ** -24, 2.0 ** -149
#: what a rounding of a value can be off by, relative (half of eps), and below the normal range, absolute
REL = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 1.2e-38, "bfloat16": 1.2e-38, "float16": 2.0 ** -25}


def terms(vocab):
    return U * (vocab / 256 + 64)


# ---- tokens -------------------------------------------------------------------------------------------------------
def tokens(x, t, dlogp=None, dneg=None, dent=None, top=0):
    """x [R, V] float64, t [R, K]; returns a dict of values, gradients and their error bounds."""
    R, V = x.shape
    K = t.shape[1]
    m = x.max(1)
    some = m > -np.inf
    with np.errstate(all="ignore"):
        e = np.where(some[:, None], np.exp(x - np.where(some, m, 0.0)[:, None]), 0.0)
        # (the maximum goes first: next to the lowest fp32 value even 64 bits have no room for the logarithm)
        lp = np.where(some[:, None], (x - np.where(some, m, 0.0)[:, None]) - np.log(np.where(some, e.sum(1), 1.0))[:, None], -np.inf)
        p = np.exp(lp)
        plogp = np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0)
        h = -plogp.sum(1)
    out = {"entropy": h}
    spread = np.where(p > 0, p * np.where(p > 0, np.abs(x - m[:, None]), 0.0), 0.0).sum(1)
    out["entropy_tol"] = terms(V) * (12.0 + spread)
    ask = t >= 0
    bad = t >= V
    i = np.clip(t, 0, V - 1)
    rows = np.arange(R)[:, None]
    with np.errstate(all="ignore"):
        logp = np.where(ask, lp[rows, i], 0.0)
        # the mass of the other tokens, summed without the asked one
        rest = np.stack([np.delete(p[r], i[r, k]).sum() if V > 1 else 0.0 for r in range(R) for k in range(K)]).reshape(R, K) if K else np.zeros((R, 0))
        rest = np.where(some[:, None], rest, 1.0)
        neg = np.where(ask, np.log(rest), 0.0)
    out["logp"] = np.where(bad, np.nan, logp)
    out["neg"] = np.where(bad, np.nan, neg)
    with np.errstate(all="ignore"):
        out["logp_tol"] = terms(V) + 4 * U * np.where(np.isfinite(logp), np.abs(logp), 0.0)
        out["neg_tol"] = terms(V) + 4 * U * np.where(np.isfinite(neg), np.abs(neg), 0.0)
    if top:
        order = np.argsort(-(x + 0.0), axis=1, kind="stable")[:, :top]
        out["top_tokens"] = order
        out["top_logp"] = lp[rows, order]
        with np.errstate(all="ignore"):
            out["top_logp_tol"] = terms(V) + 4 * U * np.where(np.isfinite(out["top_logp"]), np.abs(out["top_logp"]), 0.0)
    if dlogp is None and dneg is None and dent is None:
        return out
    dlogp = np.zeros((R, K)) if dlogp is None else dlogp
    dneg = np.zeros((R, K)) if dneg is None else dneg
    dent = np.zeros(R) if dent is None else dent
    dx, mass = np.zeros_like(x), np.zeros_like(x)
    with np.errstate(all="ignore"):
        for r in range(R):
            for k in range(K):
                if not ask[r, k]:
                    continue
                j = i[r, k]
                one = np.zeros(V)
                one[j] = 1.0
                away = 1.0 - one
                dx[r] += dlogp[r, k] * (one * rest[r, k] - away * p[r])
                mass[r] += np.abs(dlogp[r, k]) * (one * rest[r, k] + away * p[r])
                if dneg[r, k] != 0:
                    q = away * p[r] / rest[r, k] if rest[r, k] > 0 else 0 * one
                    dx[r] += dneg[r, k] * p[r, j] * (q - one)
                    mass[r] += np.abs(dneg[r, k]) * p[r, j] * (q + one)
            hp = plogp[r] + p[r] * h[r]
            dx[r] -= dent[r] * hp
            mass[r] += np.abs(dent[r]) * (np.abs(plogp[r]) + p[r] * (h[r] + (12.0 + spread[r])))
        # every share is a product of probabilities, each off by what its logarithm is off by
        out["dlogits"] = np.where(some[:, None], dx, 0.0)
        out["dlogits_tol"] = np.where(some[:, None], mass * 2 * (terms(V) + K * U + 4 * U * np.where(p > 0, np.abs(np.where(p > 0, lp, 0)), 0.0)), 0.0)
    return out


# ---- recurrence ---------------------------------------------------------------------------------------------------
REAL, LOG, MAX = 0, 1, 2


def _step(s, a, h, x):
    if s == REAL:
        return a * h + x
    with np.errstate(all="ignore"):
        return np.logaddexp(a + h, x) if s == LOG else np.maximum(a + h, x)


def _shares(a, h, x):
    with np.errstate(all="ignore"):
        y = np.logaddexp(a + h, x)
        w = np.where(y == -np.inf, 0.0, np.exp(a + h - y))
        v = np.where(y == -np.inf, 0.0, np.exp(x - y))
    return w, v


def scan(s, a, x, h0, dh=None, dfinal=None, dtype="float32"):
    """One sequence: a, x [T, C], h0 [C], all float64.  Values, gradients, error bounds before the rounding of the outputs.
    (The gradient of a gate of 16 bits is made with the state before it as the forward pass returned it, rounded to those bits.)

    REAL: h_t is a sum of products of at most t gates; a term with n gates has been through at most n + 24 roundings (its gates, the
    joins of wave, tile and chunk), so |error| <= 2 u (N + 24 M), M = sum |terms|, N = sum n |terms|.  A state below the smallest
    normal number is rounded to a multiple of 2^-149 whatever its size; gates above 1 make these errors grow as they make the terms
    grow: D = |a| D + 2^-149 a step, 24 D with the joins.  (A sequence that falls to 2^-230 and rises again by 2^200 is lost in 32
    bits step by step as well: 2^-230 is 0 there.)
    LOG: a step rounds a + h, the maximum and the sum (u |a + h|, u |h| and 4 u for the logarithm of a sum in [1, 2]) and passes the
    error before it on with the share w <= 1; the joins of wave, tile and chunk each add as much again, hence the factor 8."""
    T, C = x.shape
    h, M, N, E = np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C))
    now, m, n, e = h0.copy(), np.abs(h0), np.zeros(C), np.zeros(C)
    D, d = np.zeros((T, C)), np.zeros(C)
    size = lambda v: np.where(np.isfinite(v), np.abs(v), 0.0)  # noqa: E731
    with np.errstate(all="ignore"):
        for t in range(T):
            if s == REAL:
                d = np.abs(a[t]) * d + LEAST
                n, m = np.abs(a[t]) * (n + m) + np.abs(x[t]), np.abs(a[t]) * m + np.abs(x[t])
            before, now = now, _step(s, a[t], now, x[t])
            if s == LOG:
                w, _ = _shares(a[t], before, x[t])
                e = w * (e + U * size(a[t] + before)) + U * (4 + 2 * size(now))
            elif s == MAX:
                e = e + U * (size(a[t] + before) + size(a[t]))
            h[t], M[t], N[t], E[t], D[t] = now, m, n, e, d
    tol = 2 * U * (N + 24 * M) + 24 * D if s == REAL else 8 * E
    out = {"h": h, "h_tol": tol, "final": now, "final_tol": tol[-1] if T else np.zeros(C)}
    if dh is None:
        return out
    da, dx, da_tol, dx_tol = (np.zeros((T, C)) for _ in range(4))
    c, cm, cn, cd = dfinal.copy(), np.abs(dfinal), np.zeros(C), np.zeros(C)
    with np.errstate(all="ignore"):
        for t in range(T - 1, -1, -1):
            prev = h[t - 1] if t else h0
            prev_tol = tol[t - 1] + (REL[dtype] * np.abs(prev) + TINY[dtype] if dtype != "float32" else 0.0) if t else 0.0
            g, gm, gn = dh[t] + c, np.abs(dh[t]) + cm, np.abs(dh[t]) + cn + cm
            g_tol = 2 * U * (gn + 24 * gm) + 24 * cd
            if s == REAL:
                da[t], dx[t] = g * prev, g
                da_tol[t], dx_tol[t] = g_tol * np.abs(prev) + gm * prev_tol + 4 * U * np.abs(da[t]), g_tol
                c, cm, cn, cd = a[t] * g, np.abs(a[t]) * gm, np.abs(a[t]) * gn, np.abs(a[t]) * cd + LEAST
            else:
                w, v = _shares(a[t], prev, x[t])
                # a share is off by what the difference a + h - x of its logarithms is, and by the six operations that make it
                d = 2 * (prev_tol + U * (size(a[t]) + size(prev) + size(x[t]) + size(a[t] + prev)) + 6 * U)
                da[t], dx[t] = g * w, g * v
                c, cm, cn = g * w, gm * w, (gn + gm * d / U) * w
                da_tol[t], dx_tol[t] = 2 * U * (cn + 24 * cm), 2 * U * ((gn + gm * d / U) * v + 24 * gm * v)
    out.update(da=da, dx=dx, da_tol=da_tol, dx_tol=dx_tol, dinitial=c, dinitial_tol=2 * U * (cn + 24 * cm) + 24 * cd)
    return out


def close(got, want, tol, dtype="float32", what=""):
    """|got - want| <= tol + the rounding into dtype; infinities and NaN where `want` has them."""
    got, want, tol = np.asarray(got, np.float64), np.asarray(want, np.float64), np.asarray(tol, np.float64)
    assert got.shape == want.shape, "%s: shape %s, not %s" % (what, got.shape, want.shape)
    odd = ~np.isfinite(want)
    np.testing.assert_array_equal(got[odd], want[odd], err_msg=what)
    assert np.isfinite(got[~odd]).all(), what + ": not finite"
    bound = (np.broadcast_to(tol, want.shape) + REL[dtype] * np.abs(want) * (1 + 1e-6) + TINY[dtype])[~odd]
    err = np.abs(got[~odd] - want[~odd])
    if err.size:
        worst = (err / bound).max()
        assert worst <= 1.0, "%s: %.3g times its bound (off by %.3g)" % (what, worst, err[(err / bound).argmax()])
