"""Token log probabilities of sure rows (GPU): one token leads the others by 15 to 10^4 and by the type's whole range, so that its p rounds to 1
and the others' share R = (1 - p) / p of the mass is all there is to say about the row; down to where R itself has no place in fp32.

Bounds.  u = 2^-24, gap_j = M - x_j.  A term e^-gap is off by 4 u gap relative (the difference, the constant, the product, the reference) and a sum
of V of them by T = terms(V) on top; so
  R: T + 4 u G relative, G the mean gap of R's terms;  logp = -log1p(R), where p > 1/2: the same, and 4 u for the logarithm
  neg = (M2 - M) + ln R2 - ln S: u |neg| a rounding, T for R2
  entropy = log1p(R) + sum e^-gap gap / S: as R, with the mean gap of its own terms
  gradient: each share is a product of such numbers, so T + 8 u (1 + gap) of it, gap taken to the next largest logit where R is held that way.
What is below fp32's normal range is flushed, up to 1.2e-38 a term: R and with it logp lose up to V of them, the entropy (whose terms are multiplied by
gaps of about 100 there) up to 100 V, and its gradient as much.  (8 u in place of 4 u above leaves room for the outermost roundings.)"""
import numpy as np
import pytest
import torch

from tests import operators_ref as ref

pytestmark = pytest.mark.gpu
U, TINY = ref.U, 1.2e-38


def exact(x, t, dlogp, dneg, dent):
    """One row in 64 bits: x [V], t [K]; values, gradient, and how far fp32 may be off."""
    V, K, T = x.size, t.size, ref.terms(x.size)
    M = x.max()
    with np.errstate(all="ignore"):
        d = x - M
        e = np.exp(d)
        best = int(x.argmax())
        others = np.delete(e, best)
        far = np.delete(np.where(e > 0, -d, 0.0), best)
        R = others.sum()
        ln_s = np.log1p(R)
        mean = lambda w: float((w * far).sum() / w.sum()) if w.sum() > 0 else 0.0  # noqa: E731
        H = ln_s + (others * far).sum() / (1 + R)
        lp, p = d - ln_s, e / (1 + R)
    out = {"entropy": H, "entropy_tol": (T + 8 * U * (1 + mean(others * far))) * H + V * 100 * TINY}
    flush = np.where(e > 0, -d, 0.0)
    logp, neg, logp_tol, neg_tol = (np.zeros(K) for _ in range(4))
    dx, tol = np.zeros(V), np.zeros(V)
    for k in range(K):
        j = int(t[k])
        sure = j == best
        logp[k] = -ln_s if sure else lp[j]
        logp_tol[k] = (T + 8 * U * (1 + mean(others))) * ln_s if sure else T + 4 * U * (abs(lp[j]) if np.isfinite(lp[j]) else 0.0)
        rest = np.delete(x, j)
        m2 = rest.max() if rest.size else -np.inf
        with np.errstate(all="ignore"):
            e2 = np.exp(x - m2) if m2 > -np.inf else np.zeros(V)
            e2[j] = 0.0
            neg[k] = (m2 - M) + np.log(e2.sum()) - ln_s if m2 > -np.inf else -np.inf
        neg_tol[k] = T + 8 * U * (abs(neg[k]) if np.isfinite(neg[k]) else 0.0)
        share = e2 / e2.sum() if m2 > -np.inf else e2       # e^(x_j - M2) / R2, without the token
        one = np.zeros(V)
        one[j] = 1.0
        held = sure and R < 2.0 ** -64
        with np.errstate(all="ignore"):
            away = np.exp(neg[k])
            off = T + 8 * U * (1 + np.where(share > 0, m2 - x if held else flush, 0.0)) + K * U
            dx += dlogp[k] * (one * away - (1 - one) * p)
            tol += abs(dlogp[k]) * (one * away * (T + 8 * U * (1 + mean(others))) + (1 - one) * p * (T + 8 * U * (1 + flush)))
            dx += dneg[k] * p[j] * (share - one)
            tol += abs(dneg[k]) * p[j] * (share * off + one * (T + 8 * U * (1 + flush[j])))
    with np.errstate(all="ignore"):
        plogp = np.where(p > 0, p * lp, 0.0)
    dx -= dent * (plogp + p * H)
    tol += abs(dent) * p * (np.where(p > 0, np.abs(lp), 0.0) + H) * (T + 8 * U * (1 + np.maximum(flush, mean(others * far))))
    out.update(logp=logp, neg=neg, logp_tol=logp_tol + V * TINY, neg_tol=neg_tol, dx=dx,
               dx_tol=tol + (K * (1 + np.abs(dlogp).sum()) + 100 * V * abs(dent)) * TINY)
    return out


def rows_of(kind, rows, vocab, dtype, rng):
    """logits (in the type, as float64) and the place of each row's best token"""
    low = float(torch.finfo(getattr(torch, dtype)).min)
    x = rng.normal(size=(rows, vocab))
    best = rng.integers(0, vocab, size=rows)
    best[0], best[-1] = 0, vocab - 1
    at = np.arange(rows)
    if kind == "lowest":
        x[:] = low
        x[at, best] = 3.0
    elif kind == "lone":                                 # one other token is allowed, somewhere
        x[:] = -np.inf
        x[at, (best + 1 + rng.integers(0, max(1, vocab - 1), size=rows)) % vocab] = -9000.0
        x[at, best] = 3.0
    elif kind == "alone":                                # none
        x[:] = -np.inf
        x[at, best] = 3.0
    else:
        x -= MIXED[at % len(MIXED), None] if kind == "mixed" else kind
        x[at, best] = rng.uniform(2, 4, size=rows)
    x = torch.from_numpy(x).to(getattr(torch, dtype))
    return x, x.double().numpy(), best


def check(kind, rows, vocab, dtype, complement=True, entropy=True, looked_at=None):
    import paper_2410_11415_amd as klay
    rng = np.random.default_rng(vocab)
    x, x64, best = rows_of(kind, rows, vocab, dtype, rng)
    K = 4
    t = rng.integers(0, vocab, size=(rows, K))
    t[:, 0] = best
    t[::2, 2] = best[::2]                                # in some rows twice
    f32 = lambda *s: rng.normal(size=s).astype(np.float32)  # noqa: E731
    dlogp, dneg, dent = f32(rows, K), f32(rows, K) * complement, f32(rows) * entropy
    dlogp[rows // 2] = 0.0                               # in one row the negated literals are alone
    logits = x.cuda().requires_grad_(True)
    got = klay.token_logprobs(logits, torch.from_numpy(t).cuda(), complement=complement, entropy=entropy)
    outs, grads = [got.logp], [dlogp]
    if complement:
        outs, grads = outs + [got.neg], grads + [dneg]
    if entropy:
        outs, grads = outs + [got.entropy], grads + [dent]
    dx, = torch.autograd.grad(outs, logits, [torch.from_numpy(g).cuda() for g in grads])
    n = lambda v: v.detach().double().cpu().numpy()  # noqa: E731
    for r in looked_at or range(rows):
        want = exact(x64[r], t[r], dlogp[r].astype(float), dneg[r].astype(float), float(dent[r]))
        what = "row %d " % r
        ref.close(n(got.logp[r]), want["logp"], want["logp_tol"], what=what + "logp")
        if complement:
            ref.close(n(got.neg[r]), want["neg"], want["neg_tol"], what=what + "neg")
        if entropy:
            ref.close(n(got.entropy[r]), np.array(want["entropy"]), np.array(want["entropy_tol"]), what=what + "entropy")
        ref.close(n(dx[r]), want["dx"], want["dx_tol"], dtype, what + "dlogits")


MIXED = np.array([0.0, 60.0, 5.0, 15.0, 1e4, 1.0, 46.0, 95.0])
KINDS = [15.0, 25.0, 40.0, 46.0, 80.0, 90.0, 110.0, 1e4, "lowest", "lone", "alone"]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("vocab", [2, 3, 40, 64, 65, 300, 512, 513, 3001, 20011])
@pytest.mark.parametrize("kind", KINDS)
def test_sure_rows(kind, vocab, dtype):
    check(kind, 5, vocab, dtype)


@pytest.mark.parametrize("complement,entropy", [(False, True), (False, False), (True, False)])
@pytest.mark.parametrize("vocab", [10, 400, 2500])
@pytest.mark.parametrize("kind", [15.0, 30.0, 60.0, 100.0])
def test_what_is_asked(kind, vocab, complement, entropy):
    check(kind, 4, vocab, "float32", complement, entropy)


@pytest.mark.parametrize("dtype,vocab", [("float32", 300001), ("bfloat16", 600007), ("float16", 270001)])
@pytest.mark.parametrize("kind", [25.0, 60.0, 95.0, 1e4, "lowest", "lone", "alone"])
def test_rows_of_several_workgroups(kind, dtype, vocab):
    check(kind, 3, vocab, dtype)


@pytest.mark.parametrize("kind", [25.0, 95.0, 1e4, "lowest"])
@pytest.mark.parametrize("vocab", [50, 700, 9001])
def test_many_rows(kind, vocab):
    check(kind, 600, vocab, "float32", looked_at=[0, 1, 299, 300, 598, 599])


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("vocab", [10, 64, 300, 700, 5000])
def test_sure_rows_beside_others(vocab, dtype):
    """(four rows of up to 64 logits share a wave)"""
    check("mixed", 40, vocab, dtype)


def test_the_circuit_of_a_sure_answer():
    """a finite mask leaves a negated literal possible: log weights of -1e4, not -inf"""
    import paper_2410_11415_amd as klay
    x = torch.full((1, 6), -1e4, device="cuda")
    x[0, 2] = 0.0
    r = klay.token_logprobs(x, torch.tensor([[2, 3]], device="cuda"), complement=True)
    assert abs(float(r.neg[0, 0]) - (-1e4 + np.log(5.0))) <= 1e4 * 4 * U and float(r.neg[0, 1]) == 0.0
