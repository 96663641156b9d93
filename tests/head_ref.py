"""Plain 64-bit definitions (torch, on any device) of the losses that take a network's head along and of the divergence from a teacher's list,
with bounds on the kernels' errors that follow from the arithmetic.

u = 2^-24 is half a step of fp32.  A logit is a sum of D products, each rounded addition off by at most u of sum |h w|: off by `slip`
= (2 D + 16) u max_j sum_d |h_d w_jd| in a row (fp32 operands go through as six products of their parts: hence the 2).  The log probability
of a token and that of its negation change by no more than twice the largest change of a logit, a divergence by that over T, the entropy by
2 H of it; what is made of the logits adds `terms(V)` as in operators_ref.  An adjoint of a logit is a product of probabilities, each off by
what its logarithm is off by, and is rounded to the operands' type; the products with weights and hidden states are sums again.
"""
import torch

U = 2.0 ** -24
REL = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1.2e-38, torch.bfloat16: 1.2e-38, torch.float16: 2.0 ** -25}


def terms(vocab):
    return U * (vocab / 256 + 64)


def _safe(t):
    return torch.where(torch.isfinite(t), t.abs(), 0.0)


def logits_of(hidden, weight, bias):
    """[R, V] and the rows' slip."""
    h, w = hidden.detach().double(), weight.detach().double()
    x = h @ w.t().contiguous()
    slip = (2 * h.shape[1] + 16) * U * (h.abs() @ w.abs().t().contiguous()).amax(1)
    if bias is not None:
        b = bias.detach().double()
        x = torch.where(b == -torch.inf, -torch.inf, x + b)
        slip = slip + 2 * U * _safe(x).amax(1)
    return x, slip


def tokens(x, t, slip, dlogp=None, dneg=None, dent=None):
    """Values of rows x [R, V] and, with adjoints, (dx, its magnitude); each value with its tolerance."""
    R, V = x.shape
    ask, bad, i = (t >= 0) & (t < V), t >= V, t.clamp(0, V - 1)
    m = x.amax(1, keepdim=True)
    some = m[:, 0] > -torch.inf
    at = torch.where(m > -torch.inf, m, 0.0)
    lp = torch.where(some[:, None], (x - at) - torch.logsumexp(x - at, 1, keepdim=True), -torch.inf)
    p = lp.exp()
    plogp = torch.where(p > 0, p * lp, 0.0)
    H = -plogp.sum(1)
    K = t.shape[1]
    rest = torch.ones(R, K, dtype=x.dtype, device=x.device)
    for k in range(K):
        rest[:, k] = torch.where(some, p.scatter(1, i[:, k:k + 1], 0.0).sum(1), 1.0)
    logp = torch.where(ask, lp.gather(1, i), torch.where(bad, torch.nan, 0.0))
    neg = torch.where(ask, rest.log(), torch.where(bad, torch.nan, 0.0))
    s = slip[:, None]
    spread = torch.where(p > 0, p * (x - at).abs(), 0.0).sum(1)
    out = {"logp": (logp, 2 * s + terms(V) + 4 * U * _safe(logp)), "neg": (neg, 2 * s + terms(V) + 4 * U * _safe(neg)),
           "entropy": (H, 2 * H * slip + terms(V) * (12 + spread))}
    if dlogp is None and dneg is None and dent is None:
        return out, None, None
    dx, mass = torch.zeros_like(x), torch.zeros_like(x)
    for k in range(K):
        on = ask[:, k:k + 1] & some[:, None]
        one = torch.zeros_like(x).scatter(1, i[:, k:k + 1], 1.0)
        pk, r = p.gather(1, i[:, k:k + 1]), rest[:, k:k + 1]
        if dlogp is not None:
            g = torch.where(on, dlogp[:, k:k + 1], 0.0)
            dx += g * torch.where(one > 0, r, -p)
            mass += g.abs() * torch.where(one > 0, r, p)
        if dneg is not None:
            n = torch.where(on, dneg[:, k:k + 1], 0.0)
            q = torch.where((one == 0) & (r > 0), p / r, 0.0)
            dx += n * pk * (q - one)
            mass += n.abs() * pk * (q + one)
    if dent is not None:
        h = torch.where(some, dent, 0.0)[:, None]
        dx -= h * (plogp + p * H[:, None])
        mass += h.abs() * (plogp.abs() + p * (H[:, None] + 12 + spread[:, None]))
    steps = torch.where(p > 0, 4 * U * _safe(lp), 0.0)
    return out, dx, mass * (2 * (terms(V) + K * U + steps) + 8 * s)


def distill(x, t, teacher, temperature, rest, slip, dloss=None):
    """loss (with its tolerance), dx and its tolerance before any rounding to the operands' type."""
    R, V = x.shape
    there, bad, i = (t >= 0) & (t < V), (t >= V).any(1), t.clamp(0, V - 1)
    T = temperature
    lp = torch.log_softmax(x / T, 1)
    p = lp.exp()
    z = teacher.double().masked_fill(~there, -torch.inf)
    some = (t >= 0).any(1)
    if not rest:
        z = z / T
        top = z.amax(1, keepdim=True)
        top = torch.where(top > -torch.inf, top, 0.0)
        z = (z - top) - torch.logsumexp(z - top, 1, keepdim=True)
        some = some & there.any(1)
    q = torch.where(there, z.exp(), 0.0)
    student = lp.gather(1, i)
    loss = torch.where(q > 0, q * (z - student), 0.0).sum(1)
    size = torch.where(q > 0, q * (z.abs() + student.abs()), 0.0).sum(1)
    listed = torch.zeros_like(x)
    for k in range(t.shape[1]):
        listed.scatter_(1, i[:, k:k + 1], torch.maximum(listed.gather(1, i[:, k:k + 1]), there[:, k:k + 1].double()))
    others = torch.where(listed > 0, 0.0, p)
    left = others.sum(1)
    q_left = torch.where(left > 0, (1 - q.sum(1)).clamp(min=0), 0.0) if rest else torch.zeros_like(left)
    loss = loss + torch.where(q_left > 0, q_left * (q_left / left).log(), 0.0)
    loss = torch.where(some, loss, 0.0)
    loss = torch.where(bad, torch.nan, loss)
    # the only sums in 32 bits: the mass of the others (terms), the rounding of x - ref (u |x|) times T; the rest is in 64 bits and rounded once
    far = 4 * U * _safe(x).amax(1) / T
    tol = 2 * slip / T + 2 * terms(V) + far + 2 * U * (_safe(loss) + size)
    if dloss is None:
        return (loss, tol), None, None
    target = torch.zeros_like(x).scatter_add_(1, i, q)
    share = torch.where(left > 0, q_left / left, 0.0)[:, None] * others
    on = some[:, None]
    g = dloss[:, None] / T
    # each q pulls its own answer up against all of them: p counts as often as the q add up to (1 but for lists of more, and for ones that no rest completes)
    p = p * (q.sum(1) + q_left)[:, None]
    dx = torch.where(on, (p - target - share) * g, 0.0)
    mass = torch.where(on, (p + target + share) * g.abs(), 0.0)
    steps = torch.where(p > 0, 4 * U * _safe(lp), 0.0)
    # (1 - P) - q_left is kept as one number: what the two are off by goes to the others by their shares.  A share below fp32's normal range, 2^-126,
    # counts as 0 (the exponential of the vector unit gives no denormals): with |A| <= |dloss| / T an entry is off by at most |dloss| / T 2^-126
    return (loss, tol), dx, torch.where(on, g.abs(), 0.0) * 2.0 ** -126 + mass * (4 * terms(V) + 2 * steps + 2 * far[:, None] + 8 * slip[:, None] / T)


def gradients(dx, dx_tol, hidden, weight):
    """What goes to hidden, weight and bias: {name: (value, tolerance)}."""
    h, w = hidden.detach().double(), weight.detach().double()
    dtype = hidden.dtype
    R, V = dx.shape
    live = (dx != 0).any(1, keepdim=True)
    h = torch.where(live, h, 0.0)                      # (a row without a gradient gives none, whatever it holds)
    off = dx_tol + (REL[dtype] if dtype != torch.float32 else 2.0 ** -23) * (dx.abs() + dx_tol)
    if dtype == torch.float16:
        off = off + dx.abs().max() * 2.0 ** -37         # scaled to 2^13 and above; the least step of fp16 is 2^-24
    adx = dx.abs()
    out = {"dhidden": (dx @ w, off @ w.abs() + (2 * V + 64) * U * (adx @ w.abs())),
           "dweight": (dx.t().contiguous() @ h, off.t().contiguous() @ h.abs() + (2 * R + 64) * U * (adx.t().contiguous() @ h.abs())),
           "dbias": (dx.sum(0), dx_tol.sum(0) + (R + 64) * U * adx.sum(0))}
    return out


def close(got, want, dtype=torch.float32, what=""):
    """got against (value, tolerance): infinities and NaN in the same places, the rest within tolerance and one rounding to dtype."""
    value, tol = want
    got = got.detach().double()
    assert got.shape == value.shape, (what, got.shape, value.shape)
    odd = ~torch.isfinite(value)
    assert torch.equal(torch.isnan(got), torch.isnan(value)), what + ": NaN elsewhere"
    assert torch.equal(got[odd & ~torch.isnan(value)], value[odd & ~torch.isnan(value)]), what + ": infinities elsewhere"
    err = torch.where(odd, 0.0, (got - value).abs())
    room = torch.where(odd, 1.0, tol + REL[dtype] * (value.abs() + tol) + TINY[dtype])
    worst = (err / room).max() if err.numel() else torch.zeros(())
    assert float(worst) <= 1.0, "%s: %.3g of the tolerance (error %.3g)" % (what, float(worst), float(err.max()))
