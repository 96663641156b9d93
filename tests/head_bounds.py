"""What the gradients of a head may be off by, entry for entry, where the logits' adjoints are held in two numbers of the operands' type (one of fp32): the
results' own rounding, and next to nothing beside it.

u = 2^-24.  A matrix instruction adds sixteen products of 16 bits, or of parts of fp32, to a sum of fp32; four roundings in each, and 64 more for the joins,
are allowed: a sum of n terms is off by (n / 4 + 64) u of the sum of their magnitudes.  The logit of a row may be off by `slip` so, and a probability by four
times that of itself (its own logit and the logarithm of the sum, either way); the adjoint g (1 - p) of an asked token by g times what p is off by, and a few
steps of fp32.  A number of a type with relative error r leaves r of an adjoint, two leave r^2."""
import torch

from tests.head_ref import REL, TINY, U


def sum_of(n):
    return (n / 4 + 64) * U


def slip_of(hidden, weight):
    return sum_of(hidden.shape[1]) * (hidden.double().abs() @ weight.double().abs().t().contiguous()).amax(1, keepdim=True)


def adjoints(hidden, weight, tokens, d):
    """Of sum_i d_i logp of row i's one token: the logits' adjoints and what they may be off by."""
    x = hidden.double() @ weight.double().t().contiguous()
    p = torch.log_softmax(x, 1).exp()
    one = torch.zeros_like(x).scatter_(1, tokens, 1.0)
    d = d.double()[:, None]
    dx = d * torch.where(one > 0, p.scatter(1, tokens, 0.0).sum(1, keepdim=True), -p)
    return dx, d.abs() * (p * (4 * slip_of(hidden, weight) + 64 * U) + 8 * U * one)


def held(dx, dtype, numbers):
    """dx as `numbers` numbers of a type hold it (fp16: scaled by a power of two into its range, which is left out here)."""
    first = dx.to(dtype).double()
    return first if numbers == 1 else first + (dx - first).to(dtype).double()


def gradients(dx, off, hidden, weight, dtype):
    """{name: (value, tolerance before the rounding to its type)}"""
    h, w = hidden.double(), weight.double()
    size = dx.abs()
    off = off + REL[dtype] ** (1 if dtype == torch.float32 else 2) * size
    if dtype == torch.float16:
        off = off + 2.0 ** -38 * size.max()                     # (the largest comes to 2^13 at least, half a step is 2^-25 at least)
    dxt, offt, ht, = dx.t().contiguous(), off.t().contiguous(), h.abs()
    return {"dhidden": (dx @ w, off @ w.abs() + sum_of(2 * dx.shape[1]) * (size @ w.abs())),
            "dweight": (dxt @ h, offt @ ht + sum_of(2 * dx.shape[0]) * (size.t().contiguous() @ ht))}


def worst(got, want, dtype):
    """The largest error in units of what is allowed: the tolerance and one rounding."""
    value, tol = want
    return float(((got.double() - value).abs() / (tol + REL[dtype] * (value.abs() + tol) + TINY[dtype])).max())


def slip_by_sums(hidden, weight, bias=None):
    """What a row's logits may be off by, from the sums themselves: sixteen terms at a time join a sum S of fp32, with four roundings of S and of the magnitude of
    what joins it; fp32 operands go through as several products of their parts, twice that.  (Of wide rows the magnitudes of all terms say little: S is some
    steps of a walk, its terms together hundreds of times that.)"""
    h, w = hidden.double(), weight.double()
    s = torch.zeros(h.shape[0], w.shape[0], dtype=torch.float64, device=h.device)
    run = torch.zeros_like(s)
    for k in range(0, h.shape[1], 16):
        a, b = h[:, k:k + 16], w[:, k:k + 16].t().contiguous()
        s += a @ b
        run += s.abs() + a.abs() @ b.abs()
    slip = 4 * U * (2 if hidden.dtype == torch.float32 else 1) * run.amax(1)
    return slip if bias is None else slip + 2 * U * (s.abs().amax(1) + bias.double().abs().max())


def negated(x, t, slip, terms):
    """(log(1 - p) of row i's tokens, its tolerance): what p / (1 - p) of a change of the logarithm makes of it, and no more than all others together change."""
    p = torch.log_softmax(x, 1).exp()
    r = torch.stack([p.scatter(1, t[:, k:k + 1], 0.0).sum(1) for k in range(t.shape[1])], 1)
    neg = r.log()
    return neg, (p.gather(1, t) / r).clamp(max=1.0) * (4 * slip[:, None] + terms) + 8 * U * neg.abs()
