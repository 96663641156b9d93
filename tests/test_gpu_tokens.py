"""Log probabilities of given tokens (GPU) against the 64-bit definition: values, alternatives, gradients; row lengths around the
kernels' vectors, lane groups and row parts, every type, masks, sure rows, padding, layouts."""
import numpy as np
import pytest
import torch

from tests import operators_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = ["float32", "bfloat16", "float16"]


def klay():
    import paper_2410_11415_amd as pkg
    return pkg


def make(rows, vocab, k, dtype, seed, kind="plain"):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, vocab)) * 2.5
    t = rng.integers(0, vocab, size=(rows, k))
    sure = rng.integers(0, vocab, size=rows)
    if kind in ("sure", "masked"):
        x[np.arange(rows), sure] += rng.uniform(0, 40, size=rows)
        if k:
            t[:, 0] = sure
    if kind == "masked":
        x[rng.random(x.shape) < 0.3] = -np.inf
        x[0] = -np.inf                                   # a row that allows nothing
        if rows > 1:
            x[1] = -np.inf
            x[1, vocab // 2] = 3.0                       # one that allows a single token
        t[rng.random(t.shape) < 0.2] = -1
        if rows > 2:
            t[2] = -100
    if kind == "ties":
        x = np.round(x)
    if kind == "equal":
        x[:] = 1.25
    if kind == "lowest":                                 # a mask of the type's lowest value, in some rows everywhere
        x[rng.random(x.shape) < 0.5] = torch.finfo(getattr(torch, dtype)).min
        x[0] = torch.finfo(getattr(torch, dtype)).min
    if kind == "rising":
        x = np.sort(x, axis=1)
    if kind == "falling":
        x = -np.sort(-x, axis=1)
    logits = torch.from_numpy(x).to(getattr(torch, dtype)).cuda()
    return logits, torch.from_numpy(t).cuda(), rng


def check(logits, tokens, rng, complement=True, entropy=True, top=0, grads=True, dtype="float32", view=None):
    x = logits.double().cpu().numpy()
    t = tokens.cpu().numpy()
    R, K = t.shape
    f32 = lambda *s: rng.normal(size=s).astype(np.float32)  # noqa: E731
    g = dict(dlogp=f32(R, K), dneg=f32(R, K) if complement else None, dent=f32(R) if entropy else None) if grads else {}
    with np.errstate(all="ignore"):
        want = ref.tokens(x, t, top=top, **{n: v.astype(np.float64) for n, v in g.items() if v is not None})
    given = (view(logits) if view else logits).detach()
    if grads:
        given.requires_grad_(True)
    got = klay().token_logprobs(given, tokens, complement=complement, entropy=entropy, top=top)
    for name in ["logp"] + ["neg"] * complement + ["entropy"] * entropy + ["top_logp"] * bool(top):
        ref.close(getattr(got, name).detach().cpu().numpy(), want[name], want[name + "_tol"], what=name)
    if top:
        np.testing.assert_array_equal(got.top_tokens.cpu().numpy(), want["top_tokens"])
    if grads:
        outs = [o for o, n in ((got.logp, "dlogp"), (got.neg, "dneg"), (got.entropy, "dent")) if g[n] is not None]
        dx, = torch.autograd.grad(outs, given, [torch.from_numpy(v).cuda() for v in g.values() if v is not None])
        assert dx.dtype == logits.dtype and dx.shape == logits.shape
        ref.close(dx.double().cpu().numpy(), want["dlogits"], want["dlogits_tol"], dtype, "dlogits")


# row lengths: one, around a lane group's 64 and 512, odd ones, around the vectors of a workgroup (1024 fp32, 2048 of 16 bits)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [1, 2, 3, 10, 16, 63, 64, 65, 257, 511, 512, 513, 1023, 1025, 2047, 2049, 4099, 8195])
def test_row_lengths(vocab, dtype):
    check(*make(5, vocab, 3, dtype, vocab), dtype=dtype, top=min(vocab, 7))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["sure", "masked", "ties", "equal", "lowest", "rising", "falling"])
@pytest.mark.parametrize("rows,vocab,k,top", [(7, 10, 10, 10), (6, 300, 5, 64), (5, 3001, 4, 64), (3, 20011, 2, 20), (1100, 700, 1, 5)])
def test_kinds_of_rows(rows, vocab, k, top, kind, dtype):
    check(*make(rows, vocab, k, dtype, rows + vocab, kind), dtype=dtype, top=top, grads=rows < 1000)


@pytest.mark.parametrize("complement,entropy,top", [(False, False, 0), (True, False, 0), (False, True, 0), (False, False, 3), (True, True, 1)])
@pytest.mark.parametrize("vocab", [12, 200, 1500, 9001])
def test_what_is_asked(vocab, complement, entropy, top):
    check(*make(4, vocab, 2, "float32", 3), complement=complement, entropy=entropy, top=top)


@pytest.mark.parametrize("vocab,k", [(40, 100), (600, 1024), (400, 333), (5000, 129)])
def test_many_tokens_and_the_same_ones_again(vocab, k):
    check(*make(2, vocab, k, "float32", k, "sure"))


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 131072, "bfloat16"), (2, 100003, "float32"), (1, 262145, "float16")])
def test_long_rows(rows, vocab, dtype):
    check(*make(rows, vocab, 2, dtype, 1, "sure"), dtype=dtype, top=64)


@pytest.mark.parametrize("vocab", [20, 700, 5003])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_layouts(vocab, dtype):
    logits, tokens, rng = make(6, vocab, 3, dtype, 2)

    def padded(t):                 # rows of a wider array, from an odd element on
        wide = torch.full((6, vocab + 13), 7.0, dtype=t.dtype, device="cuda")
        wide[:, 5:5 + vocab] = t
        return wide[:, 5:5 + vocab]
    check(logits, tokens, rng, dtype=dtype, view=padded, top=5)
    check(logits, tokens, rng, dtype=dtype, view=lambda t: t.t().contiguous().t(), top=5)       # copied
    check(logits, tokens.t().contiguous().t(), rng, dtype=dtype)
    check(logits[:1].expand(6, vocab), tokens, rng, dtype=dtype)
    check(logits, tokens[:1].expand(6, 3), rng, dtype=dtype)


def test_leading_axes():
    k = klay()
    logits = torch.randn(3, 5, 70, device="cuda")
    tokens = torch.randint(0, 70, (3, 5, 2), device="cuda")
    whole = k.token_logprobs(logits, tokens, entropy=True, top=4)
    shifted = k.token_logprobs(logits[:, :-1], tokens[:, 1:], entropy=True, top=4)              # as for next tokens
    again = k.token_logprobs(logits[:, :-1].contiguous(), tokens[:, 1:].contiguous(), entropy=True, top=4)
    assert whole.logp.shape == (3, 5, 2) and whole.entropy.shape == (3, 5) and whole.top_tokens.shape == (3, 5, 4)
    for a, b in zip(shifted, again):
        assert (a is None and b is None) or torch.equal(a, b)
    four = logits[:, :, None, :].expand(3, 5, 2, 70).transpose(0, 2)                              # more strides than two: copied
    r = k.token_logprobs(four, None, entropy=True)
    assert r.logp is None and torch.equal(r.entropy, whole.entropy[:, :, None].expand(3, 5, 2).transpose(0, 2))
    one = k.token_logprobs(logits[1, 2], tokens[1, 2], entropy=True)
    assert torch.equal(one.logp, whole.logp[1, 2]) and torch.equal(one.entropy, whole.entropy[1, 2])


def test_saved_tensors_that_come_back_with_other_strides():
    """what autograd saved may lie in the same place another way (hooks that keep it elsewhere meanwhile)"""
    x = torch.randn(40, 300, device="cuda")
    tokens = torch.randint(0, 300, (40, 2), device="cuda")
    results = []
    for moved in (False, True):
        base = torch.zeros((40, 310), device="cuda")
        base[:, :300] = x
        logits = base[:, :300].requires_grad_(True)

        def unpack(t):
            if not moved or t.data_ptr() != logits.data_ptr():
                return t
            flat = base.detach().flatten()[:x.numel()]
            flat.copy_(x.flatten())
            return flat.view(x.shape)
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
            out = klay().token_logprobs(logits, tokens).logp
        results.append(torch.autograd.grad(out.sum(), logits)[0])
    # (rows from other addresses are summed in another order: the shares differ by the roundings of a sum of at most 300 terms)
    assert (results[0] - results[1]).abs().max() <= 600 * 2.0 ** -24


def test_nothing_to_do():
    k = klay()
    r = k.token_logprobs(torch.empty((0, 9), device="cuda", requires_grad=True), torch.empty((0, 2), dtype=torch.int64, device="cuda"), top=3)
    assert r.logp.shape == (0, 2) and r.top_tokens.shape == (0, 3)
    x = torch.randn(4, 900, device="cuda", requires_grad=True)
    r = k.token_logprobs(x, torch.empty((4, 0), dtype=torch.int64, device="cuda"), complement=True, entropy=True)
    assert r.logp.shape == (4, 0) and r.neg.shape == (4, 0)
    r.entropy.sum().backward()
    assert torch.isfinite(x.grad).all()


@pytest.mark.parametrize("vocab", [30, 600, 6000])
def test_rows_without_a_question_are_not_read(vocab):
    """NaN in padded rows reaches neither the outputs nor the gradient; an out-of-range token, or a NaN in an asked row, does"""
    k = klay()
    x = torch.randn(6, vocab, device="cuda")
    x[1] = float("nan")
    x[2, vocab // 2] = float("nan")
    x[3, 1] = float("inf")
    x.requires_grad_(True)
    tokens = torch.tensor([[1, -1], [-1, -7], [2, 3], [1, 2], [0, vocab], [vocab - 1, 0]], device="cuda")
    r = k.token_logprobs(x, tokens, complement=True)
    nan = torch.tensor([[0, 0], [0, 0], [1, 1], [1, 1], [0, 1], [0, 0]], dtype=torch.bool)
    assert torch.equal(torch.isnan(r.logp).cpu(), nan) and torch.equal(torch.isnan(r.neg).cpu(), nan)
    assert float(r.logp[0, 1]) == 0.0 and float(r.neg[0, 1]) == 0.0
    dx, = torch.autograd.grad([r.logp, r.neg], x, [torch.ones_like(r.logp), torch.ones_like(r.neg)])
    assert not dx[1].any() and torch.isnan(dx[2]).all() and torch.isnan(dx[4]).all()
    assert torch.isfinite(dx[0]).all() and torch.isfinite(dx[5]).all()
    top = k.token_logprobs(x.detach(), None, top=5)
    assert bool(((top.top_tokens >= 0) & (top.top_tokens < vocab)).all())
    assert torch.isfinite(top.top_logp[[0, 4, 5]]).all() and torch.isnan(top.top_logp[[1, 2, 3]]).all()


@pytest.mark.parametrize("vocab", [25, 1300])
def test_gradient_against_differences(vocab):
    k = klay()
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((3, vocab), generator=gen, device="cuda")
    v = torch.randn((3, vocab), generator=gen, device="cuda")
    tokens = torch.randint(0, vocab, (3, 4), generator=gen, device="cuda")
    weights = [torch.randn(s, generator=gen, device="cuda").double() for s in ((3, 4), (3, 4), (3,))]

    def f(y):
        r = k.token_logprobs(y, tokens, complement=True, entropy=True)
        return sum((w * o.double()).sum() for w, o in zip(weights, (r.logp, r.neg, r.entropy)))
    y = x.clone().requires_grad_(True)
    f(y).backward()
    eps = 2.0 ** -6
    slope = float((f(x + eps * v) - f(x - eps * v)) / (2 * eps))
    # third derivatives of logp, neg, H along v are below 8 max|v|^3 times the weights; fp32's error of each value is divided by eps
    total, big = float(sum(w.abs().sum() for w in weights)), float(v.abs().max())
    tol = eps ** 2 / 6 * 8 * big ** 3 * total + total * (ref.terms(vocab) * 24) / eps
    assert abs(slope - float((y.grad.double() * v.double()).sum())) <= tol


def test_the_same_bits_every_time():
    k = klay()
    x = torch.randn(64, 50021, device="cuda", dtype=torch.float16).round_(decimals=1).requires_grad_(True)
    tokens = torch.randint(0, 50021, (64, 9), device="cuda")
    first = None
    for _ in range(4):
        r = k.token_logprobs(x, tokens, complement=True, entropy=True, top=20)
        dx, = torch.autograd.grad([r.logp, r.neg, r.entropy], x, [torch.ones_like(r.logp), torch.ones_like(r.neg), torch.ones_like(r.entropy)])
        now = list(r) + [dx]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
        first = now


@pytest.mark.parametrize("rows,vocab", [(2, 30000), (50, 40), (1100, 3000)])
def test_streams_and_graphs(rows, vocab):
    """two streams at once, and a captured forward and backward call replayed over new inputs, between eager calls"""
    k = klay()
    x = torch.randn(rows, vocab, device="cuda")
    tokens = torch.randint(0, vocab, (rows, 2), device="cuda")
    args = dict(complement=True, entropy=True, top=5)
    ones = torch.ones(rows, 2, device="cuda")

    def both(logits):
        r = k.token_logprobs(logits, tokens, **args)
        y = logits.detach().requires_grad_(True)
        q = k.token_logprobs(y, tokens, complement=True)
        return list(r) + list(torch.autograd.grad([q.logp, q.neg], y, [ones, ones]))
    inputs = [x * (i + 1) for i in range(4)]
    want = [both(i) for i in inputs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i, y in enumerate(inputs):
        with torch.cuda.stream(streams[i % 2]):
            got.append(both(y))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    fixed = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(streams[0]):
        both(fixed)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = both(fixed)
    for i in (1, 3, 0):
        fixed.copy_(inputs[i])
        graph.replay()
        eager = both(inputs[i])
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, eager)) and all(torch.equal(p, q) for p, q in zip(out, want[i]))
