"""The operators (GPU) past 32-bit offsets and past one grid: the last rows and sequences of arrays of more than 2^31 elements, and of
more rows than a launch has workgroups, against the same rows by themselves."""
import pytest
import torch

from tests import operators_ref as ref

pytestmark = pytest.mark.gpu


def klay():
    import paper_2410_11415_amd as pkg
    return pkg


def test_tokens_past_32_bits():
    k = klay()
    rows, vocab = 70000, 32771
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.empty((rows, vocab), dtype=torch.bfloat16, device="cuda").normal_(0, 2, generator=gen)
    assert x.numel() > 1 << 31
    x.requires_grad_(True)
    t = torch.randint(0, vocab, (rows, 2), generator=gen, device="cuda")
    r = k.token_logprobs(x, t, complement=True, entropy=True)
    dx, = torch.autograd.grad([r.logp, r.neg, r.entropy], x, [torch.ones_like(r.logp), torch.ones_like(r.neg), torch.ones_like(r.entropy)])
    for part in (slice(0, 600), slice(rows - 600, rows)):
        y = x.detach()[part].clone().requires_grad_(True)
        q = k.token_logprobs(y, t[part], complement=True, entropy=True)
        dy, = torch.autograd.grad([q.logp, q.neg, q.entropy], y, [torch.ones_like(q.logp), torch.ones_like(q.neg), torch.ones_like(q.entropy)])
        assert torch.equal(r.logp[part], q.logp) and torch.equal(r.neg[part], q.neg) and torch.equal(r.entropy[part], q.entropy)
        assert torch.equal(dx[part], dy)


@pytest.mark.parametrize("rows,vocab", [((1 << 20) + 777, 530), ((1 << 25) + 5, 3)])
def test_more_rows_than_workgroups(rows, vocab):
    k = klay()
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((rows, vocab), device="cuda").normal_(0, 2, generator=gen).requires_grad_(True)
    t = torch.randint(0, vocab, (rows, 1), generator=gen, device="cuda")
    r = k.token_logprobs(x, t, entropy=True)
    dx, = torch.autograd.grad([r.logp, r.entropy], x, [torch.ones_like(r.logp), torch.ones_like(r.entropy)])
    part = slice(rows - 3000, rows)
    y = x.detach()[part].clone().requires_grad_(True)
    q = k.token_logprobs(y, t[part], entropy=True)
    dy, = torch.autograd.grad([q.logp, q.entropy], y, [torch.ones_like(q.logp), torch.ones_like(q.entropy)])
    # A row of 530 fp32 starts at another place within 16 bytes in the whole array than by itself, so its terms meet in another order: either
    # result is off by its bound at most, and the two differ by twice that (distances from the maximum: below 30)
    tol = 2 * ref.terms(vocab)
    assert float(((r.logp[part] - q.logp).abs() - 8 * ref.U * q.logp.abs()).max()) <= tol
    assert float((r.entropy[part] - q.entropy).abs().max()) <= tol * (12 + 30)
    # an entry: itself <= 1, and p (|ln p| + H) <= 1 with the entropy's error, times two for p's own
    assert float((dx[part] - dy).abs().max()) <= 2 * tol * (12 + 30)


@pytest.mark.parametrize("batch,time,channels", [(600, 70, 52000), (3, 12000, 62000), (1, 40000, 56000)])
def test_scan_past_32_bits(batch, time, channels):
    k = klay()
    gen = torch.Generator(device="cuda").manual_seed(2)
    a = torch.empty((batch, time, channels), dtype=torch.bfloat16, device="cuda").uniform_(0, 1, generator=gen)
    x = torch.empty_like(a).normal_(0, 1, generator=gen)
    assert a.numel() > 1 << 31
    leaves = [a.requires_grad_(True), x.requires_grad_(True)]
    h, final = k.gated_scan(*leaves)
    dh = torch.ones_like(h)
    da, dx = torch.autograd.grad([h, final], leaves, [dh, torch.ones_like(final)])
    for b in {0, batch - 1}:
        cut = slice(channels - 130, channels)
        parts = [t.detach()[b:b + 1, :, cut].clone().requires_grad_(True) for t in (a, x)]
        g, last = k.gated_scan(*parts)
        ga, gx = torch.autograd.grad([g, last], parts, [torch.ones_like(g), torch.ones_like(last)])
        # (the steps meet in another order there: the states differ by fp32's rounding, and where that decides, by one of bf16)
        for p, q in ((h[b:b + 1, :, cut], g), (final[b:b + 1, cut], last), (da[b:b + 1, :, cut], ga), (dx[b:b + 1, :, cut], gx)):
            assert torch.allclose(p.float(), q.float(), rtol=2.0 ** -6, atol=1e-3)


def test_step_past_32_bits():
    k = klay()
    batch, channels = 70000, 31000
    a = torch.full((batch, channels), 0.5, dtype=torch.bfloat16, device="cuda")
    x = torch.ones_like(a)
    state = torch.full((batch, channels), 2.0, device="cuda")
    assert state.numel() > 1 << 31
    out = k.gated_step(a, x, state)
    assert bool((state[-3:] == 2.0).all()) and bool((out[-3:] == 2.0).all())
    x[-1] = 3.0
    k.gated_step(a, x, state, out=out)
    assert bool((state[-1] == 4.0).all()) and bool((out[-1] == 4.0).all()) and bool((state[-2] == 2.0).all())


def test_the_longest_row():
    """2^31 - 1 logits: all 0 but a few.  Sums of ones are exact in fp32 up to 2^24 and off by 2^-24 a join above; with what the change of
    the reference costs (a factor that is off by 2^-22) the logarithm of the sum is off by less than 1e-5."""
    k = klay()
    vocab = (1 << 31) - 1
    x = torch.zeros((1, vocab), dtype=torch.bfloat16, device="cuda")
    best = [vocab - 1, vocab - 9, 5, vocab // 2, vocab - 4097]
    value = torch.tensor([20.0, 19.0, 18.0, 17.0, 16.0], dtype=torch.float64)
    for j, v in zip(best, value.tolist()):
        x[0, j] = v
    x.requires_grad_(True)
    t = torch.tensor([best + [7]], device="cuda")
    r = k.token_logprobs(x, t, entropy=True, top=6)
    total = (vocab - 5) + value.exp().sum()
    lp = torch.cat([value, torch.zeros(1, dtype=torch.float64)]) - total.log()
    assert float((r.logp[0].detach().cpu().double() - lp).abs().max()) <= 1e-5 + 32 * ref.U
    entropy = total.log() - (value.exp() * value).sum() / total
    assert abs(float(r.entropy[0].detach()) - float(entropy)) <= 1e-5 * 32
    assert r.top_tokens[0].tolist() == best + [0]
    dx, = torch.autograd.grad(r.logp[:, 0].sum(), x)
    p = lp.exp()
    want = torch.tensor([1 - p[0]] + [-q for q in p[1:5]] + [-p[5]], dtype=torch.float64)
    got = dx[0, torch.tensor(best + [vocab - 2], device="cuda")].cpu().double()
    assert ((got - want).abs() <= (2.0 ** -8 + 1e-4) * want.abs()).all()
    assert int((dx[0] == dx[0, 0]).sum()) == vocab - 5 and bool(dx[0, 0] < 0)
