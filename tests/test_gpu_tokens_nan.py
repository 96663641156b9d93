"""Rows of NaN (GPU): whatever is asked of a row that holds a NaN answers NaN, and so does every entry of its gradient; also where nothing in
the row is a number, or nothing but -inf.  Row lengths of every kernel: a quarter of a wave, a wave, one workgroup, several."""
import pytest
import torch

pytestmark = pytest.mark.gpu

ROWS = 8
NAN_ROWS = [1, 2, 3, 6]


def make(vocab, dtype):
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn((ROWS, vocab), generator=gen, device="cuda").to(dtype)
    x[1] = float("nan")                                  # whole
    x[2] = -float("inf")
    x[2, vocab - 1] = float("nan")                       # a NaN in a row that allows nothing
    x[3, vocab // 2] = float("nan")                      # one among numbers
    x[4] = -float("inf")                                 # a row that allows nothing: no gradient
    x[5] = float("nan")                                  # nothing is asked of it
    x[6, 0] = float("inf")
    tokens = torch.randint(0, vocab, (ROWS, 2), generator=gen, device="cuda")
    tokens[5] = -1
    return x.requires_grad_(True), tokens


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", [1, 30, 64, 65, 300, 513, 3001, 20011, 300001])
@pytest.mark.parametrize("what", ["logp", "neg", "entropy"])
def test_asked_rows_of_nan(what, vocab, dtype):
    import paper_2410_11415_amd as klay
    x, tokens = make(vocab, dtype)
    r = klay.token_logprobs(x, tokens, complement=what == "neg", entropy=what == "entropy")
    out = getattr(r, what)
    mine = out.detach().reshape(ROWS, -1)
    weight = torch.ones_like(out)
    if what == "entropy":
        weight[5] = 0.0
    dx, = torch.autograd.grad(out, x, weight)
    for row in range(ROWS):
        nan = row in NAN_ROWS
        assert bool(torch.isnan(mine[row]).all()) == (nan or (row == 5 and what == "entropy")), row
        assert bool(torch.isnan(dx[row]).all()) == nan and bool(torch.isnan(dx[row]).any()) == nan, row
    assert not dx[4].any() and not dx[5].any()


@pytest.mark.parametrize("vocab", [30, 300, 3001, 300001])
def test_adjoints_of_zero(vocab):
    """an adjoint of exactly 0 contributes 0, whatever the row holds"""
    import paper_2410_11415_amd as klay
    x, tokens = make(vocab, torch.float32)
    r = klay.token_logprobs(x, tokens, complement=True, entropy=True)
    dx, = torch.autograd.grad([r.logp, r.neg, r.entropy], x, [torch.zeros_like(t) for t in (r.logp, r.neg, r.entropy)])
    assert not dx.any()
