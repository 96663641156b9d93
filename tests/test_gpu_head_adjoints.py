"""Gradients of heads (GPU) whose results are made of few adjoints each: off by their own rounding and no more, whatever the number of rows and of terms."""
import pytest
import torch

from tests import head_bounds

pytestmark = pytest.mark.gpu


# few and many rows, products of few and of many terms, on both sides of 256 rows, of 2^32 terms and of a piece of the vocabulary
SIZES = [(1, 512, 300), (40, 256, 600), (64, 1024, 16400), (256, 2048, 8300), (257, 2048, 8300), (300, 512, 28000), (1100, 2048, 2000), (2100, 128, 20011)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=lambda v: str(v).replace("torch.", ""))
@pytest.mark.parametrize("rows,width,vocab", SIZES)
@pytest.mark.parametrize("distilled", [False, True], ids=["logprobs", "distilled"])
def test_one_adjoint_a_result(rows, width, vocab, dtype, distilled):
    """every row asks for a token of its own: its adjoint nearly alone makes a row of either gradient"""
    import paper_2410_11415_amd as klay
    g = torch.Generator(device="cuda").manual_seed(rows + width)
    hidden = torch.randn((rows, width), generator=g, device="cuda").to(dtype).requires_grad_(True)
    weight = (torch.randn((vocab, width), generator=g, device="cuda") * (0.5 / width ** 0.5)).to(dtype).requires_grad_(True)
    tokens = torch.randperm(vocab, generator=g, device="cuda")[torch.arange(rows, device="cuda") % vocab][:, None]
    d = torch.rand(rows, generator=g, device="cuda") + 0.5
    dx, off = head_bounds.adjoints(hidden.detach(), weight.detach(), tokens, d)
    want = head_bounds.gradients(dx, off, hidden.detach(), weight.detach(), dtype)
    if distilled:
        out, d = klay.head_distill(hidden, weight, tokens, torch.zeros((rows, 1), device="cuda")), -d      # (q = 1: the negated log probability)
    else:
        out = klay.head_logprobs(hidden, weight, tokens).logp[:, 0]
    for name, got in zip(("dhidden", "dweight"), torch.autograd.grad(out, (hidden, weight), d)):
        worst = head_bounds.worst(got, want[name], dtype)
        assert worst <= 1.0, (name, worst)
