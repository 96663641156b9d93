"""The bounds on heads' values and gradients, with no GPU: adjoints of two numbers of 16 bits keep to them, of one they do not; and of wide rows, of a wrong
sign or with nothing in their place, none keeps to them."""
import pytest
import torch

from tests import head_bounds
from tests import head_ref as ref


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=lambda v: str(v).replace("torch.", ""))
@pytest.mark.parametrize("rows,width,vocab", [(40, 256, 600), (257, 64, 900), (300, 128, 2000)])
def test_adjoints_in_one_number_and_in_two(rows, width, vocab, dtype):
    g = torch.Generator().manual_seed(rows)
    hidden = torch.randn((rows, width), generator=g).to(dtype)
    weight = (torch.randn((vocab, width), generator=g) * (0.5 / width ** 0.5)).to(dtype)
    tokens = torch.randperm(vocab, generator=g)[:rows, None]
    dx, off = head_bounds.adjoints(hidden, weight, tokens, torch.rand(rows, generator=g) + 0.5)
    want = head_bounds.gradients(dx, off, hidden, weight, dtype)
    for numbers in (1, 2):
        kept = head_bounds.held(dx, dtype, numbers)
        got = {"dhidden": (kept @ weight.double()).to(dtype), "dweight": (kept.t().contiguous() @ hidden.double()).to(dtype)}
        worst = {name: head_bounds.worst(got[name], want[name], dtype) for name in got}
        assert max(worst.values()) <= 1.0 if numbers == 2 else min(worst.values()) > 1.2, (numbers, worst)


WIDE = [(16, 550000, 130), (24, 40000, 2000), (40, 1027, 2000), (33, 2240, 1600), (64, 1024, 16400), (64, 1027, 16400), (33, 2240, 16001), (65, 1024, 16384),
        (32, 2560, 16384), (20000, 1024, 60), (1, 4096, 3000), (300, 8192, 700)]


def wide(rows, width, vocab, dtype, device):
    """inputs of a head, adjoints of its three values, its logits in 64 bits and what each row's may be off by"""
    g = torch.Generator(device=device).manual_seed(rows + width)
    normal = lambda *s: torch.randn(s, generator=g, device=device)  # noqa: E731
    weight = (normal(vocab, width) * (2.5 / width ** 0.5)).to(dtype)
    hidden, bias = normal(rows, width).to(dtype), normal(vocab)
    first = torch.randint(0, vocab, (rows, 1), generator=g, device=device)
    tokens = torch.cat([first, (first + 1 + torch.randint(0, vocab - 1, (rows, 1), generator=g, device=device)) % vocab], 1)
    d = normal(rows, 2), normal(rows, 2), torch.rand(rows, generator=g, device=device) + 0.5
    x = hidden.double() @ weight.double().t().contiguous() + bias.double()
    return hidden, weight, bias, tokens, d, x, head_bounds.slip_by_sums(hidden, weight, bias)


@pytest.mark.parametrize("rows,width,vocab", WIDE)
def test_wrong_values_of_wide_rows_are_seen(rows, width, vocab):
    hidden, weight, bias, tokens, d, x, slip = wide(rows, width, vocab, torch.bfloat16, "cpu")
    slip = 2 * slip                                             # (as much as fp32's)
    want, dx, off = ref.tokens(x, tokens, slip, *(v.double() for v in d))
    want["neg"] = head_bounds.negated(x, tokens, slip, ref.terms(vocab))
    loss, dx_loss, off_loss = ref.distill(x, tokens, torch.zeros(tokens.shape), 1.0, False, slip, d[2].double())
    want["loss"] = loss
    for which, (a, b) in (("", (dx, off)), (" of a divergence", (dx_loss, off_loss))):
        want.update({name + which: v for name, v in ref.gradients(a, b, hidden, weight).items()})
    for name, (value, tol) in want.items():
        dtype = torch.bfloat16 if name.startswith(("dhidden", "dweight")) else torch.float32
        ref.close(value.to(dtype), (value, tol), dtype, name)
        for wrong in (torch.zeros_like(value), -value):
            with pytest.raises(AssertionError, match="of the tolerance"):
                ref.close(wrong.to(dtype), (value, tol), dtype, name)
