"""The bounds on heads' gradients, with no GPU: adjoints of two numbers of 16 bits keep to them, of one they do not."""
import pytest
import torch

from tests import head_bounds


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
