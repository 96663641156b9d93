"""Heads of wide rows and of few rows (GPU): values and gradients within bounds that a wrong sign, or nothing in their place, is far outside of."""
import pytest
import torch

from tests import head_bounds
from tests import head_ref as ref
from tests.test_head_bounds import WIDE, wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=lambda v: str(v).replace("torch.", ""))
@pytest.mark.parametrize("rows,width,vocab", WIDE)
def test_wide(rows, width, vocab, dtype):
    import paper_2410_11415_amd as klay
    hidden, weight, bias, tokens, d, x, slip = wide(rows, width, vocab, dtype, "cuda")
    want, dx, off = ref.tokens(x, tokens, slip, *(v.double() for v in d))
    want["neg"] = head_bounds.negated(x, tokens, slip, ref.terms(vocab))
    inputs = [t.requires_grad_(True) for t in (hidden, weight, bias)]
    r = klay.head_logprobs(inputs[0], inputs[1], tokens, inputs[2], complement=True, entropy=True)
    for name in ("logp", "neg", "entropy"):
        ref.close(getattr(r, name), want[name], what=name)
    grads = ref.gradients(dx, off, hidden, weight)
    for name, got in zip(("dhidden", "dweight", "dbias"), torch.autograd.grad(list(r), inputs, d)):
        ref.close(got, grads[name], got.dtype, name)
    # ... and of a divergence from two tokens
    teacher = torch.zeros(tokens.shape, device="cuda")
    want, dx, off = ref.distill(x, tokens, teacher, 1.0, False, slip, d[2].double())
    loss = klay.head_distill(inputs[0], inputs[1], tokens, teacher, inputs[2])
    ref.close(loss, want, what="loss")
    grads = ref.gradients(dx, off, hidden, weight)
    for name, got in zip(("dhidden", "dweight", "dbias"), torch.autograd.grad(loss, inputs, d[2])):
        ref.close(got, grads[name], got.dtype, name)
