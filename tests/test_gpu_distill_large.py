"""Divergences (GPU) of more rows than a launch has workgroups, than 2^32 threads would be a wave each, and of more than 2^31 logits: the last rows against
the same rows by themselves, first ones against the definition."""
import pytest
import torch

from tests import head_ref as ref

pytestmark = pytest.mark.gpu


# short rows, a wave each: past 2^20 workgroups of four, past 2^32 threads; rows of a workgroup each, joined by a wave each
@pytest.mark.parametrize("rows,vocab,k", [((1 << 22) + 779, 5, 2), ((1 << 20) + 777, 40, 70), ((1 << 26) + 5, 3, 1), ((1 << 20) + 777, 530, 3), ((1 << 22) + 779, 513, 1)])
def test_more_rows_than_workgroups(rows, vocab, k):
    import paper_2410_11415_amd as klay
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.empty((rows, vocab), dtype=torch.float16, device="cuda").normal_(0, 2, generator=g).requires_grad_(True)
    t = torch.randint(0, vocab, (rows, k), generator=g, device="cuda")
    z = torch.randn((rows, k), generator=g, device="cuda")
    d = torch.rand(rows, generator=g, device="cuda") + 0.5
    loss = klay.token_distill(x, t, z, temperature=1.5)
    dx, = torch.autograd.grad(loss, x, d)
    first = rows - 3000 - rows % 8                              # (its logits lie to 16 bytes as the first row's)
    for part in (slice(0, 3000), slice(first - first % 8, rows)):
        y = x.detach()[part].clone().requires_grad_(True)
        alone = klay.token_distill(y, t[part], z[part], temperature=1.5)
        assert torch.equal(loss[part], alone)
        assert torch.equal(dx[part], torch.autograd.grad(alone, y, d[part])[0])
    some = slice(rows - 700, rows)
    want, dx64, tol = ref.distill(x.detach()[some].double(), t[some], z[some], 1.5, False, torch.zeros(700, dtype=torch.float64, device="cuda"), d[some].double())
    ref.close(loss[some], want, what="loss")
    ref.close(dx[some], (dx64, tol), torch.float16, "dlogits")
