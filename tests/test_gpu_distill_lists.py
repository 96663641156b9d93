"""Divergences (GPU): lists whose entries all go to another entry's place: descending, with tokens more than once and entries of nothing between them."""
import pytest
import torch

from tests.test_gpu_distill import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,vocab", [(20, 300), (20, 5000), (600, 700), (3, 40000)])
@pytest.mark.parametrize("k", [2, 33, 64, 65, 200])
@pytest.mark.parametrize("rest", [False, True])
def test_entries_change_places(rows, vocab, k, rest):
    g = torch.Generator(device="cuda").manual_seed(vocab + k)
    x = 2.5 * torch.randn((rows, vocab), generator=g, device="cuda")
    t = (torch.randint(0, vocab, (rows, 1), generator=g, device="cuda") + 3 * torch.arange(k, 0, -1, device="cuda")) % vocab
    t[:, ::5] = t[:, :1]                                        # (the same token again and again)
    t[1::3, ::4] = -1
    z = torch.log_softmax(torch.randn((rows, k), generator=g, device="cuda"), 1) - (0.2 if rest else 0.0)
    check(x, t, z, g, rest=rest)
