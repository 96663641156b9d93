"""The 64-bit reference of a divergence, with no GPU, where its q do not add up to 1: its gradient against differences of its loss, and both against a
loss written out once more and differentiated by autograd."""
import pytest
import torch

from tests import head_ref as ref


def loss_of(x, t, z, temperature, rest):
    """sum_k q_k (ln q_k - ln p_{t_k}), with `rest` + q_r (ln q_r - ln p_r), q_r = 1 - sum q (0 where negative, or where no token outside the list is allowed);
    negative tokens list nothing"""
    lp = torch.log_softmax(x / temperature, 1)
    there = t >= 0
    at = t.clamp(min=0)
    z = torch.where(there, z, -torch.inf)
    if not rest:
        z = torch.log_softmax(z / temperature, 1)
    q = torch.where(there, z.exp(), 0.0)
    loss = torch.where(q > 0, q * (torch.where(there, z, 0.0) - lp.gather(1, at)), 0.0).sum(1)
    if rest:
        others = torch.ones(x.shape[0], x.shape[1] + 1, dtype=torch.bool, device=x.device).scatter_(1, torch.where(there, at, x.shape[1]), False)[:, :-1]
        others = others & (x > -torch.inf)
        q_rest = torch.where(others.any(1), (1 - q.sum(1)).clamp(min=0), 0.0)
        p_rest = torch.where(others, lp.exp(), 0.0).sum(1)
        some = q_rest > 0
        loss = loss + torch.where(some, q_rest * (torch.where(some, q_rest, 1.0).log() - torch.where(some, p_rest, 1.0).log()), 0.0)
    return torch.where(there.any(1), loss, 0.0)


def cases():
    g = torch.Generator().manual_seed(3)
    x = torch.randn(4, 6, generator=g, dtype=torch.float64) * 2
    every = torch.stack([torch.randperm(6, generator=g) for _ in range(4)])
    some = every[:, :3].contiguous()
    only = torch.full_like(x, -torch.inf).scatter_(1, some, x.gather(1, some))
    part = some.clone()
    part[1, 2], part[2] = -1, -1

    def teacher(k, mass):
        return torch.log_softmax(torch.randn(4, k, generator=g, dtype=torch.float64), 1) + torch.tensor(mass).double().log()
    return {"every token": (x, every, teacher(6, 0.5)), "every token, above 1": (x, every, teacher(6, 1.7)), "others barred": (only, some, teacher(3, 0.4)),
            "above 1": (x, some, teacher(3, 1.3)), "below 1": (x, some, teacher(3, 0.7)), "lists of some lengths": (x, part, teacher(3, 0.8)),
            "repeated": (x, some[:, [0, 1, 1]], teacher(3, 0.6)), "repeated, above 1": (x, some[:, [0, 1, 1]], teacher(3, 1.6))}


@pytest.mark.parametrize("temperature", [1.0, 2.0, 0.5])
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("which", sorted(cases()))
def test_against_differences_and_autograd(which, rest, temperature):
    x, t, z = cases()[which]
    d = torch.tensor([1.0, -0.5, 2.0, 0.25], dtype=torch.float64)
    slip = torch.zeros(4, dtype=torch.float64)
    f = lambda x: ref.distill(x, t, z, temperature, rest, slip)[0][0]  # noqa: E731
    dx = ref.distill(x, t, z, temperature, rest, slip, d)[1]
    leaf = x.clone().requires_grad_(True)
    loss = loss_of(leaf, t, z, temperature, rest)
    assert torch.allclose(f(x), loss.detach(), rtol=1e-12, atol=1e-12)
    assert torch.allclose(torch.autograd.grad(loss, leaf, d)[0], dx, rtol=1e-10, atol=1e-12)
    for i in range(x.numel()):
        up, down = x.clone(), x.clone()
        up.view(-1)[i] += 1e-5
        down.view(-1)[i] -= 1e-5
        assert abs(float((f(up) * d).sum() - (f(down) * d).sum()) / 2e-5 - float(dx.view(-1)[i])) < 1e-8
    assert float(dx.sum(1).abs().max()) < 1e-12                # (the loss knows no constant that all logits of a row share)
