"""Heads' and distillations' calls with no GPU, the library's replaced by ones that take down their arguments: tangents, what is saved for the reverse call
and comes back elsewhere, calls under recomputation."""
import pytest
import torch
import torch.autograd.forward_ad as fwd
from torch.utils.checkpoint import checkpoint

from paper_2410_11415_amd import binding, operators

FORWARD = ("klay_head_forward", "klay_head_distill_forward", "klay_distill_forward")
BACKWARD = ("klay_head_backward", "klay_head_distill_backward", "klay_distill_backward")


@pytest.fixture
def calls(monkeypatch):
    seen = []
    monkeypatch.setattr(operators, "_check_tensor", lambda *a, **k: None)
    monkeypatch.setattr(operators, "_stream", lambda device: 0)
    monkeypatch.setattr(binding, "klay_head_workspace_bytes", lambda args, back: 0)
    for name in FORWARD + BACKWARD:
        monkeypatch.setattr(binding, name, lambda args, *a, name=name: seen.append((name, args, a)))
    return seen


T, Z = torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2)
CALLS = {
    "hidden": lambda x: operators.head_logprobs(x(4, 8), torch.ones(10, 8), T).logp,
    "weight": lambda x: operators.head_logprobs(torch.ones(4, 8), x(10, 8), T).logp,
    "bias": lambda x: operators.head_logprobs(torch.ones(4, 8), torch.ones(10, 8), T, x(10)).logp,
    "distilled hidden": lambda x: operators.head_distill(x(4, 8), torch.ones(10, 8), T, Z),
    "distilled weight": lambda x: operators.head_distill(torch.ones(4, 8), x(10, 8), T, Z),
    "distilled bias": lambda x: operators.head_distill(torch.ones(4, 8), torch.ones(10, 8), T, Z, x(10)),
    "distilled logits": lambda x: operators.token_distill(x(4, 10), T, Z),
}


@pytest.mark.parametrize("which", sorted(CALLS) + ["teacher", "teacher of a head"])
@pytest.mark.parametrize("grad", [False, True])
def test_tangents_are_refused(calls, which, grad):
    more = {"teacher": lambda x: operators.token_distill(torch.ones(4, 10), T, x(4, 2)),
            "teacher of a head": lambda x: operators.head_distill(torch.ones(4, 8), torch.ones(10, 8), T, x(4, 2))}
    call = {**CALLS, **more}[which]
    with torch.set_grad_enabled(grad), fwd.dual_level():
        with pytest.raises(RuntimeError, match="forward-mode"):
            call(lambda *shape: fwd.make_dual(torch.ones(shape), torch.ones(shape)))
        assert not calls
        call(lambda *shape: torch.ones(shape))
        assert len(calls) == 1


@pytest.mark.parametrize("which", sorted(CALLS))
def test_saved_tensors_that_move(calls, which):
    """the reverse call reads what the hooks give back, where it lies, and nothing of what they took"""
    kept = []

    def give(t):
        kept.append(t.clone())
        return kept[-1]
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, give):
        out = CALLS[which](lambda *shape: torch.ones(shape).requires_grad_())
    out.sum().backward()
    (_, _, _), (name, args, rest) = calls
    assert name in BACKWARD
    given = {t.data_ptr() for t in kept}
    read = {args.logits, args.tokens} if name == "klay_distill_backward" else {args.hidden, args.weight, args.tokens}
    if name != "klay_distill_backward" and "bias" in which:
        read.add(args.bias)
    if name != "klay_head_backward":
        read.add(rest[0].logits)
    assert read <= given


@pytest.mark.parametrize("which", sorted(CALLS))
def test_saved_tensors_that_stay(calls, which):
    """... and without hooks the reverse call's args are the forward call's"""
    out = CALLS[which](lambda *shape: torch.ones(shape).requires_grad_())
    out.sum().backward()
    assert [c[0] in BACKWARD for c in calls] == [False, True] and calls[0][1] is calls[1][1]


@pytest.mark.parametrize("which", sorted(CALLS))
def test_recomputed(calls, which):
    x = []

    def leaf(*shape):
        if not x:
            x.append(torch.ones(shape).requires_grad_())
        return x[0]
    CALLS[which](leaf)
    del calls[:]
    checkpoint(lambda t: CALLS[which](lambda *shape: t), x[0], use_reentrant=False).sum().backward()
    assert [c[0] in BACKWARD for c in calls] == [False, False, True] and x[0].grad.shape == x[0].shape


@pytest.mark.parametrize("which", sorted(CALLS))
def test_twice_differentiated_is_refused(calls, which):
    x = torch.ones(10) if "bias" in which else torch.ones(10, 8) if "weight" in which else torch.ones(4, 10) if "logits" in which else torch.ones(4, 8)
    x.requires_grad_()
    grad, = torch.autograd.grad(CALLS[which](lambda *shape: x).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable|does not require grad"):
        grad.sum().backward()
