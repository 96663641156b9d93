"""Calls of the operators that reach the library with other arguments than were meant, or not at all, with no GPU: the library's calls are
replaced by ones that take down their arguments."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paper_2410_11415_amd import binding, operators


@pytest.fixture
def calls(monkeypatch):
    seen = []
    monkeypatch.setattr(operators, "_check_tensor", lambda *a, **k: None)
    monkeypatch.setattr(operators, "_stream", lambda device: 0)
    for name in ("klay_tokens", "klay_scan"):
        monkeypatch.setattr(binding, name + "_workspace_bytes", lambda args: 0)
        monkeypatch.setattr(binding, name + "_forward", lambda args, *a: seen.append(args))
    monkeypatch.setattr(binding, "klay_scan_step", lambda *a: seen.append(a))
    return seen


TANGENTS = {
    "logits": lambda d: operators.token_logprobs(d(2, 5), None, entropy=True),
    "gates": lambda d: operators.gated_scan(d(2, 5, 3), torch.ones(2, 5, 3)),
    "inputs": lambda d: operators.gated_scan(torch.ones(2, 5, 3), d(2, 5, 3)),
    "initial": lambda d: operators.gated_scan(torch.ones(2, 5, 3), torch.ones(2, 5, 3), d(2, 3)),
    "max": lambda d: operators.gated_scan(d(2, 5, 3), torch.ones(2, 5, 3), None, 2),
    "step gates": lambda d: operators.gated_step(d(2, 3), torch.ones(2, 3), torch.ones(2, 3)),
    "step state": lambda d: operators.gated_step(torch.ones(2, 3), torch.ones(2, 3), d(2, 3)),
    "step out": lambda d: operators.gated_step(torch.ones(2, 3), torch.ones(2, 3), torch.ones(2, 3), out=d(2, 3)),
}


@pytest.mark.parametrize("which", sorted(TANGENTS))
@pytest.mark.parametrize("grad", [False, True])
def test_tangents_are_refused(calls, which, grad):
    """a dual tensor's tangent would be lost; without one the call goes through"""
    with torch.set_grad_enabled(grad), fwd.dual_level():
        with pytest.raises(RuntimeError, match="forward-mode"):
            TANGENTS[which](lambda *shape: fwd.make_dual(torch.ones(shape), torch.ones(shape)))
        assert not calls
        TANGENTS[which](lambda *shape: torch.ones(shape))
        assert len(calls) == 1


def test_transformed_functions_are_refused(calls):
    with pytest.raises(RuntimeError, match="forward-mode"):
        torch.func.jvp(lambda x: operators.token_logprobs(x, None, entropy=True).entropy, (torch.ones(2, 5),), (torch.ones(2, 5),))
    assert not calls
