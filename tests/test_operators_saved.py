"""What the operators' reverse calls are given, with no GPU: the library's calls are replaced by ones that look at the addresses in their
arguments.  Under hooks on saved tensors (which checkpointing without re-entry and saving to the host are made of) only what came back
from the hooks may be pointed at, whether the forward call had copied a layout or not; and nothing else may outlive the forward call."""
import ctypes
import gc
import weakref

import pytest
import torch
from torch.utils.checkpoint import checkpoint

from paper_2410_11415_amd import binding, operators


class Calls:
    """the arguments of the library's calls"""

    def __init__(self):
        self.forward, self.backward = [], []


@pytest.fixture
def calls(monkeypatch):
    seen = Calls()
    monkeypatch.setattr(operators, "_check_tensor", lambda *a, **k: None)
    monkeypatch.setattr(operators, "_stream", lambda device: 0)
    for name in ("klay_tokens", "klay_scan"):
        monkeypatch.setattr(binding, name + "_workspace_bytes", lambda args: 0)
        monkeypatch.setattr(binding, name + "_forward", lambda args, *a: seen.forward.append(args))
        monkeypatch.setattr(binding, name + "_backward", lambda args, *a: seen.backward.append((args, a)))
    return seen


class Elsewhere:
    """hooks that keep copies of what is saved and give back copies of those; `back`: what they gave back, which stays alive"""

    def __init__(self):
        self.back = []

    def pack(self, t):
        return t.detach().clone().contiguous()

    def unpack(self, t):
        self.back.append(t.clone())
        return self.back[-1]

    def holds(self, pointer, dtype):
        return any(t.dtype == dtype and t.data_ptr() <= pointer < t.data_ptr() + max(1, t.numel() * t.element_size()) for t in self.back)


def floats(pointer, count):
    return list((ctypes.c_float * count).from_address(pointer))




LAYOUTS = {"plain": lambda t: t, "apart": lambda t: t.transpose(0, -1).contiguous().transpose(0, -1)}


@pytest.mark.parametrize("semiring", [0, 1])
@pytest.mark.parametrize("layout", sorted(LAYOUTS))
@pytest.mark.parametrize("shared_start", [False, True])
def test_packed_sequences_under_hooks(calls, shared_start, layout, semiring):
    a = LAYOUTS[layout](torch.rand(10, 4)).requires_grad_(True)
    x = LAYOUTS[layout](torch.rand(10, 4))
    h = (torch.rand(1, 4).expand(2, 4) if shared_start else torch.rand(2, 4)).requires_grad_(True)
    offsets = torch.tensor([0, 4, 10])
    hooks = Elsewhere()
    with torch.autograd.graph.saved_tensors_hooks(hooks.pack, hooks.unpack):
        out, _ = operators.gated_scan(a, x, h, semiring, offsets=offsets)
    out.sum().backward()
    (args, rest), = calls.backward
    assert hooks.holds(args.row_info, torch.int32) and hooks.holds(args.offsets, torch.int64)
    assert hooks.holds(args.gates, torch.float32) and hooks.holds(args.initial, torch.float32) and hooks.holds(rest[0], torch.float32)
    assert floats(args.gates, 4) == a[0].tolist() and floats(args.initial + 16, 4) == h[1].tolist()
    if semiring == 1:
        assert hooks.holds(args.inputs, torch.float32) and floats(args.inputs, 4) == x[0].tolist()


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
def test_token_logprobs_under_hooks(calls, layout):
    x = LAYOUTS[layout](torch.rand(6, 5)).requires_grad_(True)
    t = torch.arange(4).expand(6, 4).transpose(0, 1).contiguous().transpose(0, 1)
    hooks = Elsewhere()
    with torch.autograd.graph.saved_tensors_hooks(hooks.pack, hooks.unpack):
        r = operators.token_logprobs(x, t, complement=True)
    (r.logp.sum() + r.neg.sum()).backward()
    (args, rest), = calls.backward
    assert hooks.holds(args.logits, torch.float32) and hooks.holds(args.tokens, torch.int64) and hooks.holds(rest[0], torch.float32)
    assert floats(args.logits + 4 * args.logit_rows.inner_stride, 5) == x[1].tolist()


def test_checkpoint_without_reentry(calls):
    """the forward call made again in the backward pass is the one whose row info is read"""
    a, h = torch.rand(10, 4, requires_grad=True), torch.rand(1, 4, requires_grad=True)
    offsets = torch.tensor([0, 4, 10])
    y = checkpoint(lambda a, h: operators.gated_scan(a, torch.ones(10, 4), h.expand(2, 4), 0, offsets=offsets)[0].sum(), a, h, use_reentrant=False)
    between = [torch.zeros(10, dtype=torch.int32) for _ in range(8)]      # takes up what the first forward call left
    y.backward()
    (args, _), = calls.backward
    assert len(calls.forward) == 2 and args.row_info == calls.forward[1].row_info
    assert args.row_info not in [t.data_ptr() for t in between]


@pytest.mark.parametrize("what", ["initial", "gates", "logits"])
def test_nothing_else_is_kept_alive(calls, what):
    """a copy of a layout is saved, not held beside what the hooks hold"""
    made = []
    real = torch.Tensor.contiguous

    def contiguous(t, *args, **kw):
        c = real(t, *args, **kw)
        if c is not t:
            made.append(weakref.ref(c))
        return c
    apart = LAYOUTS["apart"]
    a, h = torch.rand(3, 7, 4, requires_grad=True), torch.rand(1, 4).expand(3, 4)
    x = apart(torch.rand(6, 5)).requires_grad_(True)
    torch.Tensor.contiguous = contiguous
    try:
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t.detach().numpy().copy(), torch.from_numpy):
            if what == "logits":
                out = operators.token_logprobs(x, None, entropy=True).entropy
            else:
                out, _ = operators.gated_scan(apart(a) if what == "gates" else a, torch.ones(3, 7, 4), h if what == "initial" else None)
    finally:
        torch.Tensor.contiguous = real
    gc.collect()
    assert out.requires_grad and made
    assert all(r() is None for r in made)


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
def test_without_hooks_the_arguments_stay(calls, layout):
    a, x = (LAYOUTS[layout](torch.rand(3, 7, 4)).requires_grad_(True) for _ in range(2))
    out, _ = operators.gated_scan(a, x, None, 1)
    out.sum().backward(retain_graph=True)                # (what is saved stays, to be looked at below)
    assert calls.backward[0][0] is calls.forward[0]
    assert [floats(calls.backward[0][0].gates, 4), floats(calls.backward[0][0].inputs, 4)] == [a[0, 0].tolist(), x[0, 0].tolist()]
