"""What the operators refuse, with no GPU: the C entry points before anything is launched, the Python functions before they call
them.  And their 64-bit references against differences."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2410_11415_amd import KlayError, binding, operators
from tests import operators_ref as ref

P = 4096        # a pointer that no refused call looks behind


def tokens_args(**kw):
    a = dict(dtype=0, device=0, vocab=10, num_tokens=2, top=0, reserved=0, rows=4, logits=P, logit_rows=binding.klay_rows(4, 0, 10), tokens=P,
             token_rows=binding.klay_rows(4, 0, 2), token_stride=1)
    a.update(kw)
    return binding.klay_tokens_args(*a.values())


def scan_args(**kw):
    a = dict(dtype=0, semiring=0, device=0, channels=3, batch=2, time=5, sequences=0, gates=P, inputs=P, gates_batch_stride=15, gates_time_stride=3,
             inputs_batch_stride=15, inputs_time_stride=3, offsets=None, row_info=None, initial=None)
    a.update(kw)
    return binding.klay_scan_args(*a.values())


BAD_TOKENS = [dict(dtype=3), dict(dtype=-1), dict(vocab=0), dict(vocab=-5), dict(num_tokens=-1), dict(num_tokens=1025), dict(top=-1), dict(top=11),
              dict(vocab=1000, top=65), dict(rows=-1), dict(rows=1 << 31), dict(logits=None), dict(tokens=None),
              dict(logit_rows=binding.klay_rows(0, 0, 10)), dict(token_rows=binding.klay_rows(0, 0, 2))]


@pytest.mark.parametrize("bad", BAD_TOKENS, ids=lambda b: ",".join("%s=%s" % (k, getattr(v, "inner", v)) for k, v in b.items()))
def test_tokens_arguments(bad):
    for call in (lambda a: binding.klay_tokens_forward(a, P, None, None, None, P, P, P, 1 << 40),
                 lambda a: binding.klay_tokens_backward(a, P, P, None, None, P)):
        with pytest.raises(KlayError) as e:
            call(tokens_args(**bad))
        assert e.value.status == binding.KLAY_EINVAL and "klay_tokens_" in str(e.value)


def test_tokens_outputs_and_workspace():
    for args, out in ((tokens_args(), (None, None, None, None, None, None)), (tokens_args(top=2), (P, None, None, None, None, P)),
                      (tokens_args(top=2), (P, None, None, None, P, None))):
        with pytest.raises(KlayError) as e:
            binding.klay_tokens_forward(args, *out, None, 0)
        assert e.value.status == binding.KLAY_EINVAL
    for given in ((None, P), (P, None)):
        with pytest.raises(KlayError) as e:
            binding.klay_tokens_backward(tokens_args(), given[0], P, None, None, given[1])
        assert e.value.status == binding.KLAY_EINVAL
    one = tokens_args(rows=1, vocab=1000000, top=5)
    need = binding.klay_tokens_workspace_bytes(one)
    assert need > 0 and binding.klay_tokens_workspace_bytes(tokens_args()) == 0 == binding.klay_tokens_workspace_bytes(None)
    for at, size, status in ((None, need, binding.KLAY_ENOMEM), (P, need - 1, binding.KLAY_ENOMEM), (P + 4, need, binding.KLAY_EINVAL)):
        with pytest.raises(KlayError) as e:
            binding.klay_tokens_forward(one, P, None, None, None, P, P, at, size)
        assert e.value.status == status
    for call in (lambda: binding.klay_tokens_forward(None, P, None, None, None, None, None, None, 0),
                 lambda: binding.klay_tokens_backward(None, P, P, None, None, P)):
        with pytest.raises(KlayError):
            call()
    binding.klay_tokens_forward(tokens_args(rows=0, logits=None, tokens=None), None, None, None, None, None, None, None, 0)     # nothing to do
    binding.klay_tokens_backward(tokens_args(rows=0, logits=None, tokens=None), None, None, None, None, None)


BAD_SCANS = [dict(dtype=7), dict(semiring=3), dict(semiring=-1), dict(semiring=1, dtype=1), dict(semiring=2, dtype=2), dict(channels=0),
             dict(channels=(1 << 25) + 1), dict(gates_time_stride=(1 << 25) + 1), dict(inputs_time_stride=-1), dict(batch=-1), dict(batch=1 << 30), dict(time=-1), dict(time=1 << 31), dict(gates=None),
             dict(offsets=P, row_info=P), dict(offsets=P, batch=1), dict(offsets=P, batch=1, row_info=P, sequences=-1),
             dict(offsets=P, batch=1, row_info=P, sequences=1 << 30)]


@pytest.mark.parametrize("bad", BAD_SCANS, ids=lambda b: ",".join("%s=%s" % kv for kv in b.items()))
def test_scan_arguments(bad):
    for call in (lambda a: binding.klay_scan_forward(a, P, None, P, 1 << 40),
                 lambda a: binding.klay_scan_backward(a, P, P, None, P, P, None, P, 1 << 40)):
        with pytest.raises(KlayError) as e:
            call(scan_args(**bad))
        assert e.value.status == binding.KLAY_EINVAL and "klay_scan_" in str(e.value)


def test_scan_outputs_and_workspace():
    for call in (lambda: binding.klay_scan_forward(scan_args(), None, None, None, 0), lambda: binding.klay_scan_forward(None, P, None, None, 0),
                 lambda: binding.klay_scan_forward(scan_args(inputs=None), P, None, None, 0),
                 lambda: binding.klay_scan_backward(scan_args(), None, P, None, P, P, None, None, 0),
                 lambda: binding.klay_scan_backward(None, P, P, None, P, P, None, None, 0),
                 lambda: binding.klay_scan_backward(scan_args(semiring=1, inputs=None), P, P, None, P, P, None, None, 0),
                 lambda: binding.klay_scan_backward(scan_args(semiring=2), P, P, None, P, P, None, None, 0)):
        with pytest.raises(KlayError) as e:
            call()
        assert e.value.status == binding.KLAY_EINVAL
    long = scan_args(batch=1, time=100000)
    need = binding.klay_scan_workspace_bytes(long)
    assert need > 0 and binding.klay_scan_workspace_bytes(scan_args()) == 0 == binding.klay_scan_workspace_bytes(None)
    for at, size, status in ((None, need, binding.KLAY_ENOMEM), (P, need - 1, binding.KLAY_ENOMEM), (P + 8, need, binding.KLAY_EINVAL)):
        with pytest.raises(KlayError) as e:
            binding.klay_scan_forward(long, P, None, at, size)
        assert e.value.status == status


def test_more_tiles_than_a_launch_has_workgroups():
    """a workgroup a tile (that is what the workspace is for) only where they fit a launch"""
    for batch, time, some in ((1, 1 << 29, True), (1, (1 << 31) - 1, False), (100, 1 << 23, True), (100, 1 << 24, False)):
        assert (binding.klay_scan_workspace_bytes(scan_args(batch=batch, time=time)) > 0) == some


@pytest.mark.parametrize("bad", [dict(dtype=9), dict(semiring=5), dict(semiring=1, dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(channels=0),
                                 dict(channels=(1 << 25) + 1), dict(gates=None), dict(inputs=None), dict(state=None)])
def test_step_arguments(bad):
    a = dict(dtype=0, semiring=0, device=0, rows=2, channels=4, gates=P, gs=4, inputs=P, xs=4, state=P, ss=4, out=P, os=4)
    a.update(bad)
    with pytest.raises(KlayError) as e:
        binding.klay_scan_step(*a.values())
    assert e.value.status == binding.KLAY_EINVAL


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(binding.klay_rows) == 24
    assert ctypes.sizeof(binding.klay_tokens_args) == 24 + 8 + 8 + 24 + 8 + 24 + 8
    assert ctypes.sizeof(binding.klay_scan_args) == 16 + 24 + 16 + 32 + 24


# ---- the Python functions -----------------------------------------------------------------------------------------
def test_host_tensors_are_refused():
    x, t = torch.zeros(2, 5), torch.zeros((2, 1), dtype=torch.int64)
    for call in (lambda: operators.token_logprobs(x, t), lambda: operators.token_logprobs([1.0], t),
                 lambda: operators.gated_scan(torch.zeros(1, 2, 3), torch.zeros(1, 2, 3)), lambda: operators.gated_step(x, x, x)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()


@pytest.fixture
def anywhere(monkeypatch):
    """the checks that come after the first, on host tensors"""
    def check(t, name, dtypes=None):
        if dtypes is not None and t.dtype not in dtypes:
            raise ValueError(name)
    monkeypatch.setattr(operators, "_check_tensor", check)
    for name in ("klay_tokens_forward", "klay_scan_forward", "klay_scan_step"):
        monkeypatch.setattr(binding, name, lambda *a: pytest.fail("reached the library"))


def test_token_shapes(anywhere):
    x, t = torch.zeros(2, 5), torch.zeros((2, 1), dtype=torch.int64)
    for call in (lambda: operators.token_logprobs(x.double(), t), lambda: operators.token_logprobs(x, t.int()),
                 lambda: operators.token_logprobs(x, t[:1]), lambda: operators.token_logprobs(x, t[0]), lambda: operators.token_logprobs(x[:, :0], t),
                 lambda: operators.token_logprobs(x[0, 0], t), lambda: operators.token_logprobs(x, t, top=6), lambda: operators.token_logprobs(x, t, top=-1),
                 lambda: operators.token_logprobs(torch.zeros(2, 100), t, top=65), lambda: operators.token_logprobs(x, t, top=1 << 32),
                 lambda: operators.token_logprobs(x, None, complement=True), lambda: operators.token_logprobs(x, t.expand(2, 1025))):
        with pytest.raises(ValueError):
            call()


def test_recurrence_shapes(anywhere):
    a = torch.zeros(2, 4, 3)
    h = torch.zeros(2, 3)
    o = torch.tensor([0, 2])
    for call in (lambda: operators.gated_scan(a, a[:, :2]), lambda: operators.gated_scan(a, a.half()), lambda: operators.gated_scan(a.double(), a.double()),
                 lambda: operators.gated_scan(a, a, h[:1]), lambda: operators.gated_scan(a, a, h.half()), lambda: operators.gated_scan(a, a, h, 3),
                 lambda: operators.gated_scan(a.half(), a.half(), h, 1), lambda: operators.gated_scan(a.half(), a.half(), h, 2),
                 lambda: operators.gated_scan(a[0], a[0]), lambda: operators.gated_scan(a, a, offsets=o), lambda: operators.gated_scan(a[..., :0], a[..., :0]),
                 lambda: operators.gated_scan(a[0], a[0], offsets=o.int()), lambda: operators.gated_scan(a[0], a[0], offsets=o[:0]),
                 lambda: operators.gated_scan(a[0], a[0], h, offsets=o), lambda: operators.gated_scan(a[0], a[0], offsets=torch.zeros(4, dtype=torch.int64)[::2]),
                 lambda: operators.gated_step(h, h, h[:1]), lambda: operators.gated_step(a, a, a), lambda: operators.gated_step(h, h, h.half()),
                 lambda: operators.gated_step(h, h, torch.zeros(3, 2).t()), lambda: operators.gated_step(h, h, h[:1].expand(2, 3)),
                 lambda: operators.gated_step(h, h, h, out=h[:1]), lambda: operators.gated_step(h, h, h, out=h.half()),
                 lambda: operators.gated_step(h, h, h, out=torch.zeros(3, 2).t()), lambda: operators.gated_step(h, h, h, out=3)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(RuntimeError, match="not differentiated"):
        operators.gated_scan(a.clone().requires_grad_(True), a, h, 2)
    with pytest.raises(RuntimeError, match="not differentiated"):
        operators.gated_step(h, h.clone().requires_grad_(True), h)


def test_from_logits_refuses():
    from types import SimpleNamespace
    from paper_2410_11415_amd import CircuitLayer
    circuit = SimpleNamespace(num_vars=6)
    x, t = torch.zeros(2, 3, 9), torch.zeros((3, 2), dtype=torch.int64)
    with pytest.raises(ValueError, match="semiring"):
        CircuitLayer(circuit, 0).from_logits(x, t)
    layer = CircuitLayer(circuit, 1)
    for args in ((x[0], t), (x, t[:2]), (x, t[0]), (x, torch.zeros((3, 3), dtype=torch.int64)), (x[:, :2], t)):
        with pytest.raises(ValueError):
            layer.from_logits(*args)


# ---- the references themselves ------------------------------------------------------------------------------------
def test_token_reference_against_differences():
    rng = np.random.default_rng(0)
    x, t = rng.normal(size=(3, 7)), rng.integers(0, 7, size=(3, 4))
    t[0, 1] = t[0, 2] = t[0, 0]
    g = dict(dlogp=rng.normal(size=(3, 4)), dneg=rng.normal(size=(3, 4)), dent=rng.normal(size=3))

    def f(y):
        r = ref.tokens(y, t)
        return (g["dlogp"] * r["logp"]).sum() + (g["dneg"] * r["neg"]).sum() + (g["dent"] * r["entropy"]).sum()
    grad = ref.tokens(x, t, **g)["dlogits"]
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = 1e-5
        assert abs((f(x + d) - f(x - d)) / 2e-5 - grad[i]) < 1e-7


@pytest.mark.parametrize("semiring", [ref.REAL, ref.LOG])
def test_scan_reference_against_differences(semiring):
    rng = np.random.default_rng(1)
    a, x, h, dh, df = rng.normal(size=(5, 2)), rng.normal(size=(5, 2)), rng.normal(size=2), rng.normal(size=(5, 2)), rng.normal(size=2)

    def f(*s):
        r = ref.scan(semiring, *s)
        return (r["h"] * dh).sum() + (r["final"] * df).sum()
    r = ref.scan(semiring, a, x, h, dh, df)
    for n, name in enumerate(("da", "dx", "dinitial")):
        for i in np.ndindex((a, x, h)[n].shape):
            lo, hi = [a.copy(), x.copy(), h.copy()], [a.copy(), x.copy(), h.copy()]
            lo[n][i] -= 1e-5
            hi[n][i] += 1e-5
            assert abs((f(*hi) - f(*lo)) / 2e-5 - r[name][i]) < 1e-7
