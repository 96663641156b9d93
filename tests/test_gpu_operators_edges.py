"""The operators (GPU) at the borders of their kernels and under autograd's hooks: lengths and sequence borders around a tile's 128 steps and
a group's 16 tiles (eight waves of 16 steps are a tile), checkpointing and saving to the host, single steps out of larger tensors."""
import numpy as np
import pytest
import torch
from torch.utils.checkpoint import checkpoint

from tests import operators_ref as ref
from tests.test_gpu_scan import CASES, LOG, REAL, check, make

pytestmark = pytest.mark.gpu


def klay():
    import paper_2410_11415_amd as pkg
    return pkg


@pytest.mark.parametrize("semiring,dtype", CASES)
@pytest.mark.parametrize("time", [127, 128, 129, 2047, 2048, 2049, 2176, 4096, 4097])
def test_tiles_and_groups(time, semiring, dtype):
    rng = np.random.default_rng(time)
    a, x, h = make((1, time, 4), 1, semiring, dtype, rng)
    check(a, x, h, semiring, dtype, rng)


@pytest.mark.parametrize("time", [127, 128, 129, 257])
@pytest.mark.parametrize("semiring", [REAL, LOG])
def test_tiles_of_many_chains(time, semiring):
    """one workgroup for all tiles of its channels"""
    rng = np.random.default_rng(time)
    a, x, h = make((140, time, 3), 140, semiring, "float32", rng)
    check(a, x, h, semiring, "float32", rng)


BORDERS = {
    "tiles": [0, 127, 128, 129, 256, 384, 385, 512],
    "groups": [0, 2047, 2048, 2049, 4096, 4097, 6144],
    "late": [128, 2048, 2176],                           # the first tile, and the rows behind, are of no sequence
    "last": [0, 2048, 2048, 2049],
}


@pytest.mark.parametrize("semiring,dtype", CASES)
@pytest.mark.parametrize("kind", sorted(BORDERS))
def test_sequences_that_end_with_a_tile(kind, semiring, dtype):
    rng = np.random.default_rng(len(kind))
    cuts = BORDERS[kind]
    rows = cuts[-1] + (130 if kind == "late" else 0)
    a, x, h = make((rows, 3), len(cuts) - 1, semiring, dtype, rng)
    check(a, x, h, semiring, dtype, rng, list(zip(cuts[:-1], cuts[1:])), torch.tensor(cuts, device="cuda"))


def results(call, leaves):
    out = call(*leaves)
    return [out.detach()] + list(torch.autograd.grad(out, leaves))


HOW = {
    "checkpoint": lambda call: lambda *t: checkpoint(call, *t, use_reentrant=False),
    "host": lambda call: lambda *t: on_the_host(call, *t),
}


def on_the_host(call, *t):
    with torch.autograd.graph.save_on_cpu():
        return call(*t)


@pytest.mark.parametrize("semiring", [REAL, LOG])
@pytest.mark.parametrize("how", sorted(HOW))
def test_packed_sequences_with_a_shared_start(how, semiring):
    """a learned initial state for all sequences (copied), saved elsewhere or computed again: the same gradients"""
    rng = np.random.default_rng(0)
    cuts = [0, 300, 300, 901, 1400]
    a, x, h = make((1500, 6), 1, semiring, "float32", rng)
    offsets = torch.tensor(cuts, device="cuda")
    wide = torch.zeros((6, 1500), device="cuda")
    wide.copy_(a.t())                                    # gates whose channels lie apart are copied too

    def call(gates, inputs, start):
        out, final = klay().gated_scan(gates.t(), inputs, start.expand(4, 6), semiring, offsets=offsets)
        return (out * 0.5).sum() + final.sum()
    leaves = [t.clone().requires_grad_(True) for t in (wide, x, h)]
    want = results(call, leaves)
    got = results(HOW[how](call), leaves)
    assert all(torch.equal(p, q) for p, q in zip(want, got)) and torch.isfinite(want[3]).all()


@pytest.mark.parametrize("how", sorted(HOW))
def test_token_logprobs_saved_elsewhere(how):
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((700, 40), generator=gen, device="cuda").requires_grad_(True)
    tokens = torch.randint(0, 700, (40, 3), generator=gen, device="cuda")

    def call(logits):
        r = klay().token_logprobs(logits.t(), tokens, complement=True, entropy=True)
        return r.logp.sum() + r.neg.sum() + r.entropy.sum()
    assert all(torch.equal(p, q) for p, q in zip(results(call, [x]), results(HOW[how](call), [x])))


@pytest.mark.parametrize("semiring", [REAL, LOG])
def test_a_single_step_of_a_large_tensor(semiring):
    rng = np.random.default_rng(3)
    a, x, h = make((3, 1, 8), 3, semiring, "float32", rng)
    far = lambda t: t.as_strided(t.shape, (8, 1 << 26, 1))  # noqa: E731
    check(a, x, h, semiring, "float32", rng, given=(far(a), far(x)))
    row = lambda t: t[:1, 0].as_strided((1, 8), (1 << 26, 1))  # noqa: E731
    check(a[:1, 0], x[:1, 0], h[:1], semiring, "float32", rng, [(0, 1)], torch.tensor([0, 1], device="cuda"), given=(row(a), row(x)))


def test_the_state_of_a_single_sequence():
    k = klay()
    a, x = (torch.rand(1, 8, device="cuda").as_strided((1, 8), (1 << 26, 1)) for _ in range(2))
    state = torch.rand(1, 8, device="cuda")
    want = (a.double() * state.double() + x.double()).cpu().numpy()
    k.gated_step(a, x, state)
    ref.close(state.cpu().numpy(), want, 2 * ref.U * np.abs(want))
