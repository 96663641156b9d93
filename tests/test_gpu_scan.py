"""The gated recurrence (GPU) against the 64-bit definition, step by step: lengths around the kernels' waves, tiles and chunks, every
semiring and type, packed sequences (empty ones, single steps, rows of none), layouts, the single step."""
import numpy as np
import pytest
import torch

from tests import operators_ref as ref

pytestmark = pytest.mark.gpu
REAL, LOG, MAX = 0, 1, 2


def klay():
    import paper_2410_11415_amd as pkg
    return pkg


def make(shape, count, semiring, dtype, rng, impossible=False):
    C = shape[-1]
    if semiring == REAL:
        a = 1 / (1 + np.exp(-(rng.normal(size=shape) + 2.0))) * np.where(rng.random(shape) < 0.1, -1.0, 1.0)
        x, h = rng.normal(size=shape), rng.normal(size=(count, C))
        a[rng.random(shape) < 0.02] = 0.0
    else:
        a, x, h = (-np.log1p(np.exp(-(rng.normal(size=s) + b))) for s, b in ((shape, 3.0), (shape, -3.0), ((count, C), 0.0)))
        if impossible:
            for t in (a, x, h):
                t[rng.random(t.shape) < 0.2] = -np.inf
            x[..., 0] = -np.inf                          # a channel that only lives by its initial state
            a[..., -1] = -np.inf
    kind = getattr(torch, dtype)
    return torch.from_numpy(a).to(kind).cuda(), torch.from_numpy(x).to(kind).cuda(), torch.from_numpy(h).float().cuda()


def check(a, x, h0, semiring, dtype, rng, spans=None, offsets=None, train=True, given=None, scale=1.0):
    """spans: rows of the packed sequences; h0 None: no initial state; scale: of the adjoints"""
    train = train and semiring != MAX
    dh = torch.from_numpy(rng.normal(size=tuple(x.shape)) * scale).to(x.dtype).cuda()
    count = x.shape[0] if spans is None else len(spans)
    dfinal = torch.from_numpy(rng.normal(size=(count, x.shape[-1])) * scale).float().cuda()
    ga, gx = given if given else (a, x)
    leaves = [t.detach().requires_grad_(train) for t in (ga, gx) + (() if h0 is None else (h0,))]
    h, final = klay().gated_scan(leaves[0], leaves[1], leaves[2] if h0 is not None else None, semiring, offsets=offsets)
    assert h.dtype == x.dtype and h.shape == x.shape and final.dtype == torch.float32
    grads = torch.autograd.grad([h, final], leaves, [dh, dfinal]) if train else []
    n = lambda t: t.detach().double().cpu().numpy()  # noqa: E731
    first = np.full((count, x.shape[-1]), 0.0 if semiring == REAL else -np.inf) if h0 is None else n(h0)
    named = dict(zip(("da", "dx", "dinitial"), grads))
    seen = np.zeros(x.shape[0] if spans is not None else 0, bool)
    for s in range(count):
        rows = (s,) if spans is None else (slice(*spans[s]),)
        want = ref.scan(semiring, n(a[rows]), n(x[rows]), first[s], *((n(dh[rows]), n(dfinal[s])) if train else ()), dtype=dtype)
        if spans is not None:
            seen[spans[s][0]:spans[s][1]] = True
        what = "sequence %d " % s
        ref.close(n(h[rows]), want["h"], want["h_tol"], dtype, what + "h")
        ref.close(n(final[s]), want["final"], want["final_tol"], what=what + "final")
        for name, t in named.items():
            ref.close(n(t[s] if name == "dinitial" else t[rows]), want[name], want[name + "_tol"], "float32" if name == "dinitial" else dtype, what + name)
    if spans is not None:                                # rows of no sequence
        for t in [h] + [named[q] for q in ("da", "dx") if q in named]:
            assert not t[torch.from_numpy(~seen).cuda()].any()


CASES = [(REAL, "float32"), (REAL, "bfloat16"), (REAL, "float16"), (LOG, "float32"), (MAX, "float32")]


# one step, around a wave's 16, four waves' 64, sixteen waves' 256 steps and the chunks made of them
@pytest.mark.parametrize("semiring,dtype", CASES)
@pytest.mark.parametrize("time", [1, 2, 15, 16, 17, 63, 64, 65, 255, 256, 257, 600])
def test_lengths(time, semiring, dtype):
    rng = np.random.default_rng(time)
    a, x, h = make((2, time, 5), 2, semiring, dtype, rng)
    check(a, x, h, semiring, dtype, rng)


@pytest.mark.parametrize("semiring,dtype", CASES)
@pytest.mark.parametrize("batch,time,channels", [(1, 2500, 3), (1, 1100, 130), (70, 40, 7), (3, 300, 64), (300, 70, 2), (1, 90, 65), (2, 520, 129)])
def test_shapes(batch, time, channels, semiring, dtype):
    rng = np.random.default_rng(batch + time)
    a, x, h = make((batch, time, channels), batch, semiring, dtype, rng)
    check(a, x, h, semiring, dtype, rng)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("batch,time,channels", [(520, 16, 100), (260, 50, 130), (110, 300, 520), (256, 70, 256)])
def test_two_channels_a_lane(batch, time, channels, dtype):
    rng = np.random.default_rng(channels)
    a, x, h = make((batch, time, channels), batch, REAL, dtype, rng)
    check(a, x, h, REAL, dtype, rng)
    wide = torch.zeros((batch, time, 2 * channels + 1), dtype=a.dtype, device="cuda")       # the same from odd addresses: one a lane
    wide[..., 1:channels + 1], wide[..., channels + 1:] = a, x
    check(a, x, h, REAL, dtype, rng, given=(wide[..., 1:channels + 1], wide[..., channels + 1:]))


@pytest.mark.parametrize("semiring", [LOG, MAX])
@pytest.mark.parametrize("time", [1, 20, 300, 1500])
def test_impossible_steps(time, semiring):
    rng = np.random.default_rng(time)
    a, x, h = make((2, time, 6), 2, semiring, "float32", rng, impossible=True)
    check(a, x, h, semiring, "float32", rng)
    check(a, x, None, semiring, "float32", rng)


PACKED = {
    "ragged": [0, 5, 5, 6, 40, 41, 300, 300, 555], "one": [0, 700], "singles": list(range(0, 90)), "none": [0, 0, 0],
    "behind": [0, 30, 64, 64, 200], "before": [17, 33, 48, 48, 260], "long": [0, 1, 1500, 1501, 2300],
}


@pytest.mark.parametrize("semiring,dtype", CASES)
@pytest.mark.parametrize("kind", sorted(PACKED))
def test_packed(kind, semiring, dtype):
    rng = np.random.default_rng(len(kind))
    cuts = PACKED[kind]
    rows = cuts[-1] + (37 if kind in ("behind", "before", "none") else 0)
    a, x, h = make((rows, 9), len(cuts) - 1, semiring, dtype, rng)
    spans = list(zip(cuts[:-1], cuts[1:]))
    # what lies in rows of no sequence is not looked at
    for b, e in ((0, cuts[0]), (cuts[-1], rows)):
        a[b:e], x[b:e] = float("nan"), float("nan")
    offsets = torch.tensor(cuts, device="cuda")
    check(a, x, h, semiring, dtype, rng, spans, offsets)
    check(a, x, None, semiring, dtype, rng, spans, offsets)


@pytest.mark.parametrize("semiring", [REAL, LOG])
def test_a_sequence_does_not_reach_into_the_next(semiring):
    """infinities and NaN of one packed sequence stay in it"""
    rng = np.random.default_rng(0)
    a, x, h = make((900, 4), 3, semiring, "float32", rng)
    x[300:310] = float("nan")
    spans = [(0, 290), (290, 600), (600, 900)]
    out, final = klay().gated_scan(a, x, h, semiring, offsets=torch.tensor([0, 290, 600, 900], device="cuda"))
    assert torch.isfinite(out[:290]).all() and torch.isnan(out[310:600]).all() and torch.isfinite(out[600:]).all()
    assert torch.isfinite(final[[0, 2]]).all() and torch.isnan(final[1]).all()
    for s in (0, 2):
        alone = klay().gated_scan(a[None, slice(*spans[s])], x[None, slice(*spans[s])], h[s:s + 1], semiring)
        want = ref.scan(semiring, *(t[slice(*spans[s])].double().cpu().numpy() for t in (a, x)), h[s].double().cpu().numpy())
        ref.close(out[slice(*spans[s])].cpu().numpy(), want["h"], want["h_tol"])
        ref.close(alone[0][0].cpu().numpy(), want["h"], want["h_tol"])


# Gates above 1: the product of a stretch of them is past the largest number, what they are applied to is as small, or 0.  (Runs of gates up
# and down by `bits` bits each, 2^200 a run: past a wave's 16 steps, a tile's 128, a group of tiles.)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("run,bits", [(20, 10.0), (200, 1.0), (400, 0.5)])
@pytest.mark.parametrize("batch,time,channels", [(1, 4500, 3), (2, 1200, 130), (50, 210, 200), (260, 150, 130), (70, 60, 130)])
def test_products_out_of_range(batch, time, channels, run, bits, dtype):
    rng = np.random.default_rng(run + time)
    kind, tiny = getattr(torch, dtype), 2.0 ** -120
    shape = (batch, time, channels)
    up = np.where(np.arange(time) // run % 2 == 0, bits, -bits)[None, :, None]
    a = 2.0 ** up * rng.uniform(0.97, 1.03, size=shape) * np.where(rng.random(shape) < 0.1, -1.0, 1.0)
    x = np.where(rng.random(shape) < 0.02, tiny * rng.normal(size=shape), 0.0)
    h = tiny * rng.normal(size=(batch, channels))
    x[..., 0], h[..., 0] = 0.0, 0.0                      # a channel of zeros
    a, x, h = torch.from_numpy(a).to(kind).cuda(), torch.from_numpy(x).to(kind).cuda(), torch.from_numpy(h).float().cuda()
    check(a, x, h, REAL, dtype, rng, scale=tiny)
    if batch == 2:                                       # the same as packed sequences, one behind the other
        rows = lambda t: t.reshape(batch * time, channels)  # noqa: E731
        cuts = [0, 130, 131, time, time, 2 * time]
        check(rows(a), rows(x), torch.cat([h, h, h[:1]]), REAL, dtype, rng, list(zip(cuts[:-1], cuts[1:])), torch.tensor(cuts, device="cuda"),
              scale=tiny)


@pytest.mark.parametrize("batch,channels", [(1, 5), (150, 64)])
def test_what_is_infinite_stays_in_its_channel(batch, channels):
    rng = np.random.default_rng(batch)
    a, x, h = make((batch, 2500, channels), batch, REAL, "float32", rng)
    a = a.abs() + 0.01
    want = ref.scan(REAL, *(t[0].double().cpu().numpy() for t in (a, x, h)))
    x[:, 700, 1], a[:, 800, 2], x[:, 900, 3] = float("inf"), float("-inf"), float("nan")
    out, final = klay().gated_scan(a, x, h)
    for c, t in ((1, 700), (2, 800), (3, 900)):
        assert torch.isfinite(out[:, :t, c]).all() and not torch.isfinite(out[:, t:, c]).any() and not torch.isfinite(final[:, c]).any()
    for c in (0, 4):
        ref.close(out[0, :, c].cpu().numpy(), want["h"][:, c], want["h_tol"][:, c])


@pytest.mark.parametrize("semiring", [REAL, LOG])
def test_saved_tensors_that_come_back_with_other_strides(semiring):
    """what autograd saved may lie in the same place another way (hooks that keep it elsewhere meanwhile)"""
    rng = np.random.default_rng(1)
    a, x, h = make((3, 200, 6), 3, semiring, "float32", rng)
    dh = torch.from_numpy(rng.normal(size=a.shape)).float().cuda()
    results = []
    for moved in (False, True):
        base = torch.zeros((3, 201, 6), device="cuda")
        base[:, :-1] = a
        gates = base[:, :-1].requires_grad_(True)

        def unpack(t):
            if not moved or t.data_ptr() != gates.data_ptr():
                return t
            flat = base.detach().flatten()[:a.numel()]
            flat.copy_(a.flatten())
            return flat.view(a.shape)
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
            out, _ = klay().gated_scan(gates, x, h, semiring)
        results.append(torch.autograd.grad(out, gates, dh)[0])
    assert torch.equal(*results)


@pytest.mark.parametrize("semiring,dtype", CASES)
def test_layouts(semiring, dtype):
    rng = np.random.default_rng(9)
    a, x, h = make((3, 280, 10), 3, semiring, dtype, rng)
    wide = torch.zeros((3, 280, 33), dtype=a.dtype, device="cuda")
    wide[..., 3:13], wide[..., 15:25] = a, x
    check(a, x, h, semiring, dtype, rng, given=(wide[..., 3:13], wide[..., 15:25]))               # parts of one projection, odd starts
    swapped = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (a, x)]
    check(a, x, h, semiring, dtype, rng, given=tuple(swapped))                                    # time first in memory
    far = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (a, x)]
    check(a, x, h, semiring, dtype, rng, given=tuple(far))                                        # channels apart: copied
    shared = a[:, :, :1].expand(3, 280, 10)
    check(shared.contiguous(), x, h, semiring, dtype, rng, given=(shared, x))                     # one gate for all channels
    same = a[:1].expand(3, 280, 10)
    check(same.contiguous(), x, h, semiring, dtype, rng, given=(same, x))                         # one for all sequences


@pytest.mark.parametrize("semiring", [REAL, LOG])
def test_shared_gates_and_parts_of_the_gradient(semiring):
    k = klay()
    rng = np.random.default_rng(4)
    a, x, h = make((2, 50, 8), 2, semiring, "float32", rng)
    gate = a[:, :, :1].clone().requires_grad_(True)
    out, final = k.gated_scan(gate.expand(2, 50, 8), x, h, semiring)
    (out.sum() + final.sum()).backward()
    full = a[:, :, :1].expand(2, 50, 8).contiguous().requires_grad_(True)
    out, final = k.gated_scan(full, x, h, semiring)
    (out.sum() + final.sum()).backward()
    assert torch.allclose(gate.grad, full.grad.sum(-1, keepdim=True), rtol=1e-5, atol=1e-5)
    leaves = [t.detach().clone().requires_grad_(True) for t in (a, x, h)]
    whole = torch.autograd.grad(k.gated_scan(*leaves, semiring)[0].sum(), leaves)
    for i in range(3):               # one input at a time, and one result at a time
        one = [t.detach().requires_grad_(i == j) for j, t in enumerate((a, x, h))]
        got, = torch.autograd.grad(k.gated_scan(*one, semiring)[0].sum(), one[i])
        assert torch.equal(got, whole[i])
    last = torch.autograd.grad(k.gated_scan(*leaves, semiring)[1].sum(), leaves)
    again = torch.autograd.grad(k.gated_scan(*leaves, semiring)[0][:, -1].sum(), leaves)
    assert all(torch.allclose(p, q, rtol=1e-6, atol=1e-7) for p, q in zip(last, again))


@pytest.mark.parametrize("semiring", [REAL, LOG])
def test_gradient_against_differences(semiring):
    k = klay()
    rng = np.random.default_rng(5)
    a, x, h = make((2, 40, 3), 2, semiring, "float32", rng)
    leaves = [t.detach().requires_grad_(True) for t in (a, x, h)]
    w = [torch.from_numpy(rng.normal(size=s)).cuda() for s in ((2, 40, 3), (2, 3))]
    v = [torch.from_numpy(rng.normal(size=tuple(t.shape))).float().cuda() for t in leaves]

    def f(move):
        out = k.gated_scan(*[t.detach() + move * d for t, d in zip(leaves, v)], semiring)
        return float(sum((q * o.double()).sum() for q, o in zip(w, out)))
    out = k.gated_scan(*leaves, semiring)
    grads = torch.autograd.grad(list(out), leaves, [q.float() for q in w])
    slope = float(sum((g.double() * d.double()).sum() for g, d in zip(grads, v)))
    # the error of a central difference falls with the square of the step: two steps, and their extrapolation; fp32's own error of
    # f, u * sum |w| max |h| * 40 steps, is divided by the smaller step
    e = 2.0 ** -6
    d1, d2 = (f(e) - f(-e)) / (2 * e), (f(e / 2) - f(-e / 2)) / e
    noise = ref.U * 40 * float(sum(q.abs().sum() for q in w)) * max(1.0, float(out[0].detach().abs().max())) / (e / 2)
    assert abs((4 * d2 - d1) / 3 - slope) <= noise + 0.1 * abs(d1 - d2) + 1e-3 * abs(slope)


def test_no_steps():
    k = klay()
    h = torch.randn(3, 4, device="cuda", requires_grad=True)
    for semiring, none in ((REAL, 0.0), (LOG, float("-inf"))):
        empty = torch.empty((3, 0, 4), device="cuda")
        out, final = k.gated_scan(empty, empty, h, semiring)
        assert out.shape == (3, 0, 4) and torch.equal(final, h)
        g, = torch.autograd.grad(final, h, torch.full_like(final, 2.0))
        assert torch.equal(g, torch.full_like(h, 2.0))
        assert bool((k.gated_scan(empty, empty, None, semiring)[1] == none).all())
    none = torch.empty((0, 5, 4), device="cuda")
    assert k.gated_scan(none, none)[0].shape == (0, 5, 4)


def test_offsets_that_are_none_stay_in_the_arrays():
    """descending and negative offsets, and some past the rows: whatever comes out, the arrays around stay as they were"""
    k = klay()
    around = torch.full((3, 64, 8), 5.0, device="cuda")
    a, x = around[1] * 0.1, around[1].clone()
    for cuts in ([0, 50, 20, 64], [-5, 10, 90], [70, 80, 90], [64, 32, 0], [3, 3, -9]):
        out, final = k.gated_scan(a, x, None, REAL, offsets=torch.tensor(cuts, device="cuda"))
        torch.cuda.synchronize()
        assert out.shape == (64, 8) and bool((around == 5.0).all())


@pytest.mark.parametrize("semiring,dtype", CASES)
@pytest.mark.parametrize("batch,channels", [(1, 1), (3, 5), (17, 64), (70000, 3), (2, 1030)])
def test_one_step(batch, channels, semiring, dtype):
    k = klay()
    rng = np.random.default_rng(channels)
    a, x, h = make((batch, channels), batch, semiring, dtype, rng, impossible=semiring != REAL)
    n = lambda t: t.double().cpu().numpy()  # noqa: E731
    with np.errstate(all="ignore"):
        want = ref._step(semiring, n(a), n(h), n(x))
        tol = ref.U * (8 + 4 * np.abs(np.where(np.isfinite(want), want, 0)) + 4 * np.abs(np.where(np.isfinite(n(a) + n(h)), n(a) * n(h), 0)))
    wide = torch.zeros((batch, channels + 3), device="cuda")
    wide[:, 2:2 + channels] = h
    for state in (h.clone(), wide[:, 2:2 + channels]):
        out = k.gated_step(a, x, state, semiring)
        assert out.dtype == x.dtype
        ref.close(n(state), want, tol)
        ref.close(n(out), want, tol, dtype)
    assert not wide[:, :2].any() and not wide[:, 2 + channels:].any()
    given = torch.empty_like(a)
    assert k.gated_step(a, x, h.clone(), semiring, out=given) is given and torch.equal(given, out)


@pytest.mark.parametrize("semiring", [REAL, LOG])
@pytest.mark.parametrize("shape", [(2, 30, 7), (1, 3000, 64), (40, 300, 64)])
def test_streams_and_graphs(shape, semiring):
    """two streams at once, and a captured forward and backward call replayed over new inputs, between eager calls"""
    k = klay()
    rng = np.random.default_rng(6)
    sets = [make(shape, shape[0], semiring, "float32", rng) for _ in range(4)]

    def both(a, x, h):
        leaves = [t.detach().requires_grad_(True) for t in (a, x, h)]
        out, final = k.gated_scan(*leaves, semiring)
        return [out.detach(), final.detach()] + list(torch.autograd.grad([out, final], leaves, [torch.ones_like(out), torch.ones_like(final)]))
    want = [both(*s) for s in sets]
    assert all(torch.equal(p, q) for p, q in zip(want[0], both(*sets[0])))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i, s in enumerate(sets):
        with torch.cuda.stream(streams[i % 2]):
            got.append(both(*s))
    torch.cuda.synchronize()
    for p, q in zip(want, got):
        assert all(torch.equal(b, c) for b, c in zip(p, q))
    fixed = [t.clone() for t in sets[0]]
    with torch.cuda.stream(streams[0]):
        both(*fixed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both(*fixed)
    for i in (1, 3, 0):
        for t, s in zip(fixed, sets[i]):
            t.copy_(s)
        graph.replay()
        eager = both(*sets[i])
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want[i])) and all(torch.equal(p, q) for p, q in zip(eager, want[i]))


def test_the_step_follows_the_scan():
    """prefill a prompt with the scan, go on one token at a time: the states of the scan over all of it"""
    k = klay()
    rng = np.random.default_rng(8)
    for semiring, dtype in CASES:
        a, x, h = make((4, 60, 33), 4, semiring, dtype, rng)
        with torch.no_grad():
            out, final = k.gated_scan(a, x, h, semiring)
            _, state = k.gated_scan(a[:, :40], x[:, :40], h, semiring)
            for t in range(40, 60):
                y = k.gated_step(a[:, t], x[:, t], state, semiring)
        want = [ref.scan(semiring, *(q[b].double().cpu().numpy() for q in (a, x)), h[b].double().cpu().numpy()) for b in range(4)]
        for b in range(4):
            ref.close(state[b].cpu().numpy(), want[b]["final"], want[b]["final_tol"])
            ref.close(final[b].cpu().numpy(), want[b]["final"], want[b]["final_tol"])
            ref.close(y[b].double().cpu().numpy(), want[b]["h"][-1], want[b]["h_tol"][-1], dtype)
