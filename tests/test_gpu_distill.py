"""Divergence of given logits from a teacher's list (GPU) against the 64-bit definition: row lengths around the kernels' waves, vectors and chunks,
lists at their borders, every type, masks, sure students and teachers, layouts, temperatures."""
import pytest
import torch

from tests import head_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
ids = lambda v: str(v).replace("torch.", "")  # noqa: E731


def klay():
    import paper_2410_11415_amd as pkg
    return pkg


def make(rows, vocab, k, dtype, seed=0, kind="plain", rest=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + rows * 31 + vocab * 5 + k)
    x = 2.5 * torch.randn((rows, vocab), generator=g, device="cuda")
    t = torch.randint(0, vocab, (rows, k), generator=g, device="cuda")
    if k <= vocab:                                      # different tokens
        t = torch.rand((rows, vocab), generator=g, device="cuda").topk(k, dim=1)[1] if vocab <= 4096 else t
    if kind in ("sure", "masked"):
        x.scatter_add_(1, t[:, :1], 60.0 * torch.rand((rows, 1), generator=g, device="cuda"))
    if kind == "masked":
        x[torch.rand(x.shape, generator=g, device="cuda") < 0.3] = -torch.inf
        x.scatter_(1, t, 2.5 * torch.randn((rows, k), generator=g, device="cuda"))
        t[torch.rand(t.shape, generator=g, device="cuda") < 0.2] = -1
        t[0] = -1
    z = 2.5 * torch.randn((rows, k), generator=g, device="cuda")
    if rest:
        z = torch.log_softmax(z, 1) + torch.log(0.1 + 0.899 * torch.rand((rows, 1), generator=g, device="cuda"))
    return x.to(dtype), t, z, g


def check(x, t, z, g, temperature=1.0, rest=False, given=None):
    R = x.shape[0]
    d = torch.randn(R, generator=g, device="cuda")
    want, dx, dx_tol = ref.distill(x.detach().double(), t, z, temperature, rest, torch.zeros(R, dtype=torch.float64, device="cuda"), d.double())
    leaf = (x if given is None else given).detach().requires_grad_(True)
    loss = klay().token_distill(leaf, t, z, temperature=temperature, rest=rest)
    assert loss.dtype == torch.float32
    ref.close(loss, want, what="loss")
    dl, = torch.autograd.grad(loss, leaf, d)
    assert dl.dtype == x.dtype and dl.shape == x.shape
    ref.close(dl, (dx, dx_tol), x.dtype, "dlogits")


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("vocab", [1, 2, 3, 10, 63, 64, 65, 511, 512, 513, 520, 1023, 2047, 2049, 4099, 8195, 33000])
def test_row_lengths(vocab, dtype):
    for i, k in enumerate((1, min(vocab, 7))):
        check(*make(5, vocab, k, dtype, i, rest=bool(i)), rest=bool(i), temperature=1.0 + i)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,vocab,k", [(700, 70001, 20), (2, 300007, 64), (513, 600, 5), (2000, 10, 3)])
def test_many_and_long_rows(rows, vocab, k, dtype):
    """a workgroup of four waves a row, of sixteen; more vectors than are marked at a time"""
    if dtype == torch.float32 and rows == 700:
        vocab = 35003
    check(*make(rows, vocab, k, dtype, 3, "sure", True), rest=True)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("kind", ["sure", "masked"])
@pytest.mark.parametrize("vocab,k", [(40, 4), (600, 20), (5001, 64)])
def test_masks_and_sure_students(vocab, k, kind, dtype):
    check(*make(40, vocab, k, dtype, 4, kind, True), rest=True)
    check(*make(40, vocab, k, dtype, 5, kind), temperature=3.0)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_lists_at_the_borders_of_vectors(shift, dtype):
    """neighbouring tokens, whole vectors of them, a row's first and last"""
    x, _, _, g = make(6, 9000, 1, dtype, 6)
    wide = torch.zeros((6, 9016), dtype=dtype, device="cuda")
    wide[:, shift:shift + 9000] = x
    lists = [list(range(16)), list(range(8984, 9000)), list(range(5, 21)), [0, 1, 7, 8, 9, 15, 16, 17, 8191, 8192, 8193, 4095, 4096, 8998, 8999, 2048],
             list(range(4090, 4106)), list(range(2043, 2059))]
    t = torch.tensor(lists, device="cuda")
    for rest in (False, True):
        z = torch.log_softmax(torch.randn(t.shape, generator=g, device="cuda"), 1) - 0.3
        check(x, t, z, g, rest=rest, given=wide[:, shift:shift + 9000])


@pytest.mark.parametrize("vocab,k", [(30, 100), (3000, 1024), (700, 65)])
def test_long_and_repeated_lists(vocab, k):
    for rest in (False, True):
        x, _, z, g = make(9, vocab, k if k <= vocab else 1, torch.float32, 7, rest=rest)
        t = torch.randint(0, vocab, (9, k), generator=g, device="cuda")
        z = torch.log_softmax(torch.randn(t.shape, generator=g, device="cuda"), 1) - (0.2 if rest else 0)
        check(x, t, z, g, rest=rest)


@pytest.mark.parametrize("temperature", [0.001, 0.05, 1000.0])
def test_temperatures(temperature):
    check(*make(20, 700, 5, torch.float32, 8), temperature=temperature)
    check(*make(20, 300, 5, torch.bfloat16, 8, rest=True), temperature=temperature, rest=True)


def test_a_student_that_knows():
    """the student's distribution is the teacher's: a divergence near 0, to what 2^-24 of the logarithms allows"""
    x, t, _, g = make(50, 1000, 20, torch.float32, 9)
    z = torch.log_softmax(x.double(), 1).gather(1, t).float()
    check(x, t, z, g, rest=True)
    loss = klay().token_distill(x, t, z, rest=True)
    assert float(loss.abs().max()) < 1e-6


def test_every_token_listed():
    x, _, _, g = make(50, 12, 1, torch.float32, 10)
    t = torch.stack([torch.randperm(12, generator=g, device="cuda") for _ in range(50)])
    z = torch.randn(t.shape, generator=g, device="cuda")
    check(x, t, z, g)
    check(x, t, torch.log_softmax(z, 1), g, rest=True)


@pytest.mark.parametrize("vocab", [50, 2000])
def test_what_is_not_there(vocab):
    """lists of nothing, forbidden tokens, tokens out of range, teachers and students of NaN and infinities"""
    x, t, z, g = make(12, vocab, 4, torch.float32, 11)
    t[1] = -1
    t[2, 1] = vocab
    z[3, 2] = float("nan")
    z[4, 0] = float("inf")
    z[5, 1] = -torch.inf                                # the teacher excludes one of its own
    z[6] = -torch.inf                                   # all of them
    x[7] = float("nan")
    x[8, int(t[8, 0]) ^ 1] = float("inf")
    x[9, t[9, 2]] = -torch.inf                          # the student excludes one that the teacher gives mass to
    x[10] = -torch.inf
    leaf = x.requires_grad_(True)
    loss = klay().token_distill(leaf, t, z)
    nan = torch.isnan(loss)
    assert nan.tolist() == [False, False, True, True, True, False, False, True, True, False, False, False]
    assert float(loss[1]) == 0 and float(loss[6]) == 0 and float(loss[9]) == float("inf") and float(loss[10]) == float("inf")
    d, = torch.autograd.grad(loss, leaf, torch.ones_like(loss))
    assert bool((d[[1, 6, 10]] == 0).all()) and bool(torch.isfinite(d[[0, 5, 9, 11]]).all())
    d, = torch.autograd.grad(klay().token_distill(leaf, t, z), leaf, torch.zeros_like(loss))
    assert bool((d == 0).all())                         # an adjoint of 0 gives 0, whatever the row holds
    keep = [0, 5, 11]
    want, _, _ = ref.distill(x.detach().double()[keep], t[keep], z[keep], 1.0, False, torch.zeros(3, dtype=torch.float64, device="cuda"))
    ref.close(loss[keep], want, what="loss")


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("layout", ["sequences", "across", "teacher across", "vector"])
def test_layouts(layout, dtype):
    x, t, z, g = make(24, 700, 5, dtype, 12)
    want = klay().token_distill(x, t, z)
    if layout == "sequences":
        wide = torch.zeros((4, 7, 705), dtype=dtype, device="cuda")
        wide[:, 1:, 2:702] = x.view(4, 6, 700)
        got = klay().token_distill(wide[:, 1:, 2:702], t.view(4, 6, 5), z.view(4, 6, 5)).flatten()
    elif layout == "across":
        got = klay().token_distill(x.t().contiguous().t(), t, z)
    elif layout == "teacher across":
        got = klay().token_distill(x, t.t().contiguous().t(), z.t().contiguous().t())
    else:
        got, want = klay().token_distill(x[3], t[3], z[3]), want[3]
    # (rows that start elsewhere are summed in another order)
    assert float((got - want).abs().max()) <= 4 * ref.terms(700) + 4 * ref.U * float(want.abs().max())


def test_the_same_bits_and_graphs():
    x, t, z, g = make(30, 3000, 6, torch.bfloat16, 13)
    leaf = x.requires_grad_(True)

    def step():
        loss = klay().token_distill(leaf, t, z, temperature=2.0)
        return loss, torch.autograd.grad(loss, leaf, torch.ones_like(loss))[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        with torch.no_grad():
            leaf.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        want = step()
        again = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(out, want, again):
            assert torch.equal(a, b) and torch.equal(b, c)
