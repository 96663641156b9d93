"""Heads whose rows begin and end anywhere (GPU): starts and strides of single elements, widths behind whole pieces of 16 bytes, memory of others around
the inputs and the gradients; weights that the bias bars, many and few; two calls at once; all of the operators in one step of training."""
import pytest
import torch

from paper_2410_11415_amd import binding, operators
from tests import head_ref as ref
from tests.test_gpu_head import DTYPES, adjoints, check_distill, check_tokens, ids, klay, make

pytestmark = pytest.mark.gpu


def among(t, start, extra, fill=float("nan")):
    """t in memory of others: its first element `start` behind a multiple of 256 bytes, its rows `extra` elements apart"""
    rows, width = t.shape
    stride = width + extra
    big = torch.full((start + rows * stride + 64,), fill, dtype=t.dtype, device="cuda")
    view = big.as_strided((rows, width), (stride, 1), start)
    view.copy_(t)
    return view


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("width", [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 17, 30, 31, 33, 62, 63, 66, 71, 127, 129])
def test_widths(width, dtype):
    hidden, weight, bias, tokens, g = make(37, width, 141, 2, dtype, 40)
    check_tokens(hidden, weight, bias, tokens, g)
    check_distill(hidden, weight, bias, tokens, g, temperature=0.7)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("width", [3, 8, 21, 66])
@pytest.mark.parametrize("hidden_at,weight_at", [((0, 0), (1, 0)), ((1, 1), (0, 2)), ((2, 0), (2, 2)), ((3, 4), (6, 0)), ((2, 6), (5, 3)), ((4, 1), (0, 1)), ((0, 3), (0, 8))])
def test_rows_anywhere(hidden_at, weight_at, width, dtype):
    """nothing of what lies around a row is taken for a part of it"""
    hidden, weight, bias, tokens, g = make(41, width, 150, 3, dtype, 41)
    given = among(hidden, *hidden_at), among(weight, *weight_at)
    check_tokens(hidden, weight, bias, tokens, g, given=given)
    check_distill(hidden, weight, bias, tokens, g, given=given, rest=True)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,width,vocab", [(300, 45, 9000), (600, 130, 3001), (40, 1027, 2000)])
def test_large_tiles_of_odd_widths(rows, width, vocab, dtype):
    hidden, weight, bias, tokens, g = make(rows, width, vocab, 2, dtype, 42)
    given = among(hidden, 2, 2 + width % 2), among(weight, 4, 2 + width % 2)
    check_tokens(hidden, weight, bias, tokens, g, given=given)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,width,vocab", [(64, 1024, 16400), (64, 1027, 16400), (33, 2240, 16001), (65, 1024, 16384), (32, 2560, 16384), (20000, 1024, 60),
                                             (24, 40000, 2000), (16, 550000, 130)])
def test_few_rows_of_large_weights(rows, width, vocab, dtype):
    hidden, weight, bias, tokens, g = make(rows, width, vocab, 1, dtype, 47)
    check_tokens(hidden, weight, bias, tokens, g)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,width,vocab", [(5, 3, 7), (33, 19, 130), (70, 66, 257), (300, 45, 9000)])
def test_gradients_end_where_they_end(rows, width, vocab, dtype):
    """what lies behind the gradients stays as it was"""
    hidden, weight, bias, tokens, g = make(rows, width, vocab, 1, dtype, 43)
    args, _ = operators._head_args(hidden, weight, bias, tokens)
    logp, kept = torch.empty(rows, 1, device="cuda"), operators._kept(hidden, args)
    work, size = operators._workspace(hidden, args, False)
    stream = operators._stream(args.device)
    binding.klay_head_forward(args, logp.data_ptr(), None, None, kept.data_ptr(), work.data_ptr(), size, stream)
    d = torch.randn(rows, 1, generator=g, device="cuda")
    room = [torch.full((t.numel() + 100,), 7.0, dtype=t.dtype, device="cuda") for t in (hidden, weight, bias)]
    work, size = operators._workspace(hidden, args, True)
    binding.klay_head_backward(args, kept.data_ptr(), d.data_ptr(), None, None, *(t.data_ptr() for t in room), work.data_ptr(), size, stream)
    inputs = [t.detach().requires_grad_(True) for t in (hidden, weight, bias)]
    want = torch.autograd.grad(klay().head_logprobs(inputs[0], inputs[1], tokens, inputs[2]).logp, inputs, d)
    for got, grad in zip(room, want):
        assert torch.equal(got[:grad.numel()].view(grad.shape), grad) and bool((got[grad.numel():] == 7).all())


# weights of a few bytes, which are copied along; of more than 4 MB, which are only if need be; in several pieces of the vocabulary
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,width,vocab", [(30, 40, 500), (40, 520, 9001), (21, 1101, 4003), (2100, 121, 20011)])
@pytest.mark.parametrize("first", [0, 0.9])
def test_barred_weights_hold_anything(first, rows, width, vocab, dtype):
    hidden, weight, bias, tokens, g = make(rows, width, vocab, 1, dtype, 44)
    gone = torch.rand(vocab, generator=g, device="cuda") < 0.3
    gone[:int(first * vocab)] = False
    bias[gone] = -torch.inf
    d = torch.randn(rows, 1, generator=g, device="cuda")
    out = []
    for hole in (0.0, float("nan"), float("inf"), -float("inf")):
        w = weight.clone()
        w[gone, :: 7] = hole
        inputs = [t.detach().requires_grad_(True) for t in (hidden, w, bias)]
        r = klay().head_logprobs(inputs[0], inputs[1], tokens, inputs[2])
        grads = torch.autograd.grad(r.logp, inputs, d)
        assert all(bool(torch.isfinite(t).all()) for t in grads)
        out.append((r.logp, *grads))
    for other in out[1:]:
        for a, b in zip(out[0], other):
            assert torch.equal(a, b)


def test_calls_on_two_streams_at_once():
    made = [make(rows, 130, 5000, 2, torch.bfloat16, 45) for rows in (70, 300)]
    streams = [torch.cuda.Stream() for _ in made]

    def step(hidden, weight, bias, tokens, grad):
        inputs = [t.detach().requires_grad_(True) for t in (hidden, weight, bias)]
        r = klay().head_logprobs(inputs[0], inputs[1], tokens, inputs[2], entropy=True)
        return (r.logp, *torch.autograd.grad([r.logp, r.entropy], inputs, grad))
    grads = [adjoints(m[4], m[3].shape, m[3].shape[:1]) for m in made]
    want = [step(*m[:4], d) for m, d in zip(made, grads)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(step(*made[i][:4], grads[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for turn in got[i]:
            for a, b in zip(turn, want[i]):
                assert torch.equal(a, b)


def test_the_same_index_twice_and_the_same_tensor_as_both():
    """tokens listed twice count twice; weights that are the hidden states themselves get both gradients"""
    x = torch.randn(24, 40, device="cuda")
    t = torch.tensor([[3, 3, 5]], device="cuda").expand(24, 3)
    a = x.clone().requires_grad_(True)
    both, = torch.autograd.grad(klay().head_logprobs(a, a, t).logp.sum(), a)
    b, c = x.clone().requires_grad_(True), x.clone().requires_grad_(True)
    one, other = torch.autograd.grad(klay().head_logprobs(b, c, t).logp.sum(), (b, c))
    assert torch.equal(both, one + other)
    z = torch.tensor([[1.0, 1.0, -1.0]], device="cuda").expand(24, 3)
    check_distill(x, x.clone(), None, t.contiguous(), torch.Generator(device="cuda").manual_seed(3))
    assert bool(torch.isfinite(klay().head_distill(x, x, t, z)).all())


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_a_step_of_training_from_a_teacher(dtype):
    """the teacher's top tokens, the student's divergence from them, its own answers' log probabilities: as they are used together"""
    hidden, weight, bias, tokens, g = make(60, 48, 700, 1, dtype, 46)
    teacher = hidden.float() @ weight.float().t() + 0.5 * torch.randn(60, 700, generator=g, device="cuda")
    top = klay().token_logprobs(teacher, top=8)
    inputs = [t.detach().requires_grad_(True) for t in (hidden, weight, bias)]
    loss = klay().head_distill(inputs[0], inputs[1], top.top_tokens, top.top_logp, inputs[2], rest=True).mean() - \
        klay().head_logprobs(inputs[0], inputs[1], tokens, inputs[2]).logp.mean()
    got = torch.autograd.grad(loss, inputs)
    x, slip = ref.logits_of(hidden, weight, bias)
    up = torch.full((60,), 1 / 60.0, device="cuda").double()
    a, dx_a, tol_a = ref.distill(x, top.top_tokens, top.top_logp, 1.0, True, slip, up)
    b, dx_b, tol_b = ref.tokens(x, tokens, slip, -up[:, None])
    want = ref.gradients(dx_a, tol_a, hidden, weight), ref.gradients(dx_b, tol_b, hidden, weight)
    for grad, name in zip(got, ("dhidden", "dweight", "dbias")):
        (va, ta), (vb, tb) = want[0][name], want[1][name]
        # two gradients rounded to the type, and their sum, no larger than both
        half = torch.finfo(grad.dtype).eps / 2
        most = va.abs() + vb.abs() + ta + tb
        assert bool(((grad.double() - va - vb).abs() <= ta + tb + 2 * half * (1 + half) * most + 3 * ref.TINY[grad.dtype]).all()), name


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,vocab", [(20, 2), (60, 2), (200, 4000), (900, 20000)])
def test_long_sums_lean_to_no_side(rows, vocab, dtype):
    """The mean error of many logits, each a sum of 8192 terms most of which have its sign.  A row's sum is rounded once every sixteen k's, by half a step of
    at most the sum, 2^-24: spread like a walk of 512 steps of 2^-24 / sqrt(3), 7.8e-7 of it, and their mean over the rows 1 / sqrt(rows) of that, five times
    of which are allowed; to this the products of parts of fp32 that are not made, 2^-24, and a rounding of the result."""
    g = torch.Generator(device="cuda").manual_seed(48)
    w0 = torch.randn(8192, generator=g, device="cuda")
    hidden = (torch.randn(rows, 8192, generator=g, device="cuda") + 0.5 * w0).to(dtype)
    weight = torch.zeros(vocab, 8192, dtype=dtype, device="cuda")
    weight[0] = (w0 * (80 / 8192)).to(dtype)
    x = hidden.double() @ weight[0].double()
    assert float(x.min()) > 30
    tokens = torch.zeros(rows, 1, dtype=torch.int64, device="cuda")
    got = -klay().head_logprobs(hidden, weight, tokens, complement=True).neg[:, 0].double()     # ln(1 + e^x / (V - 1))
    want = x - torch.log(torch.tensor(vocab - 1.0).double()) + torch.log1p((vocab - 1) * torch.exp(-x))
    mean = ((got - want) / x).mean().abs()
    assert float(mean) <= 5 * 7.8e-7 / rows ** 0.5 + 2.0 ** -24 + 2.0 ** -24


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,width,vocab", [(5, 24, 300), (70, 65, 1000), (300, 48, 9000)])
def test_biases_of_the_lowest_value(rows, width, vocab, dtype):
    """A bias of fp32's lowest value bars a token as -inf does, to the last bit; where it is everywhere, all tokens are alike."""
    hidden, weight, bias, tokens, g = make(rows, width, vocab, 2, dtype, 49)
    gone = torch.rand(vocab, generator=g, device="cuda") < 0.5
    gone[0] = False
    tokens = torch.where(gone[tokens], 0, tokens)
    low = torch.finfo(torch.float32).min
    d = adjoints(g, (rows, 2), (rows, 2), (rows,))
    out = []
    for least in (low, -torch.inf):
        inputs = [t.detach().requires_grad_(True) for t in (hidden, weight, torch.where(gone, least, bias))]
        r = klay().head_logprobs(inputs[0], inputs[1], tokens, inputs[2], complement=True, entropy=True)
        out.append((*r, *torch.autograd.grad(list(r), inputs, d)))
    for a, b in zip(*out):
        assert torch.equal(a, b)
    inputs = [t.detach().requires_grad_(True) for t in (hidden, weight, torch.full_like(bias, low))]
    r = klay().head_logprobs(inputs[0], inputs[1], tokens, inputs[2], complement=True, entropy=True)
    ln_v = torch.tensor(float(vocab)).double().log().item()
    # (ln V from sums of V ones: one rounding of the result and of V's logarithm in it)
    assert float((r.logp.double() + ln_v).abs().max()) <= 4 * 2.0 ** -24 * ln_v
    assert float((r.entropy.double() - ln_v).abs().max()) <= 4 * 2.0 ** -24 * ln_v
    assert all(bool(torch.isfinite(t).all()) for t in torch.autograd.grad(list(r), inputs, d))


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_barred_weights_change_under_a_graph(dtype):
    """whether the weights have to be copied is found out at every replay"""
    hidden, weight, bias, tokens, g = make(40, 520, 9001, 1, dtype, 50)
    gone = torch.rand(9001, generator=g, device="cuda") < 0.3
    bias[gone] = -torch.inf
    ins = [t.detach().clone().requires_grad_(True) for t in (hidden, weight, bias)]
    ones = torch.ones(40, 1, device="cuda")

    def step():
        r = klay().head_logprobs(ins[0], ins[1], tokens, ins[2])
        return [r.logp.detach(), *torch.autograd.grad(r.logp, ins, ones)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for turn, hole in enumerate((0.5, float("nan"), 0.25, float("inf"), float("nan"), 0.0)):
        with torch.no_grad():
            ins[0].copy_(torch.randn(hidden.shape, generator=g, device="cuda"))
            ins[1][gone, ::5] = hole
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), turn
        assert all(bool(torch.isfinite(t).all()) for t in out[1:])         # (a barred token's own logp is -inf)
