"""Log probabilities and divergences straight from hidden states (GPU) against the 64-bit definition: sizes around tiles, waves, matrix
instructions and pieces, every type, masks, sure rows, repeated tokens, padding, layouts; the same call twice, on streams, in graphs, under hooks."""
import pytest
import torch

from tests import head_ref as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
ids = lambda v: str(v).replace("torch.", "")  # noqa: E731


def klay():
    import paper_2410_11415_amd as pkg
    return pkg


def make(rows, width, vocab, k, dtype, seed=0, kind="plain", bias=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + rows * 31 + width * 17 + vocab * 5 + k)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    weight = normal(vocab, width) * (2.5 / width ** 0.5)
    sure = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    hidden = normal(rows, width)
    tokens = torch.randint(0, vocab, (rows, k), generator=g, device="cuda")
    b = normal(vocab) if bias else None
    if kind in ("sure", "masked"):
        lean = weight[sure] / (weight[sure] ** 2).sum(1, keepdim=True)
        hidden = hidden + 40.0 * torch.rand((rows, 1), generator=g, device="cuda") * lean
        if k:
            tokens[:, 0] = sure
    if kind == "masked":
        b = normal(vocab)
        b[torch.rand(vocab, generator=g, device="cuda") < 0.3] = -torch.inf
        tokens[torch.rand(tokens.shape, generator=g, device="cuda") < 0.2] = -1
        if rows > 2:
            tokens[2] = -100
    return hidden.to(dtype), weight.to(dtype), b, tokens, g


def adjoints(g, *shapes):
    return [None if s is None else torch.randn(s, generator=g, device="cuda") for s in shapes]


def check_tokens(hidden, weight, bias, tokens, g, complement=True, entropy=True, grads=True, given=None):
    R, K = hidden.shape[0], tokens.shape[1]
    x, slip = ref.logits_of(hidden, weight, bias)
    d = adjoints(g, (R, K), (R, K) if complement else None, (R,) if entropy else None) if grads else [None] * 3
    want, dx, dx_tol = ref.tokens(x, tokens, slip, *(None if v is None else v.double() for v in d))
    inputs = [t.detach().requires_grad_(grads) for t in (given or (hidden, weight)) + ((bias,) if bias is not None else ())]
    got = klay().head_logprobs(inputs[0], inputs[1], tokens, inputs[2] if bias is not None else None, complement=complement, entropy=entropy)
    for name in ["logp"] + ["neg"] * complement + ["entropy"] * entropy:
        assert getattr(got, name).dtype == torch.float32
        ref.close(getattr(got, name), want[name], what=name)
    assert (got.neg is None) == (not complement) and (got.entropy is None) == (not entropy)
    if grads:
        outs = [(o, v) for o, v in ((got.logp, d[0]), (got.neg, d[1]), (got.entropy, d[2])) if v is not None]
        check_gradients(torch.autograd.grad([o for o, _ in outs], inputs, [v for _, v in outs]), inputs, dx, dx_tol, hidden, weight)


def check_gradients(got, inputs, dx, dx_tol, hidden, weight):
    want = ref.gradients(dx, dx_tol, hidden, weight)
    for t, given, name in zip(got, inputs, ("dhidden", "dweight", "dbias")):
        assert t.dtype == given.dtype and t.shape == given.shape
        ref.close(t, want[name], t.dtype, name)


def check_distill(hidden, weight, bias, tokens, g, temperature=1.0, rest=False, grads=True, given=None):
    x, slip = ref.logits_of(hidden, weight, bias)
    teacher = torch.randn(tokens.shape, generator=g, device="cuda") * 2
    if rest:
        teacher = torch.log_softmax(teacher, 1) + torch.log(0.1 + 0.85 * torch.rand((tokens.shape[0], 1), generator=g, device="cuda"))
    d = torch.randn(hidden.shape[0], generator=g, device="cuda") if grads else None
    want, dx, dx_tol = ref.distill(x, tokens, teacher, temperature, rest, slip, None if d is None else d.double())
    inputs = [t.detach().requires_grad_(grads) for t in (given or (hidden, weight)) + ((bias,) if bias is not None else ())]
    loss = klay().head_distill(inputs[0], inputs[1], tokens, teacher, inputs[2] if bias is not None else None,
                               temperature=temperature, rest=rest)
    ref.close(loss, want, what="loss")
    if grads:
        check_gradients(torch.autograd.grad(loss, inputs, d), inputs, dx, dx_tol, hidden, weight)


# rows around a tile's (32, 64, 128), widths around pieces of 16 bytes and stages, vocabularies around a tile's columns
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,width,vocab,k", [(1, 1, 1, 1), (1, 8, 2, 1), (2, 7, 3, 2), (5, 16, 10, 10), (31, 64, 127, 3), (32, 65, 128, 1),
                                                (33, 63, 129, 4), (64, 128, 255, 2), (65, 129, 257, 5), (127, 100, 300, 1), (130, 33, 513, 3),
                                                (257, 136, 1000, 2), (3, 515, 77, 6), (300, 12, 1, 1), (16, 1024, 640, 2)])
def test_sizes(rows, width, vocab, k, dtype):
    check_tokens(*make(rows, width, vocab, k, dtype))
    check_distill(*make(rows, width, vocab, k, dtype, 1), rest=bool(k % 2), temperature=1.5 if k > 2 else 1.0)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("kind", ["sure", "masked"])
@pytest.mark.parametrize("rows,width,vocab,k", [(9, 24, 40, 3), (70, 40, 300, 4), (200, 96, 700, 2)])
def test_masks_and_sure_rows(rows, width, vocab, k, kind, dtype):
    check_tokens(*make(rows, width, vocab, k, dtype, 2, kind))
    check_distill(*make(rows, width, vocab, k, dtype, 3, kind), rest=True)
    check_distill(*make(rows, width, vocab, k, dtype, 4, "sure"), temperature=2.0)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("complement,entropy", [(False, False), (True, False), (False, True)])
def test_single_outputs(complement, entropy, dtype):
    check_tokens(*make(40, 48, 260, 3, dtype, 5), complement=complement, entropy=entropy)
    check_tokens(*make(40, 48, 260, 3, dtype, 5, bias=False), complement=complement, entropy=entropy, grads=False)


# 256 x 256 tiles, in one piece and in several, the last one ragged
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,width,vocab,k", [(400, 72, 25000, 3), (2100, 40, 20011, 1)])
def test_large_tiles_and_pieces(rows, width, vocab, k, dtype):
    check_tokens(*make(rows, width, vocab, k, dtype, 6, "sure"), complement=False)
    check_distill(*make(rows, width, vocab, k, dtype, 7, bias=False), rest=True)


def test_many_rows():
    """more rows than are worked on at a time, of a teacher whose rows lie at two strides"""
    hidden, weight, bias, tokens, g = make(16384 + 300, 16, 40, 3, torch.bfloat16, 8)
    check_tokens(hidden, weight, bias, tokens, g)
    check_distill(hidden, weight, bias, tokens, g, rest=True)
    rows = (16384 + 300) // 4
    x = hidden.view(4, rows, 16)
    teacher = torch.randn((4, rows + 1, 3), generator=g, device="cuda")
    apart = torch.full((4, rows + 1, 3), -1, device="cuda")
    apart[:, 1:] = tokens.view(4, rows, 3)
    a = klay().head_distill(x, weight, apart[:, 1:], teacher[:, 1:], bias)
    b = klay().head_distill(hidden, weight, tokens, teacher[:, 1:].reshape(-1, 3), bias)
    assert torch.equal(a.flatten(), b)


@pytest.mark.parametrize("vocab,k", [(30, 100), (3000, 1024), (700, 65), (700, 64)])
def test_long_lists(vocab, k):
    """lists beyond a wave's lanes, most of the vocabulary among them, tokens more than once"""
    check_tokens(*make(20, 32, vocab, k, torch.float32, 9))
    check_tokens(*make(20, 32, vocab, k, torch.bfloat16, 9, "masked"))
    check_distill(*make(20, 32, vocab, k, torch.float32, 10), rest=True)
    check_distill(*make(20, 32, vocab, k, torch.bfloat16, 10, "masked"))


def test_every_token_listed():
    """nothing is left for the others"""
    hidden, weight, bias, _, g = make(50, 24, 10, 1, torch.float32, 11)
    every = torch.stack([torch.randperm(10, generator=g, device="cuda") for _ in range(50)])
    check_tokens(hidden, weight, bias, every, g)
    check_distill(hidden, weight, bias, every, g, rest=True)
    check_distill(hidden, weight, bias, every, g)


def test_no_tokens():
    hidden, weight, bias, _, g = make(40, 24, 100, 1, torch.float32, 12)
    check = klay().head_logprobs(hidden, weight, None, bias, entropy=True)
    none = klay().head_logprobs(hidden, weight, torch.zeros((40, 0), dtype=torch.int64, device="cuda"), bias, entropy=True)
    assert check.logp is None and none.logp.shape == (40, 0) and torch.equal(check.entropy, none.entropy)
    check_tokens(hidden, weight, bias, torch.zeros((40, 0), dtype=torch.int64, device="cuda"), g, complement=False)


def test_nothing_allowed():
    hidden, weight, _, tokens, g = make(6, 16, 50, 2, torch.float32, 13)
    bias = torch.full((50,), -torch.inf, device="cuda")
    ins = [t.requires_grad_(True) for t in (hidden, weight, bias)]
    r = klay().head_logprobs(ins[0], ins[1], tokens, ins[2], complement=True, entropy=True)
    assert bool((r.logp == -torch.inf).all()) and bool((r.neg == 0).all()) and bool((r.entropy == 0).all())
    grads = torch.autograd.grad([r.logp.sum(), r.neg.sum(), r.entropy.sum()], ins)
    assert all(bool((t == 0).all()) for t in grads)


def test_tokens_out_of_range():
    hidden, weight, bias, tokens, g = make(40, 16, 50, 3, torch.bfloat16, 14)
    tokens[3, 1], tokens[7] = 50, 1 << 40
    r = klay().head_logprobs(hidden, weight, tokens, bias, complement=True)
    want, _, _ = ref.tokens(*[ref.logits_of(hidden, weight, bias)[0], tokens, ref.logits_of(hidden, weight, bias)[1]])
    ref.close(r.logp, want["logp"], what="logp")
    ref.close(r.neg, want["neg"], what="neg")
    w = weight.detach().requires_grad_(True)
    h = hidden.detach().requires_grad_(True)
    dh, = torch.autograd.grad(klay().head_logprobs(h, weight, tokens, bias).logp[7].sum(), h)
    assert bool(torch.isnan(dh[7]).all()) and bool((dh[:7] == 0).all()) and bool((dh[8:] == 0).all())
    loss = klay().head_distill(hidden, w, tokens, torch.zeros(tokens.shape, device="cuda"), bias)
    assert bool(torch.isnan(loss[[3, 7]]).all()) and int(torch.isnan(loss).sum()) == 2


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("hole", [float("nan"), float("inf")])
def test_rows_of_padding(dtype, hole):
    """rows that nothing is asked of may hold anything: they change no other row and no gradient"""
    hidden, weight, bias, tokens, g = make(70, 40, 300, 2, dtype, 15)
    tokens[::3] = -1
    clean = hidden.clone()
    clean[::3] = 0
    dirty = hidden.clone()
    dirty[::3] = hole
    out = []
    for h in (clean, dirty):
        ins = [h.requires_grad_(True), weight.detach().requires_grad_(True), bias.detach().requires_grad_(True)]
        r = klay().head_logprobs(ins[0], ins[1], tokens, ins[2], complement=True)
        loss = klay().head_distill(ins[0], ins[1], tokens, torch.zeros(tokens.shape, device="cuda"), ins[2])
        out.append([r.logp, r.neg, loss] + list(torch.autograd.grad([r.logp.sum(), r.neg.sum()], ins)) + list(torch.autograd.grad(loss.sum(), ins)))
    for a, b in zip(*out):
        assert torch.equal(a, b)
    assert bool((out[1][3][::3] == 0).all())


def test_forbidden_tokens_hold_anything():
    hidden, weight, bias, tokens, g = make(70, 40, 300, 2, torch.bfloat16, 16)
    tokens %= 290
    bias[295:] = -torch.inf
    out = []
    for hole in (0.0, float("nan"), float("inf")):
        w = weight.clone()
        w[295:] = hole
        ins = [hidden.detach().requires_grad_(True), w.requires_grad_(True), bias.detach().requires_grad_(True)]
        r = klay().head_logprobs(ins[0], ins[1], tokens, ins[2], complement=True, entropy=True)
        out.append([r.logp, r.neg, r.entropy] + list(torch.autograd.grad([r.logp.sum(), r.neg.sum(), r.entropy.sum()], ins)))
    for other in out[1:]:
        for a, b in zip(out[0], other):
            assert torch.equal(a, b)


def test_bad_rows_stay_by_themselves():
    hidden, weight, bias, tokens, g = make(70, 40, 300, 2, torch.bfloat16, 17)
    hidden[11] = float("nan")
    h = hidden.requires_grad_(True)
    r = klay().head_logprobs(h, weight, tokens, bias, complement=True, entropy=True)
    loss = klay().head_distill(h, weight, tokens, torch.zeros(tokens.shape, device="cuda"), bias, rest=False)
    for t in (r.logp, r.neg, r.entropy, loss):
        bad = torch.isnan(t).reshape(70, -1)
        assert bool(bad[11].all()) and int(bad.any(1).sum()) == 1
    dh, = torch.autograd.grad(r.logp.sum() + loss.sum(), h)
    assert bool(torch.isnan(dh[11]).all()) and int(torch.isnan(dh).any(1).sum()) == 1


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("layout", ["columns", "unaligned", "shifted", "across", "weight rows", "weight across", "one row for all"])
def test_layouts(layout, dtype):
    hidden, weight, bias, tokens, g = make(67, 48, 200, 3, dtype, 18)

    def inside(t, pad, skip):
        big = torch.full((t.shape[0], t.shape[1] + pad), 77.0, dtype=t.dtype, device="cuda")
        big[:, skip:skip + t.shape[1]] = t
        return big[:, skip:skip + t.shape[1]]
    h, w = hidden, weight
    if layout == "columns":
        h = inside(hidden, 16, 0)
    elif layout == "unaligned":
        h, w = inside(hidden, 3, 0), inside(weight, 5, 0)
    elif layout == "shifted":
        h, w = inside(hidden, 16, 1), inside(weight, 16, 3)
    elif layout == "across":
        h, tokens = hidden.t().contiguous().t(), tokens.t().contiguous().t()
    elif layout == "weight rows":
        w = inside(weight, 64, 16)
    elif layout == "weight across":
        w = weight.t().contiguous().t()
    else:
        hidden = hidden[:1].expand(67, -1)
        h = hidden
    check_tokens(hidden, weight, bias, tokens, g, given=(h, w))
    check_distill(hidden, weight, bias, tokens, g, given=(h, w), rest=True)


def test_sequences_but_their_last_token():
    """hidden[:, :-1] predicts tokens[:, 1:]: rows at two strides"""
    hidden, weight, bias, _, g = make(5 * 9, 40, 130, 1, torch.bfloat16, 19)
    text = torch.randint(0, 130, (5, 9), generator=g, device="cuda")
    x = hidden.view(5, 9, 40).requires_grad_(True)
    a = klay().head_logprobs(x[:, :-1], weight, text[:, 1:, None], bias, entropy=True)
    plain = hidden.detach().view(5, 9, 40)[:, :-1].reshape(40, 40).clone().requires_grad_(True)
    b = klay().head_logprobs(plain, weight, text[:, 1:].reshape(40, 1), bias, entropy=True)
    assert torch.equal(a.logp.flatten(), b.logp.flatten()) and torch.equal(a.entropy.flatten(), b.entropy)
    da, = torch.autograd.grad(a.logp.sum() + a.entropy.sum(), x)
    db, = torch.autograd.grad(b.logp.sum() + b.entropy.sum(), plain)
    assert torch.equal(da[:, :-1].reshape(40, 40), db) and bool((da[:, -1] == 0).all())


def test_single_vectors_and_no_rows():
    hidden, weight, bias, tokens, g = make(3, 16, 50, 2, torch.float32, 20)
    one = klay().head_logprobs(hidden[1], weight, tokens[1], bias, entropy=True)
    all_ = klay().head_logprobs(hidden, weight, tokens, bias, entropy=True)
    assert one.logp.shape == (2,) and one.entropy.shape == () and torch.equal(one.logp, all_.logp[1])
    ins = [t.detach().requires_grad_(True) for t in (hidden[:0], weight, bias)]
    r = klay().head_logprobs(ins[0], ins[1], tokens[:0], ins[2])
    loss = klay().head_distill(ins[0], ins[1], tokens[:0], torch.zeros((0, 2), device="cuda"), ins[2])
    assert r.logp.shape == (0, 2) and loss.shape == (0,)
    for t in torch.autograd.grad(r.logp.sum() + loss.sum(), ins):
        assert bool((t == 0).all())


@pytest.mark.parametrize("wanted", [(0,), (1,), (2,), (0, 2), (1, 2)])
def test_some_gradients(wanted):
    hidden, weight, bias, tokens, g = make(70, 40, 300, 2, torch.bfloat16, 21)
    full = [t.detach().requires_grad_(True) for t in (hidden, weight, bias)]
    want = torch.autograd.grad(klay().head_logprobs(full[0], full[1], tokens, full[2], entropy=True).logp.sum(), full)
    part = [t.detach().requires_grad_(i in wanted) for i, t in enumerate((hidden, weight, bias))]
    got = torch.autograd.grad(klay().head_logprobs(part[0], part[1], tokens, part[2], entropy=True).logp.sum(), [part[i] for i in wanted])
    for i, t in zip(wanted, got):
        assert torch.equal(t, want[i])


@pytest.mark.parametrize("scale", [2.0 ** -30, 2.0 ** 20])
def test_small_and_large_adjoints_in_half(scale):
    """fp16: the adjoints come into its range and go out of it again"""
    hidden, weight, bias, tokens, g = make(70, 40, 300, 2, torch.float16, 22)
    ins = [hidden.requires_grad_(True), weight.requires_grad_(True)]
    r = klay().head_logprobs(ins[0], ins[1], tokens, bias).logp
    dh, dw = torch.autograd.grad(r, ins, torch.full_like(r, scale))
    base = torch.autograd.grad(klay().head_logprobs(ins[0], ins[1], tokens, bias).logp.sum(), ins)
    for a, b in zip((dh, dw), base):
        want = (b.float() * scale).to(torch.float16)
        assert bool(torch.isfinite(want).all()) or scale > 1
        assert torch.equal(torch.isinf(a), torch.isinf(want))
        fine = torch.isfinite(want)
        assert float((a[fine].double() - b[fine].double() * scale).abs().max()) <= 2.0 ** -11 * float((b[fine].double() * scale).abs().max()) + 2.0 ** -24


def test_the_same_bits_again_and_on_another_stream():
    args = make(300, 136, 5000, 3, torch.bfloat16, 23, "sure")
    hidden, weight, bias, tokens, g = args

    def once():
        ins = [t.detach().requires_grad_(True) for t in (hidden, weight, bias)]
        r = klay().head_logprobs(ins[0], ins[1], tokens, ins[2], complement=True, entropy=True)
        loss = klay().head_distill(ins[0], ins[1], tokens, torch.zeros(tokens.shape, device="cuda"), ins[2])
        return [r.logp, r.neg, r.entropy, loss] + list(torch.autograd.grad([r.logp.sum() + r.neg.sum() + loss.sum(), r.entropy.sum()], ins))
    first = once()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        second = once()
    third = once()
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_graphs(dtype):
    """two captured calls, forward and backward, replayed with other inputs and eager work between"""
    hidden, weight, bias, tokens, g = make(90, 72, 1500, 2, dtype, 24)
    teacher = torch.randn(tokens.shape, generator=g, device="cuda")
    ins = [t.detach().clone().requires_grad_(True) for t in (hidden, weight, bias)]

    def step():
        r = klay().head_logprobs(ins[0], ins[1], tokens, ins[2], entropy=True)
        loss = klay().head_distill(ins[0], ins[1], tokens, teacher, ins[2], rest=False)
        ones = [torch.ones_like(r.logp), torch.ones_like(r.entropy), torch.ones_like(loss)]
        return [r.logp, r.entropy, loss] + list(torch.autograd.grad([r.logp, r.entropy, loss], ins, ones))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for turn in range(4):
        with torch.no_grad():
            ins[0].copy_(torch.randn(hidden.shape, generator=g, device="cuda"))
            tokens.copy_(torch.randint(0, 1500, tokens.shape, generator=g, device="cuda"))
        want = step()
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for a, b in zip(out, want):
                assert torch.equal(a, b), turn


def test_saved_elsewhere():
    """tensors that are saved to host memory and come back at other addresses"""
    hidden, weight, bias, tokens, g = make(40, 24, 100, 2, torch.float32, 25)
    teacher = torch.randn(tokens.shape, generator=g, device="cuda")
    out = []
    for moved in (False, True):
        ins = [t.detach().requires_grad_(True) for t in (hidden, weight, bias)]
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t.cpu() if moved else t, lambda t: t.cuda()):
            total = klay().head_logprobs(ins[0], ins[1], tokens, ins[2], complement=True).neg.sum() + \
                klay().head_distill(ins[0], ins[1], tokens, teacher, ins[2]).sum() + \
                klay().token_distill(ins[0] @ ins[1].t(), tokens, teacher).sum()
        out.append(torch.autograd.grad(total, ins, allow_unused=True))
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_no_logits_in_memory():
    rows, width, vocab = 2048, 64, 60000
    hidden, weight, bias, tokens, g = make(rows, width, vocab, 1, torch.bfloat16, 26)
    h, w = hidden.requires_grad_(True), weight.requires_grad_(True)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    r = klay().head_logprobs(h, w, tokens, bias).logp
    forward = torch.cuda.max_memory_allocated() - before
    torch.autograd.grad(r.sum(), (h, w))
    backward = torch.cuda.max_memory_allocated() - before
    logits = rows * vocab * 2
    assert forward < logits / 8 and backward < 1.2 * logits        # (a piece of 2^25 adjoints, twice: 128 of 246 MB, and the gradients)


def test_from_hidden():
    """a circuit on the answers of a network's last layer: as from the logits of the same layer"""
    from klay_synth import tiny_ddnnf
    k = klay().Circuit(*tiny_ddnnf(3, 12, 30)[0].arrays(), device=0)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    B, G, K, V, D = 9, 4, 3, 50, 24
    tokens = torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(B * G)]).view(B, G, K)
    out = []
    for t in (tokens, tokens[0]):
        for complement in (True, False):
            pair = []
            for straight in (True, False):
                g.manual_seed(6)
                ins = [torch.randn(s, generator=g, device="cuda").requires_grad_(True) for s in ((B, G, D), (V, D), (V,))]
                layer = klay().CircuitLayer(k, klay().KLAY_LOG)
                y = layer.from_hidden(ins[0], ins[1], t, ins[2], complement=complement) if straight else \
                    layer.from_logits(ins[0] @ ins[1].t() + ins[2], t, complement=complement)
                pair.append([y.detach()] + list(torch.autograd.grad(y.sum(), ins)))
            out.append(pair)
    for a, b in out:
        for x, y in zip(a, b):
            # (logits of up to 30, each off by some 24 steps of 2^-24 either way, through a circuit of a few hundred nodes)
            assert float((x - y).abs().max()) <= 2e-4 * max(1.0, float(y.abs().max()))


def test_teacher_and_student():
    """the whole run: a teacher's top tokens with their log probabilities, the student's divergence from them by logits and by hidden states, both
    against 64 bits"""
    hidden, weight, bias, _, g = make(130, 72, 3000, 1, torch.float32, 27)
    x = torch.randn((130, 3000), generator=g, device="cuda") * 3
    told = klay().token_logprobs(x, top=20)
    lp = torch.log_softmax(x.double(), 1)
    assert float((told.top_logp.double() - lp.gather(1, told.top_tokens)).abs().max()) < 1e-5
    for temperature, rest in ((1.0, True), (2.0, False)):
        logits, slip = ref.logits_of(hidden, weight, bias)
        d = torch.rand((130,), generator=g, device="cuda") + 0.1
        want, dx, dx_tol = ref.distill(logits, told.top_tokens, told.top_logp, temperature, rest, slip, d.double())
        ins = [t.detach().requires_grad_(True) for t in (hidden, weight, bias)]
        loss = klay().head_distill(ins[0], ins[1], told.top_tokens, told.top_logp, ins[2], temperature=temperature, rest=rest)
        ref.close(loss, want, what="loss")
        check_gradients(torch.autograd.grad(loss, ins, d), ins, dx, dx_tol, hidden, weight)
        y = logits.float().requires_grad_(True)
        by_logits = klay().token_distill(y, told.top_tokens, told.top_logp, temperature=temperature, rest=rest)
        want, dx, dx_tol = ref.distill(y.detach().double(), told.top_tokens, told.top_logp, temperature, rest, torch.zeros_like(slip), d.double())
        ref.close(by_logits, want, what="loss of logits")
        ref.close(torch.autograd.grad(by_logits, y, d)[0], (dx, dx_tol), what="dlogits")
