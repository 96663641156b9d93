"""What a program asks of the operators between a network and a circuit's leaf weights, as a list of measurable cases.

Three operators: the log probabilities of given tokens under a row of logits (with the weights of the negated literals,
the entropy and the top alternatives), the gated recurrence h_t = a_t (x) h_{t-1} (+) x_t of a semiring over long
sequences, and its single step.  ``own`` false: the plain form, elementary torch operations in 32 bits (64 for
log(1 - p), which 32 lose next to p = 1), rounded once at the end.  ``own`` true: this package's kernels.

Case fields
  op        "tokens", "scan" or "step"
  dtype     type of logits, gates and inputs: "float32", "bfloat16", "float16"
  train     forward and backward
 tokens
  rows, vocab, k     logits [rows, vocab], tokens [rows, k]
  complement, entropy, top    what is asked beside the log probabilities (top: so many alternatives, 0 for none)
  masked    a fifth of the logits are -inf, the first row whole, and one token in six is -1 (nothing asked)
  strided   the logits are the leading columns of a wider array, as the output of a padded head is
 scan, step
  batch, time, channels    gates and inputs [batch, time, channels]; step: [batch, channels]
  semiring  "real", "log" or "max"
  sequences 0: dense; else that many sequences of ragged lengths packed into [time, channels] (batch is 1)
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}


# ---- the cases --------------------------------------------------------------------------------------------------
def _tokens(name, rows, vocab, k, dtype="float32", train=False, complement=False, entropy=False, top=0, masked=False, strided=False):
    return dict(name=name, op="tokens", rows=rows, vocab=vocab, k=k, dtype=dtype, train=train, complement=complement,
                entropy=entropy, top=top, masked=masked, strided=strided)


def _scan(name, batch, time, channels, dtype="float32", semiring="real", train=False, sequences=0):
    return dict(name=name, op="scan", batch=batch, time=time, channels=channels, dtype=dtype, semiring=semiring, train=train,
                sequences=sequences)


def _step(name, batch, channels, dtype="float32", semiring="real"):
    return dict(name=name, op="step", batch=batch, time=1, channels=channels, dtype=dtype, semiring=semiring, train=False, sequences=0)


def listed():
    return [
        # leaf weights of a sum-of-digits circuit: 8 digits of a batch of 256, ten classes each, both literals, a training step
        _tokens("digits_train", 2048, 10, 10, train=True, complement=True),
        # one answer of a large vocabulary while it is generated: its log probability, the entropy, eight alternatives
        _tokens("answer_top8", 1, 131072, 1, "bfloat16", entropy=True, top=8),
        # a served batch, the 20 best alternatives that an interface shows; an odd vocabulary
        _tokens("batch_top20", 64, 50021, 1, "float16", top=20),
        # scoring given texts: log probability and entropy of every token; odd row length
        _tokens("score_4k", 4096, 32771, 1, "bfloat16", entropy=True),
        # training through a constrained head: masked tokens, several literals a row, padding, a padded head's strides
        _tokens("train_masked", 1021, 8191, 5, train=True, complement=True, entropy=True, masked=True, strided=True),
        # the largest: a policy-gradient step over 4096 tokens of a large vocabulary, with an entropy bonus
        _tokens("train_128k", 4096, 131072, 1, "bfloat16", train=True, entropy=True),
        # one generated token of a recurrent network: a single sequence
        _step("step_b1", 1, 2048, "bfloat16"),
        # a large served batch of it
        _step("step_b512", 512, 8192, "float16"),
        # a recurrent layer in training
        _scan("train_4k", 8, 4096, 2048, "bfloat16", train=True),
        # one very long sequence: little beside the time axis to split the work over
        _scan("train_64k", 1, 65536, 512, train=True),
        # log-probabilities of ragged sequences: a chain of gates per literal in the log semiring, trained through
        _scan("packed_log", 1, 30011, 256, semiring="log", train=True, sequences=97),
        # heaviest path through short chains, odd sizes
        _scan("best_path", 3, 777, 33, semiring="max"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: vocabularies of 2 .. 131072, 1 .. 4096 rows; 1 .. 65536 steps, 1 .. 4096 channels, up to 2^26 elements."""
    op = rng.choice(["tokens", "tokens", "scan", "scan", "step"])
    dtype = rng.choice(["float32", "bfloat16", "float16"])
    if op == "tokens":
        vocab = _log_uniform(rng, 2, 131072)
        rows = _log_uniform(rng, 1, min(4096, (1 << 28) // vocab))
        return dict(op=op, rows=rows, vocab=vocab, k=min(vocab, rng.choice([1, 1, 2, 5, 10, 33])), dtype=dtype, train=rng.random() < 0.5,
                    complement=rng.random() < 0.4, entropy=rng.random() < 0.5, top=rng.choice([0, 0, min(vocab, 5), min(vocab, 20), min(vocab, 64)]),
                    masked=rng.random() < 0.3, strided=rng.random() < 0.3)
    semiring = rng.choice(["real", "real", "log", "max"])
    dtype = dtype if semiring == "real" else "float32"
    channels = _log_uniform(rng, 1, 4096)
    if op == "step":
        return dict(op=op, batch=_log_uniform(rng, 1, 1024), time=1, channels=channels, dtype=dtype, semiring=semiring, train=False, sequences=0)
    time = _log_uniform(rng, 1, min(65536, (1 << 25) // channels))
    packed = rng.random() < 0.3
    batch = 1 if packed else _log_uniform(rng, 1, max(1, min(64, (1 << 25) // (channels * time))))
    return dict(op=op, batch=batch, time=time, channels=channels, dtype=dtype, semiring=semiring,
                train=semiring != "max" and rng.random() < 0.6, sequences=_log_uniform(rng, 1, 200) if packed else 0)


# ---- inputs -----------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = getattr(torch, case["dtype"])

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    def whole(high, *shape):
        return torch.randint(0, high, shape, generator=g, device="cuda")

    state = {"case": case}
    if case["op"] == "tokens":
        rows, vocab, k = case["rows"], case["vocab"], case["k"]
        x = torch.empty((rows, vocab + (64 if case["strided"] else 0)), dtype=dtype, device="cuda").normal_(0.0, 2.5, generator=g)
        sure = whole(vocab, rows, 1)                       # the token the network leans to, by nothing .. nearly all of the mass
        x.scatter_add_(1, sure, (25.0 * torch.rand((rows, 1), generator=g, device="cuda")).to(dtype))
        tokens = whole(vocab, rows, k)
        tokens[:, :1] = torch.where(whole(3, rows, 1) > 0, sure, tokens[:, :1])       # most of what is asked for is likely
        if case["k"] == vocab:
            tokens = torch.arange(vocab, device="cuda").expand(rows, vocab).contiguous()
        if case["masked"]:
            x[torch.rand(x.shape, generator=g, device="cuda") < 0.2] = -math.inf
            x[0] = -math.inf
            tokens[whole(6, rows, k) == 0] = -1
        state["logits"] = x[:, :vocab].requires_grad_(case["train"])
        state["tokens"] = tokens
        state["grads"] = [normal(rows, k)] + ([normal(rows, k)] if case["complement"] else []) + ([0.1 * normal(rows)] if case["entropy"] else [])
        return state
    shape = (case["batch"], case["channels"]) if case["op"] == "step" else (case["batch"], case["time"], case["channels"])
    shape = shape[1:] if case["sequences"] else shape
    count = case["sequences"] or case["batch"]
    if case["semiring"] == "real":
        a = torch.sigmoid(normal(*shape) + 3.0)
        x = normal(*shape) * torch.sqrt(1.0 - a * a)
        h = normal(count, case["channels"])
    else:                                                  # the log-probabilities of a chain's literals
        a = torch.nn.functional.logsigmoid(normal(*shape) + 3.0)
        x = torch.nn.functional.logsigmoid(normal(*shape) - 3.0)
        h = torch.nn.functional.logsigmoid(normal(count, case["channels"]))
    train = case["train"]
    state.update(gates=a.to(dtype).requires_grad_(train), inputs=x.to(dtype).requires_grad_(train), initial=h.requires_grad_(train), offsets=None)
    if case["sequences"]:
        # ragged lengths, some of them zero, and a few rows behind the last sequence
        cuts = torch.sort(whole(case["time"] - case["time"] // 100 + 1, case["sequences"]))[0]
        state["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), cuts])
    if case["op"] == "scan" and train:
        state["grads"] = [normal(*shape).to(dtype), normal(count, case["channels"])]
    return state


# ---- one pass ---------------------------------------------------------------------------------------------------
def run(state):
    if own:
        return _run_own(state)
    return {"tokens": _plain_tokens, "scan": _plain_scan, "step": _plain_step}[state["case"]["op"]](state)


def _run_own(state):
    import paper_2410_11415_amd as klay
    case = state["case"]
    if case["op"] == "tokens":
        r = klay.token_logprobs(state["logits"], state["tokens"], complement=case["complement"], entropy=case["entropy"], top=case["top"])
        out = _named(case, r.logp, r.neg, r.entropy, r.top_logp, r.top_tokens)
        if case["train"]:
            asked = [t for t in (r.logp, r.neg, r.entropy) if t is not None]
            out["dlogits"], = torch.autograd.grad(asked, [state["logits"]], state["grads"])
        return out
    semiring = {"real": klay.KLAY_REAL, "log": klay.KLAY_LOG, "max": klay.KLAY_MAXLOG}[case["semiring"]]
    if case["op"] == "step":
        h = klay.gated_step(state["gates"], state["inputs"], state["initial"], semiring)
        return {"h": h, "state": state["initial"]}
    h, last = klay.gated_scan(state["gates"], state["inputs"], state["initial"], semiring, offsets=state["offsets"])
    out = {"h": h, "final": last}
    if case["train"]:
        out["dgates"], out["dinputs"], out["dinitial"] = torch.autograd.grad(
            [h, last], [state["gates"], state["inputs"], state["initial"]], state["grads"])
    return out


def _named(case, logp, neg, entropy, top_logp, top_tokens):
    out = {"logp": logp}
    if case["complement"]:
        out["neg"] = neg
    if case["entropy"]:
        out["entropy"] = entropy
    if case["top"]:
        out["top_logp"], out["top_tokens"] = top_logp, top_tokens
    return out


# ---- the plain form: tokens ---------------------------------------------------------------------------------------
def _plain_tokens(state):
    case, tokens = state["case"], state["tokens"]
    vocab = case["vocab"]
    logits = state["logits"].detach()
    x = logits.to(torch.float64 if case["complement"] else torch.float32)      # log(1 - p) next to p = 1: 64 bits
    m = x.amax(1, keepdim=True)
    empty = m == -math.inf                                                     # nothing is allowed in this row
    d = x - torch.where(empty, 0.0, m)
    e = torch.exp(d)
    s = torch.where(empty, 1.0, e.sum(1, keepdim=True))
    log_s = torch.log(s)
    asked = tokens >= 0
    at = torch.where(asked, tokens, 0)
    lp = torch.gather(d, 1, at) - log_s
    p = torch.exp(lp)
    out_lp = torch.where(asked, lp, 0.0)
    out = {"logp": out_lp.float()}
    if case["complement"]:
        out["neg"] = torch.where(asked, torch.log1p(-p), 0.0).float()
    if case["entropy"]:
        h = torch.where(empty, 0.0, log_s - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / s)
        out["entropy"] = h[:, 0].float()
    if case["top"]:
        # one whole number an element that orders by value, then by the lowest index
        bits = (logits.float() + 0.0).view(torch.int32).to(torch.int64)
        key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * (1 << 20) + (vocab - 1 - torch.arange(vocab, device=x.device))
        best = torch.topk(key, case["top"], dim=1)[0]
        out["top_tokens"] = vocab - 1 - (best & ((1 << 20) - 1))
        out["top_logp"] = (torch.gather(d, 1, out["top_tokens"]) - log_s).float()
    if case["train"]:
        grads = state["grads"]
        q = e / s
        g = torch.where(asked, grads[0].to(x.dtype), 0.0)
        if case["complement"]:
            g = g - torch.where(asked, grads[1].to(x.dtype), 0.0) * p / (1.0 - p)
        dx = -q * g.sum(1, keepdim=True)
        dx.scatter_add_(1, at, g)
        if case["entropy"]:
            lq = torch.where(q > 0, d - log_s, 0.0)
            dx = dx - grads[-1].to(x.dtype)[:, None] * q * (lq + h)
        out["dlogits"] = torch.where(empty, 0.0, dx).to(logits.dtype)
    return out


# ---- the plain form: the recurrence -------------------------------------------------------------------------------
def _real(a, h, x):
    return a * h + x


def _log(a, h, x):
    return torch.logaddexp(a + h, x)


def _max(a, h, x):
    return torch.maximum(a + h, x)


_GATES = {"real": (torch.mul, _real, 0.0), "log": (torch.add, _log, -math.inf), "max": (torch.add, _max, -math.inf)}


def _prefixes(a, x, join, step):
    """h_t = step(a_t, h_{t-1}, x_t) along the last axis but one from h_0 = x_0: pairs of steps as one step, half as many of them."""
    n = x.shape[-2]
    if n == 1:
        return x
    m = n // 2 * 2
    odd = _prefixes(join(a[..., 1:m:2, :], a[..., 0:m:2, :]), step(a[..., 1:m:2, :], x[..., 0:m:2, :], x[..., 1:m:2, :]), join, step)
    h = torch.empty_like(x)
    h[..., 1:m:2, :] = odd
    h[..., :1, :] = x[..., :1, :]
    h[..., 2::2, :] = step(a[..., 2::2, :], odd[..., : (n - 1) // 2, :], x[..., 2::2, :])
    return h


def _plain_scan(state):
    case = state["case"]
    join, step, nothing = _GATES[case["semiring"]]
    a, x, h0 = (state[n].detach().float() for n in ("gates", "inputs", "initial"))
    offsets = state["offsets"]
    dense = offsets is None
    if dense:
        first = torch.zeros(case["time"], dtype=torch.bool, device=a.device)
        first[0] = True
        before, live = h0[:, None, :], None
    else:
        rows = torch.arange(case["time"], device=a.device)
        which = torch.searchsorted(offsets, rows, right=True) - 1
        live = (which < case["sequences"])[:, None]
        which = which.clamp(max=case["sequences"] - 1)
        first = rows == offsets[which]
        before = h0[which]
    first = first[:, None]
    # the first step of a sequence: the state before it enters its input, and no gate reaches further back
    h = _prefixes(torch.where(first, nothing, a), torch.where(first, step(a, before, x), x), join, step)
    prev = torch.where(first, before, torch.roll(h, 1, -2))
    if dense:
        last = h[:, -1, :]
    else:
        none = (offsets[1:] == offsets[:-1])[:, None]
        last = torch.where(none, h0, h[(offsets[1:] - 1).clamp(min=0)])
    dtype = state["inputs"].dtype
    out = {"h": (h if dense else torch.where(live, h, 0.0)).to(dtype), "final": last}
    if not case["train"]:
        return out
    dh, dlast = (t.float() for t in state["grads"])
    if dense:
        end = torch.zeros(case["time"], dtype=torch.bool, device=a.device)
        end[-1] = True
        end, after = end[:, None], dlast[:, None, :]
    else:
        end = (rows == offsets[which + 1] - 1)[:, None]
        after = dlast[which]
    if case["semiring"] == "log":
        w = torch.sigmoid(a + prev - x)
        w = torch.where(torch.isnan(w), 0.0, w)
        v = torch.sigmoid(x - a - prev)
        v = torch.where(torch.isnan(v), 0.0, v)
    else:
        w, v = a, None
    gate = torch.where(end, 0.0, torch.roll(w, -1, -2))
    g = _prefixes(gate.flip(-2), torch.where(end, dh + after, dh).flip(-2), torch.mul, _real).flip(-2)
    da = g * (w if v is not None else prev)
    dx = g * v if v is not None else g
    c = g * w
    if dense:
        dinitial = c[:, 0, :]
    else:
        da, dx = torch.where(live, da, 0.0), torch.where(live, dx, 0.0)
        dinitial = torch.where(none, dlast, c[offsets[:-1].clamp(max=case["time"] - 1)])
    out["dgates"], out["dinputs"], out["dinitial"] = da.to(dtype), dx.to(dtype), dinitial
    return out


def _plain_step(state):
    _, step, _ = _GATES[state["case"]["semiring"]]
    h = step(state["gates"].float(), state["initial"], state["inputs"].float())
    state["initial"].copy_(h)
    return {"h": h.to(state["inputs"].dtype), "state": state["initial"]}


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    s = _BYTES[case["dtype"]]
    if case["op"] == "tokens":
        n, k = case["rows"] * case["vocab"], case["rows"] * case["k"]
        asked = 1 + case["complement"]
        moved = n * s + k * (8 + 4 * asked) + 4 * case["rows"] * case["entropy"] + 12 * case["rows"] * case["top"]
        # an element: difference, exponential, sum; entropy: product and sum
        ops = n * (3 + 2 * case["entropy"])
        if case["train"]:
            moved += n * s + 4 * k * asked + 4 * case["rows"] * case["entropy"]
            ops += n * (3 + 3 * case["entropy"])
        return {"bytes": moved, "flops": ops}
    n = case["batch"] * case["time"] * case["channels"]
    states = 4 * (case["sequences"] or case["batch"]) * case["channels"]
    if case["op"] == "step":
        return {"bytes": 3 * n * s + 2 * states, "flops": n * (2 if case["semiring"] != "log" else 6)}
    ops = n * (2 if case["semiring"] != "log" else 6)
    moved = 3 * n * s + 2 * states + 8 * (case["sequences"] + 1 if case["sequences"] else 0)
    if case["train"]:
        moved += 3 * n * s + 2 * states                    # the adjoint of h in, those of gates and inputs out
        ops += n * (3 if case["semiring"] != "log" else 8)
    return {"bytes": moved, "flops": ops}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    return {"tokens": _exact_tokens, "scan": _exact_scan, "step": _exact_scan}[case["op"]](case, state)


def _exact_tokens(case, state):
    """Row by row (blocks of them): probabilities of the allowed tokens, everything else from them."""
    rows, k = case["rows"], case["k"]
    parts = []
    block = max(1, (1 << 26) // case["vocab"])
    for b in range(0, rows, block):
        x = state["logits"].detach()[b:b + block].double()
        t = state["tokens"][b:b + block]
        lse = torch.logsumexp(x, 1, keepdim=True)
        some = lse > -math.inf
        lp = torch.where(some, x - lse, -math.inf)
        p = lp.exp()
        ask = t >= 0
        i = t.clamp(min=0)
        r = {"logp": torch.where(ask, lp.gather(1, i), 0.0)}
        # the mass of all other tokens, summed without the asked one
        rest = torch.stack([p.scatter(1, i[:, j:j + 1], 0.0).sum(1) for j in range(k)], 1) if case["complement"] else None
        rest = torch.where(some, rest, 1.0) if rest is not None else None
        if case["complement"]:
            r["neg"] = torch.where(ask, rest.log(), 0.0)
        plogp = torch.where(p > 0, p * lp, 0.0)
        h = -plogp.sum(1)
        if case["entropy"]:
            r["entropy"] = h
        if case["top"]:
            order = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :case["top"]]
            r["top_logp"], r["top_tokens"] = lp.gather(1, order), order
        if case["train"]:
            grads = [q[b:b + block].double() for q in state["grads"]]
            dx = torch.zeros_like(x)
            pk = p.gather(1, i)
            for j in range(k):
                own_p, on = pk[:, j:j + 1], ask[:, j:j + 1]
                one = torch.zeros_like(x).scatter(1, i[:, j:j + 1], 1.0)
                dx += torch.where(on, grads[0][:, j:j + 1] * (one - p), 0.0)
                if case["complement"]:
                    others = torch.where(one > 0, 0.0, p) / rest[:, j:j + 1]        # the distribution without the asked token
                    dx += torch.where(on, grads[1][:, j:j + 1] * own_p * (others - one), 0.0)
            if case["entropy"]:
                dx -= grads[-1][:, None] * (plogp + p * h[:, None])
            r["dlogits"] = torch.where(some, dx, 0.0)
        parts.append(r)
    return {n: torch.cat([r[n] for r in parts]) for n in parts[0]}


def _exact_scan(case, state):
    """Step by step, in numpy."""
    a, x, h0 = (state[n].detach().cpu().double().numpy() for n in ("gates", "inputs", "initial"))
    semiring = case["semiring"]

    def step(a, h, x):
        if semiring == "real":
            return a * h + x
        return np.logaddexp(a + h, x) if semiring == "log" else np.maximum(a + h, x)

    if case["op"] == "step":
        h = step(a, h0, x)
        return {"h": torch.from_numpy(h), "state": torch.from_numpy(h)}
    if case["sequences"]:
        o = state["offsets"].cpu().numpy()
        spans = [(slice(int(o[s]), int(o[s + 1])), s) for s in range(case["sequences"])]
    else:
        a, x = a.swapaxes(0, 1).copy(), x.swapaxes(0, 1).copy()       # time first
        spans = [(slice(0, case["time"]), slice(None))]
    h, last = np.zeros_like(x), h0.copy()
    for span, s in spans:
        now = h0[s]
        for t in range(span.start, span.stop):
            h[t] = now = step(a[t], now, x[t])
        last[s] = now
    out = {"h": h, "final": last}
    if case["train"]:
        dh, dlast = (g.cpu().double().numpy() for g in state["grads"])
        dh = dh if case["sequences"] else dh.swapaxes(0, 1).copy()
        da, dx, dinitial = np.zeros_like(x), np.zeros_like(x), dlast.copy()
        for span, s in spans:
            c = dlast[s]
            for t in range(span.stop - 1, span.start - 1, -1):
                g = dh[t] + c
                prev = h[t - 1] if t > span.start else h0[s]
                if semiring == "real":
                    da[t], dx[t], c = g * prev, g, g * a[t]
                else:
                    c = da[t] = g * np.exp(a[t] + prev - h[t])
                    dx[t] = g * np.exp(x[t] - h[t])
            dinitial[s] = c
        out.update(dgates=da, dinputs=dx, dinitial=dinitial)
    out = {n: torch.from_numpy(v) for n, v in out.items()}
    if not case["sequences"]:
        out = {n: v.transpose(0, 1) if n in ("h", "dgates", "dinputs") else v for n, v in out.items()}
    return out
