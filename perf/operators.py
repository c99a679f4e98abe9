"""The operators at the two ends of a training step around the Monarch layers, as timed cases.

A case is one of four uses (``use``):

* ``score``  the loss of given tokens over a vocabulary, no gradient (evaluation; one token: serving)
* ``train``  the loss and its gradients with respect to the last hidden state and the vocabulary's weights
* ``ortho``  a stack of blocks orthogonalised by Newton-Schulz products
* ``muon``   the optimiser's step on a list of factors: momentum, orthogonalisation, decay, update in place

Sizes: ``rows`` tokens, ``vocab``, ``width``; ``blocks`` blocks of ``m x n`` (a Monarch factor), ``count`` such factors of one shape.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_COEFFICIENTS = (3.4445, -4.7750, 2.0315)
_STEPS = 5
_EPS = 1e-7
_LR, _MOMENTUM, _DECAY = 0.02, 0.95, 0.01
_IGNORE = -100


def _loss(use, dtype, rows, vocab, width, ignored=0.0, reduction="mean"):
    return dict(use=use, dtype=dtype, rows=rows, vocab=vocab, width=width, ignored=ignored, reduction=reduction)


def _blocks(use, dtype, blocks, m, n, count=1):
    return dict(use=use, dtype=dtype, blocks=blocks, m=m, n=n, count=count)


def listed():
    return [
        # serving GPT-2 small: how likely one given token is (bound by reading the vocabulary's weights)
        dict(_loss("score", "bf16", 1, 50257, 768), name="score_1tok"),
        # the same with fp32 weights of GPT-2 medium, a few candidates at once
        dict(_loss("score", "f32", 24, 50257, 1024), name="score_24tok_f32"),
        # evaluation of GPT-2 medium: one full context
        dict(_loss("score", "bf16", 1024, 50257, 1024), name="score_1024tok"),
        # training, a small odd vocabulary and width, weights of its own for each row, a third of the rows masked (prompts)
        dict(_loss("train", "bf16", 777, 8191, 330, 0.34, "none"), name="train_odd"),
        # training GPT-2 small in fp32: two contexts
        dict(_loss("train", "f32", 2048, 50257, 768), name="train_gpt2s_f32"),
        # training GPT-2 small: eight contexts, the tails of sequences masked
        dict(_loss("train", "bf16", 8192, 50257, 768, 0.1), name="train_gpt2s"),
        # training GPT-2 medium: sixteen contexts
        dict(_loss("train", "bf16", 16384, 50257, 1024), name="train_gpt2m"),
        # the factor of the smallest square transform: launches and latency
        dict(_blocks("ortho", "f32", 16, 16, 16), name="ortho_16x16"),
        # a factor of the square transform at n = 4096
        dict(_blocks("ortho", "bf16", 64, 64, 64), name="ortho_64x64"),
        # blocks that are multiples of nothing, wider than high
        dict(_blocks("ortho", "f32", 8, 150, 333), name="ortho_odd"),
        # one step on the first factors of the four layers of a GPT-2 small block, fp32 weights
        dict(_blocks("muon", "f32", 4, 192, 192, 4), name="muon_gpt2s"),
        # one step on the wide factors of the feed-forward layers of GPT-2 medium, bf16 weights with fp32 masters
        dict(_blocks("muon", "bf16", 4, 1024, 256, 12), name="muon_gpt2m"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    use = rng.choice(["score", "train", "ortho", "muon"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if use in ("score", "train"):
        rows = _log_uniform(rng, 1, 4096 if use == "score" else 6000)
        vocab = _log_uniform(rng, 500, 60000)
        width = _log_uniform(rng, 16, 1280)
        if rng.random() < 0.5:  # widths of layers are mostly multiples of something
            width = max(64, width // 64 * 64)
        if use == "score":
            return _loss(use, dtype, rows, vocab, width, rng.choice([0.0, 0.0, 0.25]))
        return _loss(use, dtype, rows, vocab, width, rng.choice([0.0, 0.05, 0.5]), rng.choice(["mean", "sum", "none"]))
    m, n = _log_uniform(rng, 8, 1024), _log_uniform(rng, 8, 1024)
    if rng.random() < 0.5:
        m, n = max(16, m // 16 * 16), max(16, n // 16 * 16)
    most = max(1, (12 << 20) // (m * n))
    blocks = min(most, _log_uniform(rng, 1, 64))
    if use == "ortho":
        return _blocks(use, dtype, blocks, m, n)
    return _blocks(use, dtype, blocks, m, n, max(1, min(12, most // blocks, _log_uniform(rng, 1, 12))))


def _kept(case):
    """How many rows have a target."""
    return case["rows"] - int(case["rows"] * case["ignored"])


def _gradient(gen, blocks, m, n, dtype):
    """What a weight's gradient looks like: noise and a few directions that stand out of it."""
    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    rank = 4
    strong = normal(blocks, m, rank) @ normal(blocks, rank, n)
    return ((normal(blocks, m, n) + 0.5 * strong) * 1e-3).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dtype = _DTYPES[case["dtype"]]
    state = dict(case)
    if case["use"] in ("score", "train"):
        rows, vocab, width = case["rows"], case["vocab"], case["width"]
        # the last hidden state is normalised; the weights give logits of standard deviation 2
        state["x"] = torch.randn((rows, width), generator=gen, device="cuda").to(dtype)
        state["weight"] = (torch.randn((vocab, width), generator=gen, device="cuda") * (2.0 / math.sqrt(width))).to(dtype)
        # a few tokens are common, most are rare
        target = (torch.rand((rows,), generator=gen, device="cuda").pow(3) * vocab).long().clamp_(max=vocab - 1)
        target[torch.randperm(rows, generator=gen, device="cuda")[_kept(case):]] = _IGNORE
        state["target"] = target
        if case["use"] == "train":
            state["x"].requires_grad_()
            state["weight"].requires_grad_()
            none = case["reduction"] == "none"
            state["dloss"] = torch.rand((rows,), generator=gen, device="cuda") / rows if none else torch.ones((), device="cuda")
        return state
    blocks, m, n, count = case["blocks"], case["m"], case["n"], case["count"]
    state["grads"] = [_gradient(gen, blocks, m, n, dtype) for _ in range(count)]
    if case["use"] == "muon":
        def weight():
            return torch.randn((blocks, m, n), generator=gen, device="cuda") / math.sqrt(n)
        kept = [weight() for _ in range(count)]
        state["momenta"] = [_gradient(gen, blocks, m, n, torch.float32) * 5 for _ in range(count)]
        state["weights"] = [w.to(dtype) for w in kept]
        state["masters"] = kept if case["dtype"] == "bf16" else None
    return state


# ---- the framework's calls ----

def _run_own(state):
    from paper_2204_00595_amd import autograd, binding

    use = state["use"]
    if use == "score":
        loss, lse = binding.monarch_xent_fwd(state["x"], state["weight"], state["target"], ignore_index=_IGNORE)
        return {"loss": loss, "lse": lse}
    if use == "train":
        loss = autograd.vocab_cross_entropy(state["x"], state["weight"], state["target"], ignore_index=_IGNORE,
                                            reduction=state["reduction"])
        dx, dweight = torch.autograd.grad(loss, (state["x"], state["weight"]), state["dloss"])
        return {"loss": loss.detach(), "dx": dx, "dweight": dweight}
    if use == "ortho":
        return binding.monarch_orthogonalize(state["grads"][0], steps=_STEPS, coefficients=_COEFFICIENTS, eps=_EPS)
    binding.monarch_muon_step(state["weights"], state["grads"], state["momenta"], lr=_LR, momentum=_MOMENTUM,
                              weight_decay=_DECAY, nesterov=True, steps=_STEPS, coefficients=_COEFFICIENTS, eps=_EPS,
                              masters=state["masters"])
    return {k: state[k] for k in ("weights", "momenta", "masters")}


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end ----

def _plain_loss(x, weight, target):
    """(loss of each row, its log sum, the softmax's numerators and their sum, the rows that count, their targets)"""
    logits = x @ weight.t()
    top = logits.amax(dim=1, keepdim=True)
    picked = torch.where(target == _IGNORE, 0, target)
    counts = target != _IGNORE
    hit = logits.gather(1, picked[:, None])[:, 0]
    logits = (logits - top).exp_()
    total = logits.sum(dim=1)
    lse = top[:, 0] + total.log()
    return torch.where(counts, lse - hit, 0.0), lse, logits, total, counts, picked


def _plain_train(state):
    with torch.no_grad():
        x, weight = state["x"].float(), state["weight"].float()
        loss, _, e, total, counts, picked = _plain_loss(x, weight, state["target"])
        upstream = state["dloss"] * torch.ones_like(loss)
        if state["reduction"] == "mean":
            number = counts.sum().clamp(min=1)
            loss, upstream = loss.sum() / number, upstream / number
        elif state["reduction"] == "sum":
            loss = loss.sum()
        upstream = torch.where(counts, upstream, 0.0)
        e.mul_((upstream / total)[:, None])
        e[torch.arange(len(picked), device=e.device), picked] -= upstream
        dx, dweight = e @ weight, e.t() @ x
        return {"loss": loss, "dx": dx.to(state["x"].dtype), "dweight": dweight.to(state["weight"].dtype)}


def _newton_schulz(g):
    x = g / (g.square().sum(dim=(1, 2), keepdim=True).sqrt() + _EPS)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    a, b, c = _COEFFICIENTS
    for _ in range(_STEPS):
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return x.transpose(1, 2).contiguous() if tall else x


def _muon_scale(m, n):
    return math.sqrt(max(1.0, m / n))


def _run_plain(state):
    use = state["use"]
    if use == "score":
        loss, lse = _plain_loss(state["x"].float(), state["weight"].float(), state["target"])[:2]
        return {"loss": loss, "lse": lse}
    if use == "train":
        return _plain_train(state)
    if use == "ortho":
        g = state["grads"][0]
        return _newton_schulz(g.float()).to(g.dtype)
    grads, momenta, weights = state["grads"], state["momenta"], state["weights"]
    masters = weights if state["masters"] is None else state["masters"]
    g = torch.cat([t.float() for t in grads])
    v = torch.cat(momenta) * _MOMENTUM + g
    update = _newton_schulz(g + _MOMENTUM * v) * (_LR * _muon_scale(state["m"], state["n"]))
    new = torch.cat(masters) * (1 - _LR * _DECAY) - update
    torch._foreach_copy_(momenta, v.split(state["blocks"]))
    torch._foreach_copy_(masters, new.split(state["blocks"]))
    if state["masters"] is not None:
        torch._foreach_copy_(weights, masters)
    return {k: state[k] for k in ("weights", "momenta", "masters")}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the same in 64 bits, from the definitions ----

def _exact_rows(x, weight, target, upstream):
    """Loss, log sum and, where `upstream` is given, the gradients, a slice of the rows at a time."""
    losses, sums, dx, dweight = [], [], [], torch.zeros_like(weight) if upstream is not None else None
    for at in range(0, x.shape[0], 1024):
        part, t = x[at:at + 1024], target[at:at + 1024]
        valid = t != _IGNORE
        t = torch.where(valid, t, torch.zeros_like(t))
        logits = torch.mm(part, weight.t().contiguous())
        lse = torch.logsumexp(logits, dim=1)
        losses.append((lse - logits.gather(1, t[:, None]).squeeze(1)) * valid)
        sums.append(lse)
        if upstream is not None:
            g = torch.exp(logits - lse[:, None])
            g.scatter_add_(1, t[:, None], torch.full_like(g[:, :1], -1.0))
            g *= (upstream[at:at + 1024] * valid)[:, None]
            dx.append(torch.mm(g, weight))
            dweight += torch.mm(g.t().contiguous(), part)
    return torch.cat(losses), torch.cat(sums), torch.cat(dx) if dx else None, dweight


def _exact_orthogonal(g):
    """Newton-Schulz steps block by block, on the shorter side."""
    out = []
    a, b, c = _COEFFICIENTS
    for block in g:
        block = block / (torch.linalg.matrix_norm(block) + _EPS)
        wide = block if block.shape[0] <= block.shape[1] else block.t()
        for _ in range(_STEPS):
            gram = wide.mm(wide.t().contiguous())
            wide = a * wide + b * gram.mm(wide) + c * gram.mm(gram.mm(wide))
        out.append(wide if block.shape[0] <= block.shape[1] else wide.t())
    return torch.stack(out)


def exact(case, seed):
    state = prepare(case, seed)
    use = case["use"]
    if use in ("score", "train"):
        x, weight, target = state["x"].detach().double(), state["weight"].detach().double(), state["target"]
        if use == "score":
            loss, lse, _, _ = _exact_rows(x, weight, target, None)
            return {"loss": loss, "lse": lse}
        share = 1.0 / max(1, _kept(case)) if case["reduction"] == "mean" else 1.0
        upstream = state["dloss"].double() * share * torch.ones(case["rows"], dtype=torch.float64, device="cuda")
        loss, _, dx, dweight = _exact_rows(x, weight, target, upstream)
        return {"loss": loss if case["reduction"] == "none" else loss.sum() * share, "dx": dx, "dweight": dweight}
    grads = [g.double() for g in state["grads"]]
    if use == "ortho":
        return _exact_orthogonal(grads[0])
    momenta = [_MOMENTUM * v.double() + g for v, g in zip(state["momenta"], grads)]
    kept = state["weights"] if state["masters"] is None else state["masters"]
    size = _LR * _muon_scale(case["m"], case["n"])
    new = [(1 - _LR * _DECAY) * w.double() - size * _exact_orthogonal(g + _MOMENTUM * v)
           for w, g, v in zip(kept, grads, momenta)]
    return {"weights": new, "momenta": momenta, "masters": None if state["masters"] is None else new}


def work(case):
    """What a pass cannot do without: inputs read and outputs written once, products of the rows that count."""
    size = {"bf16": 2, "f32": 4}[case["dtype"]]
    if case["use"] in ("score", "train"):
        rows, vocab, width = case["rows"], case["vocab"], case["width"]
        tensors = (rows + vocab) * width * size
        train = case["use"] == "train"
        return {"bytes": tensors * (2 if train else 1) + rows * (12 if train else 16),
                "flops": 2.0 * (_kept(case) if train else rows) * vocab * width * (3 if train else 1)}
    blocks, m, n = case["blocks"] * case["count"], case["m"], case["n"]
    r, c = min(m, n), max(m, n)
    flops = blocks * _STEPS * (3.0 * r * r * c + r ** 3)  # the two symmetric products by halves
    if case["use"] == "ortho":
        return {"bytes": blocks * m * n * 2 * size, "flops": flops}
    each = size + 8 + 8 + (2 if case["dtype"] == "bf16" else 0)  # gradient; momentum and weight, read and written; the bf16 copy
    return {"bytes": blocks * m * n * each, "flops": flops}
