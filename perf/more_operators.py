"""What the speed of the losses that a masked model is retrained with is measured on: single calls as a program makes them that scores
or retrains a model, from the final hidden states of its tokens to the losses and their gradients.

h (tokens, width) are hidden states, the head W (vocab, width) makes logits z = h W^T of them.  A case is a dict of plain values:
  op "entropy"   softmax cross entropy against the next token: loss = lse(z) - z[target]; targets outside the vocabulary leave
                 their tokens out (loss, lse and gradients 0)
  op "distill"   divergence from a teacher's top logits, k of them for each token, with a temperature: q = softmax(u / temperature)
                 over the entries whose id is in the vocabulary, loss = sum q (log q - z[id] / temperature + lse(z / temperature))
  tokens, vocab, width, dtype (h, W and their gradients); left_out: share of the tokens that is left out; dh, dweight: whether the
  gradients of h and of W are wanted, for a gradient of each token's loss that is one over the tokens that count; lse: whether the
  logarithm of the sum of exponentials is wanted too
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LEFT_OUT = -100


def _entropy(name, tokens, vocab, width, dtype="bf16", left_out=0.0, dh=False, dweight=False, lse=False):
    return {"name": name, "op": "entropy", "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype, "left_out": left_out,
            "dh": dh, "dweight": dweight, "lse": lse, "k": 1, "temperature": 1.0}


def _distill(name, tokens, vocab, width, k, dtype="bf16", left_out=0.0, dh=False, dweight=False, lse=False, temperature=1.0):
    return {**_entropy(name, tokens, vocab, width, dtype, left_out, dh, dweight, lse), "op": "distill", "k": k, "temperature": temperature}


def listed():
    return [
        # how likely one token is under a small model: the smallest call, where latency counts
        _entropy("score_1x8192x512", 1, 8192, 512),
        # the same with a large vocabulary, a token of a sequence that is being answered: all of the head for one row
        _entropy("score_1x128256x4096", 1, 128256, 4096, lse=True),
        # the last tokens of a batch of candidate answers
        _entropy("score_48x32000x4096", 48, 32000, 4096, lse=True),
        # a training step of a small model on an odd number of tokens, prompts left out, an odd vocabulary
        _entropy("train_2047x50257x1024", 2047, 50257, 1024, left_out=0.3, dh=True, dweight=True),
        # single precision, odd in every size
        _entropy("train_1000x5003x769_f32", 1000, 5003, 769, dtype="f32", left_out=0.1, dh=True, dweight=True),
        # masked layers retrained under a head that is kept as it is
        _entropy("frozen_4096x128256x4096", 4096, 128256, 4096, dh=True),
        # a training step with the head: the largest call
        _entropy("train_8192x128256x4096", 8192, 128256, 4096, left_out=0.05, dh=True, dweight=True),
        # one token against its teacher
        _distill("distill_1x32000x2048_k8", 1, 32000, 2048, 8, lse=True),
        # a small step of a masked layer's recovery: the head is kept
        _distill("distill_512x32000x4096_k32", 512, 32000, 4096, 32, dh=True),
        # a step with the head, softened by a temperature, padding left out
        _distill("distill_3001x50257x2048_k64", 3001, 50257, 2048, 64, left_out=0.1, dh=True, dweight=True, temperature=2.0),
        # single precision, odd sizes
        _distill("distill_700x4099x1000_k17_f32", 700, 4099, 1000, 17, dtype="f32", dh=True, dweight=True, temperature=1.5),
        # a large step against many of the teacher's logits
        _distill("distill_4096x128256x4096_k128", 4096, 128256, 4096, 128, dh=True),
    ]


def _size(rng, low, high):
    """A whole number from 2^low to 2^high, spread over its logarithm; half of them multiples of 64."""
    n = max(1, int(2.0 ** rng.uniform(low, high)))
    return n if n < 128 or rng.random() < 0.5 else n // 64 * 64


def draw(rng):
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    width, vocab = _size(rng, 6, 13), _size(rng, 8, 17)
    tokens = max(1, min(_size(rng, 0, 13), (1 << (41 if dtype == "bf16" else 37)) // (vocab * width)))
    dh, dweight = rng.choice(((False, False), (True, False), (True, True), (True, True)))
    more = {"dtype": dtype, "left_out": rng.choice((0.0, 0.0, rng.uniform(0.0, 0.7))), "dh": dh, "dweight": dweight, "lse": rng.random() < 0.5}
    if rng.random() < 0.5:
        c = _entropy("", tokens, vocab, width, **more)
    else:
        c = _distill("", tokens, vocab, width, min(_size(rng, 0, 7), vocab), temperature=rng.choice((1.0, 1.0, rng.uniform(0.5, 4.0))), **more)
    del c["name"]
    return c


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _active(case):
    """Tokens that count, at least one."""
    return max(1, case["tokens"] - int(case["tokens"] * case["left_out"]))


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens, vocab, width, k, dtype = case["tokens"], case["vocab"], case["width"], case["k"], TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    s = {"case": case}
    # logits of a spread of 2.5, as a trained head makes them of normed states
    s["weight"] = normal(vocab, width).mul_(2.5 / width ** 0.5).to(dtype)
    h = normal(tokens, width)
    out = torch.randperm(tokens, device="cuda", generator=gen)[_active(case):]
    if case["op"] == "entropy":
        # small numbers are frequent tokens
        ids = torch.pow(float(vocab), uniform(tokens)).sub_(1.0).long().clamp_(0, vocab - 1)
        s["targets"] = ids.clone()
        s["targets"][out] = LEFT_OUT
        ids = ids[:, None]
    else:
        # k tokens a step apart (all different), the teacher's logits falling from the first to the last
        begin = torch.pow(float(vocab), uniform(tokens, 1)).sub_(1.0).long()
        step = 1 + (uniform(tokens, 1) * (vocab // k - 1)).long()
        s["ids"] = (begin + step * torch.arange(k, device="cuda")) % vocab
        s["logits"] = 12.0 - torch.cumsum(torch.empty(tokens, k, device="cuda").exponential_(3.0, generator=gen), 1)
        ids = s["ids"][:, :4].clone()
        s["ids"][out] = -1
    # the model has learned something: the first of these tokens are more likely than others
    for j in range(ids.shape[1]):
        h += s["weight"][ids[:, j]].float() * (2.0 / (j + 1)) * uniform(tokens, 1)
    s["h"] = h.to(dtype)
    s["dloss"] = torch.full((tokens,), 1.0 / _active(case), device="cuda") if case["dh"] or case["dweight"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _plan(s)
    return s


def _plan(s):
    """The outputs, the workspace and the description of the call, which a program keeps from step to step."""
    from paper_2505_23949_amd import loss

    case = s["case"]
    s["out"] = {"loss": torch.empty(case["tokens"], device="cuda")}
    if case["lse"]:
        s["out"]["lse"] = torch.empty(case["tokens"], device="cuda")
    if case["dh"]:
        s["out"]["dh"] = torch.empty_like(s["h"])
    if case["dweight"]:
        s["out"]["dweight"] = torch.empty_like(s["weight"])
    if case["op"] == "entropy":
        s["problem"] = loss.make_cross_entropy(s["h"], s["weight"], s["targets"], dloss=s["dloss"], **s["out"])
        size = loss.tsenor_cross_entropy_workspace_bytes(s["problem"])
    else:
        s["problem"] = loss.make_distill(s["h"], s["weight"], s["ids"], s["logits"], temperature=case["temperature"], dloss=s["dloss"], **s["out"])
        size = loss.tsenor_distill_workspace_bytes(s["problem"])
    s["work"] = torch.empty(size, dtype=torch.uint8, device="cuda")


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2505_23949_amd import loss

    if s["case"]["op"] == "entropy":
        loss.tsenor_cross_entropy(s["problem"], s["work"])
    else:
        loss.tsenor_distill(s["problem"], s["work"])
    return s["out"]


# ---- the operators in plain torch, 32 bits -------------------------------------------------------------------------------

def _run_plain(s):
    case, dtype = s["case"], s["h"].dtype
    h, weight = s["h"].float(), s["weight"].float()
    z = (h @ weight.t()) / case["temperature"]
    largest = z.amax(1, keepdim=True)
    lse = (z - largest).exp().sum(1).log() + largest[:, 0]
    if case["op"] == "entropy":
        ids = s["targets"][:, None]
        counts = (ids >= 0) & (ids < case["vocab"])
        q = counts.float()
        ids = torch.where(counts, ids, 0)
        loss = lse - z.gather(1, ids)[:, 0]
    else:
        counts = (s["ids"] >= 0) & (s["ids"] < case["vocab"])
        ids = torch.where(counts, s["ids"], 0)
        u = torch.where(counts, s["logits"] / case["temperature"], -math.inf)
        top = u.amax(1, keepdim=True)
        e = torch.where(counts, (u - top).exp(), 0.0)
        total = e.sum(1, keepdim=True)
        q = torch.where(counts, e / total, 0.0)
        log_q = torch.where(counts, u - top - total.log(), 0.0)
        loss = (q * (log_q - z.gather(1, ids) + lse[:, None])).sum(1)
    counts = counts.any(1)
    out = {"loss": torch.where(counts, loss, 0.0)}
    if case["lse"]:
        out["lse"] = torch.where(counts, lse, 0.0)
    if s["dloss"] is not None:
        g = (z - lse[:, None]).exp().scatter_add_(1, ids, -q)
        g = torch.where(counts[:, None], g * (s["dloss"] / case["temperature"])[:, None], 0.0)
        if case["dh"]:
            out["dh"] = (g @ weight).to(dtype)
        if case["dweight"]:
            out["dweight"] = (g.t() @ h).to(dtype)
    return out


# ---- bytes and operations ------------------------------------------------------------------------------------------------

def work(case):
    """Of the tokens that count: the others need no product."""
    b, tokens, vocab, width = 4 if case["dtype"] == "f32" else 2, _active(case), case["vocab"], case["width"]
    nbytes = b * (tokens + vocab) * width + case["tokens"] * (8 if case["op"] == "entropy" else 12 * case["k"])
    nbytes += case["tokens"] * 4 * (1 + case["lse"] + (case["dh"] or case["dweight"]))
    nbytes += b * width * (case["tokens"] * case["dh"] + vocab * case["dweight"])
    return {"bytes": nbytes, "flops": 2 * tokens * vocab * width * (1 + case["dh"] + case["dweight"])}


# ---- the definitions, 64 bits ---------------------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    weight, tokens, vocab, width = s["weight"].double(), case["tokens"], case["vocab"], case["width"]
    loss = torch.zeros(tokens, dtype=torch.float64, device="cuda")
    lse, dh = torch.zeros_like(loss), torch.zeros(tokens, width, dtype=torch.float64, device="cuda")
    dweight = torch.zeros(vocab if case["dweight"] else 0, width, dtype=torch.float64, device="cuda")
    for t0 in range(0, tokens, 1024):
        rows = slice(t0, t0 + 1024)
        if case["op"] == "entropy":
            y = s["targets"][rows]
            kept = torch.nonzero(y != LEFT_OUT)[:, 0]
            ids, q = y[kept, None], torch.ones(len(kept), 1, dtype=torch.float64, device="cuda")
        else:
            kept = torch.nonzero(s["ids"][rows, 0] >= 0)[:, 0]
            ids = s["ids"][rows][kept]
            q = torch.softmax(s["logits"][rows][kept].double() / case["temperature"], 1)
        if not len(kept):
            continue
        h = s["h"][rows][kept].double()
        log_p = torch.matmul(h, weight.t()).div_(case["temperature"])
        at = kept + t0
        lse[at] = torch.logsumexp(log_p, 1)
        log_p -= lse[at][:, None]
        loss[at] = torch.special.xlogy(q, q).sum(1) - (q * torch.gather(log_p, 1, ids)).sum(1)
        if s["dloss"] is None:
            continue
        g = log_p.exp_()
        g[torch.arange(len(kept), device="cuda")[:, None], ids] -= q
        g *= s["dloss"][at].double()[:, None] / case["temperature"]
        if case["dh"]:
            dh[at] = g @ weight
        if case["dweight"]:
            dweight += g.t() @ h
    out = {"loss": loss}
    if case["lse"]:
        out["lse"] = lse
    if case["dh"]:
        out["dh"] = dh
    if case["dweight"]:
        out["dweight"] = dweight
    return out
