"""Cross entropies of words that a model has learned (from 1e-6 to 0.1), and their gradients: right to a share of themselves, whichever
kernels make them.

loss = log(1 + y), y = sum_{j != target} exp(z_j - z_target), so that an error of y is one of the loss, of at most the same share; dz of the
target is -y / (1 + y), of another word exp(z_j - z_target) / (1 + y)."""
import math

import pytest
import torch

from test_gpu_loss import DTYPES, HALF_STEP, U, Case, loss  # noqa: F401  (loss: a fixture)

pytestmark = pytest.mark.gpu


def learned(tokens, vocab, width, dtype, whole, seed=0):
    """Hidden states along the rows of their targets.  `whole`: all products and their sums are exact in single precision in any order
    (rows of 1/2 and 1, states that are multiples of them by small numbers over a power of two)."""
    case = Case(tokens, vocab, width, dtype, dloss=False, seed=seed)
    gen = torch.Generator().manual_seed(seed + 17 * tokens + vocab)
    rows = torch.tensor([-1.0, -0.5, 0.5, 1.0])[torch.randint(0, 4, (vocab, width), generator=gen)] if whole else torch.randn(vocab, width, generator=gen) * 0.79
    case.weight = rows.to(DTYPES[dtype])
    # z of the target is about 5/8 of this, of the others 0 with a spread of that over the root of the width
    more = 2.0 + 200.0 / width + 10.0 * torch.rand(tokens, generator=gen).double()
    scale = 1.6 * (math.log(vocab) + more)
    if whole:
        scale = torch.floor(scale)
    case.h = (case.weight[case.targets].double() * (scale / width)[:, None]).to(DTYPES[dtype])
    return case


def expect(case, whole):
    """Values in 64 bits, and how far off they may be."""
    h, w, t = case.h.double(), case.weight.double(), case.targets[:, None]
    z = h @ w.t()
    own = z.gather(1, t)
    rest = (z - own).exp().scatter_(1, t, 0.0)                  # exp(z_j - z_target), none for the target
    y = rest.sum(1, keepdim=True)
    case.want = {"loss": torch.log1p(y)[:, 0], "lse": (own + torch.log1p(y))[:, 0]}
    # of y: the arguments of its exponentials (their products by log2 e, rounded twice, and once more where 15 is added to them, at up to 16), the
    # exponentials (2 last places), sums of at most 64 + 16 + vocab / 64 terms behind each other, division and logarithm; and the logits, which are
    # sums of `width` products
    share = (2 * (z.amax(1) - z.amin(1)) + 16 + 4 + 80 + case.vocab / 64 + 8) * U
    dz = torch.zeros(case.tokens, dtype=torch.float64) if whole else 2 * ((case.width + 2) * U * (h.abs() @ w.abs().t()).amax(1))
    share = 1.01 * (share + dz)
    case.off = {"loss": share * case.want["loss"], "lse": share * case.want["loss"] + dz + 8 * U * own[:, 0].abs()}
    weight = (torch.ones(case.tokens, dtype=torch.float64) if case.dloss is None else case.dloss.double())[:, None]
    g = weight * rest.scatter(1, t, -y) / (1 + y)
    case.want["dh"], case.want["dweight"] = g @ w, g.t() @ h
    # gradients of logits: the same share (twice: of the word's own and of the sum) and a few last places; bf16: fp16's 2^-11 and steps of 2^-39 of the
    # largest, then bf16's 2^-8
    off = g.abs() * (2 * share[:, None] + 8 * U)
    if case.dtype == "bf16":
        off = off + 1.02 * (2.0 ** -11 + 2.0 ** -8) * g.abs() + 2.0 ** -39 * weight.abs()
    step = HALF_STEP[case.dtype]
    case.off["dh"] = off @ w.abs() + (case.vocab + 2) * U * (g.abs() @ w.abs()) + step * case.want["dh"].abs()
    case.off["dweight"] = off.t() @ h.abs() + (case.tokens + 2) * U * (g.abs().t() @ h.abs()) + step * case.want["dweight"].abs()
    return case


def check(case):
    got = case.out["loss"].double().cpu()
    assert (got >= 0).all(), float(got.min())
    for name, value in case.out.items():
        value = value.double().cpu()
        err, off = (value - case.want[name]).abs(), case.off[name] + 1e-30
        assert (err <= off).all(), (name, float((err / off).max()), int((err > off).sum()), float((err / case.want[name].abs()).max()))


# (tokens, vocab, width, dh, dweight): few tokens alone and with gradients; tiles that read everything in place; tiles, with rows by 256, 64 and 1024
# threads; sums of logits shared; large tiles; exponentials counted from one number for a row
CALLS = [(1, 8192, 512, 0, 0), (16, 1000, 64, 0, 0), (1, 8192, 512, 1, 1), (9, 1000, 256, 1, 1), (1, 17000, 64, 0, 0), (48, 17000, 256, 0, 0),
         (300, 2048, 64, 1, 1), (1100, 2048, 64, 1, 1), (1100, 2048, 64, 0, 0), (100, 70000, 64, 1, 0), (18, 130, 2048, 1, 0), (71, 200, 1024, 1, 1),
         (265, 37543, 64, 1, 1), (538, 40884, 64, 1, 0), (64, 5, 64, 1, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("tokens,vocab,width,dh,dweight", CALLS)
def test_learned_words(loss, tokens, vocab, width, dh, dweight, whole, dtype):  # noqa: F811
    case = expect(learned(tokens, vocab, width, dtype, whole), whole)
    case.run(loss, dh=bool(dh), dweight=bool(dweight))
    check(case)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_learned_words_with_weights(loss, dtype):  # noqa: F811
    case = learned(300, 1000, 128, dtype, True)
    case.dloss = torch.randn(300, generator=torch.Generator().manual_seed(2))
    expect(case, True).run(loss)
    check(case)


# few tokens alone and with gradients, tiles that read everything in place, tiles with rows by 256, 64 and 1024 threads, shared sums, large tiles,
# exponentials counted from one number for a row
DISTILLED = [(1, 8192, 512, 0, 0), (9, 1000, 256, 1, 1), (1, 17000, 64, 0, 0), (48, 17000, 256, 0, 0), (300, 2048, 64, 1, 1), (300, 2048, 2048, 1, 1),
             (1100, 2048, 64, 1, 1), (18, 130, 2048, 1, 0), (265, 37543, 64, 1, 1), (538, 40884, 64, 1, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("tokens,vocab,width,dh,dweight", DISTILLED)
def test_learned_from_a_teacher_with_one_entry(loss, tokens, vocab, width, dh, dweight, whole, dtype):  # noqa: F811
    """As of a target: q is 1, whatever the teacher's logit is."""
    case = expect(learned(tokens, vocab, width, dtype, whole, seed=1), whole)
    case.k, case.ids, case.logits = 1, case.targets[:, None].clone(), 5.0 * torch.randn(tokens, 1, generator=torch.Generator().manual_seed(3))
    case.run(loss, dh=bool(dh), dweight=bool(dweight))
    check(case)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", [c[:3] for c in DISTILLED])
def test_divergence_of_what_is_learned(loss, tokens, vocab, width, dtype):  # noqa: F811
    """Several entries, of which the teacher means one: an error of the logits counts by how far the two distributions are apart, as the loss and
    its sum of exponentials have the same ones."""
    case, k = learned(tokens, vocab, width, dtype, False, seed=2), 8
    gen = torch.Generator().manual_seed(4)
    case.k, case.ids = k, torch.randint(0, vocab, (tokens, k), generator=gen)
    case.ids[:, 0] = case.targets
    case.logits = torch.randn(tokens, k, generator=gen) - 14.0
    case.logits[:, 0] = 0.0
    case.run(loss, dh=False, dweight=False)
    h, w, u = case.h.double(), case.weight.double(), case.logits.double()
    z, log_q = h @ w.t(), torch.log_softmax(u, 1)
    q, lse = log_q.exp(), torch.logsumexp(z, 1)
    off, p = lse[:, None] - z.gather(1, case.ids), (z - lse[:, None]).exp()
    want = (q * (log_q + off)).sum(1)
    apart = p.scatter_add(1, case.ids, -q).abs()
    rest = 1.0 - p.gather(1, case.targets[:, None])[:, 0]
    # logits: sums of `width` products; the sum of exponentials: arguments of those that are not the largest, and additions.  It has the largest in it, here
    # about all of it, from the first lane that adds it on: each of the at most 4 + 64 + 16 + vocab / 64 additions behind each other that follow
    # rounds a number of at least 1/2 and below 2, by U at the most, however small what is added is, and an error of a sum near 1 is one of its logarithm;
    # q, of 8 exponentials, their sum and a division; what is summed with it
    bound = 2 * (apart * ((width + 2) * U * (h.abs() @ w.abs().t()))).sum(1) + 2 * (z.amax(1) - z.amin(1)) * U * rest + (84 + vocab / 64 + 8) * U
    bound += (q * ((2 * log_q.abs() + 40) * U * (log_q + off).abs() + 8 * U * (u.abs() + log_q.abs() + off))).sum(1)
    err = (case.out["loss"].double().cpu() - want).abs()
    assert (err <= bound).all(), (float((err / bound).max()), float(err.max()))
    assert float(bound.median()) < (100 + vocab / 64) * U + 2e-5
