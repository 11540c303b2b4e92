"""Logits of minus infinity (products beyond single precision): a word of probability 0, whichever kernels make the call."""
import math

import pytest
import torch

from test_gpu_loss import Case, loss  # noqa: F401  (loss: a fixture)

pytestmark = pytest.mark.gpu

# (tokens, vocab, width, dtype, dh, dweight): exponentials counted from one number for a row; large tiles; small ones; few tokens; scores in place
CALLS = [(538, 40884, 72, "bf16", True, False), (300, 38000, 64, "bf16", True, True), (100, 300, 64, "bf16", True, True), (100, 300, 64, "f32", True, True),
         (6, 300, 64, "bf16", True, True), (6, 300, 72, "f32", True, False), (40, 300, 64, "bf16", False, False), (6, 300, 64, "f32", False, False)]


@pytest.mark.parametrize("k", [0, 1, 3])
@pytest.mark.parametrize("tokens,vocab,width,dtype,dh,dweight", CALLS)
def test_a_word_of_probability_zero(loss, tokens, vocab, width, dtype, dh, dweight, k):  # noqa: F811
    word, its = 7, torch.arange(0, tokens, 5)
    case = Case(tokens, vocab, width, dtype, k=k)
    if k:
        case.ids = torch.where(case.ids == word, word + 1, case.ids)
        case.ids[its, k - 1] = word
    else:
        case.targets = torch.where(case.targets == word, word + 1, case.targets)
        case.targets[its] = word
    case.h[:, 0], case.weight[:, 0] = 1.0, 0.0
    case.weight[word, 0] = -300.0                    # e^-300 is 0 in single precision as well: what is wanted but for the word's own logit
    case.reference("cuda")
    case.h[:, 0], case.weight[word, 0] = 2.0 ** 100, -2.0 ** 100
    case.run(loss, dh=dh, dweight=dweight)
    got = {name: value.double().cpu() for name, value in case.out.items()}
    theirs = torch.ones(tokens, dtype=torch.bool)
    theirs[its] = False
    assert (got["loss"][its] == math.inf).all()
    assert ((got["loss"] - case.want["loss"]).abs() <= case.off["loss"])[theirs].all()
    assert ((got["lse"] - case.want["lse"]).abs() <= case.off["lse"]).all()
    if dh:
        assert ((got["dh"] - case.want["dh"]).abs() <= case.off["dh"])[:, 1:].all()
        # dz of the word is -q dloss and what the word's row is multiplied with: two roundings to bf16, or some of single precision (q: its exponential, a
        # sum of k and a division)
        q = torch.softmax(case.logits.double(), 1)[its, k - 1] if k else 1.0
        want = 2.0 ** 100 * q * case.dloss[its].double()
        assert (got["dh"][theirs, 0] == 0).all()
        assert ((got["dh"][its, 0] - want).abs() <= (2.02 * 2.0 ** -8 if dtype == "bf16" else 128 * 2.0 ** -24) * want.abs()).all()
    if dweight:
        assert ((got["dweight"] - case.want["dweight"]).abs() <= case.off["dweight"])[:, 1:].all()


@pytest.mark.parametrize("k", [0, 3])
@pytest.mark.parametrize("tokens,vocab,width,dh,dweight", [(100, 300, 64, True, True), (100, 300, 77, False, False), (400, 2000, 64, True, False), (9, 300, 64, True, True)])
def test_the_largest_numbers_of_single_precision(loss, tokens, vocab, width, dh, dweight, k):  # noqa: F811
    """They round up to infinity in bf16, of which matrices in single precision are put together."""
    most = torch.finfo(torch.float32).max
    case = Case(tokens, vocab, width, "f32", k=k)
    case.h[:, 0], case.weight[:, 0] = 2.0 ** -125, 0.0
    case.h[:, 1], case.weight[:, 1] = 0.0, 2.0 ** -125
    case.weight[3, 0], case.h[5, 1] = most, -most
    case.weight[vocab - 1, 0], case.h[tokens - 1, 1] = -3.3999e38, 3.395e38
    case.dloss = 0.25 + 0.5 * torch.rand(tokens, generator=torch.Generator().manual_seed(1))  # (half the largest, or its neighbour in dweight has no room)
    case.dloss[5] = case.dloss[tokens - 1] = 0.1
    case.reference().run(loss, dh=dh, dweight=dweight).check()


@pytest.mark.parametrize("teacher", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,dh", [(5, False), (40, False), (40, True), (200, True)])
def test_teachers_of_the_largest_and_lowest_numbers(loss, tokens, dh, teacher):  # noqa: F811
    """Finite logits take part, though over the temperature they are beyond single precision (a mask of the type's lowest value)."""
    case = Case(tokens, 300, 64, "bf16", k=4, temperature=0.25, teacher=teacher)
    most = torch.finfo(teacher).max
    case.logits[0, :], case.logits[1, 1:], case.logits[2, :2], case.logits[3, :] = -most, -most, most, torch.tensor([most, -most, 0.0, -math.inf])
    case.logits[4, :] = torch.tensor([-math.inf, -most, -math.inf, -most])
    case.reference().run(loss, dh=dh, dweight=dh).check()
    assert (case.out["loss"][:5] != 0).all()


@pytest.mark.parametrize("k", [0, 3])
@pytest.mark.parametrize("tokens,vocab,width,dtype,dweight", [(100, 300, 64, "bf16", True), (100, 300, 64, "f32", True), (9, 300, 64, "f32", False), (538, 40884, 64, "bf16", False)])
def test_weights_far_apart(loss, tokens, vocab, width, dtype, dweight, k):  # noqa: F811
    """Gradients are made relative to the largest weight: those of a token whose own is 2^-80 of it are as right as its neighbours'."""
    case = Case(tokens, vocab, width, dtype, k=k)
    case.dloss[1::2] *= 2.0 ** -80
    case.dloss[0] = 2.0 ** 20
    case.reference("cuda").run(loss, dweight=dweight).check()
    small = case.out["dh"].float().cpu()[1::2]
    assert (small.abs().amax(1) > 0).all() and float(small.abs().max()) < 2.0 ** -60
