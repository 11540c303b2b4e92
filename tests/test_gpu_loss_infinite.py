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
