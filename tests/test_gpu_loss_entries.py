"""Distillation with one entry to a token and with several, by each of the ways that their logits come."""
import pytest
import torch

from test_gpu_loss import DTYPES, HALF_STEP, U, Case, loss  # noqa: F401  (loss: a fixture)

pytestmark = pytest.mark.gpu

# (tokens, vocab, width, dtype, k): gathered calls whose entries' logits come from the tiles, of one entry and of several; rows by 64, by 256
# and by 1024 threads
FROM_TILES = [(4096, 2500, 4096, "bf16", 1), (2100, 130, 8192, "bf16", 1), (1000, 600, 8192, "f32", 1), (1500, 2500, 4096, "bf16", 3), (2100, 1500, 8192, "bf16", 16),
              (400, 900, 2048, "f32", 40), (60, 70001, 64, "bf16", 1), (18, 66000, 72, "f32", 1)]


@pytest.mark.parametrize("tokens,vocab,width,dtype,k", FROM_TILES)
def test_entries_from_the_tiles(loss, tokens, vocab, width, dtype, k):  # noqa: F811
    case = Case(tokens, vocab, width, dtype, k=k, left_out=0.1, temperature=1.5).reference("cuda")
    case.run(loss).check()


# (tokens, vocab, width, dtype, k) of scores that look through all entries: few tokens, tiles that read everything in place; one round of entries and many
SCORES = [(1, 700, 72, "bf16", 2), (1, 700, 72, "f32", 256), (16, 1003, 64, "bf16", 33), (16, 1003, 515, "f32", 5), (7, 40, 64, "bf16", 40), (1, 17000, 64, "bf16", 8),
          (17, 900, 192, "bf16", 3), (48, 17000, 64, "bf16", 70), (64, 333, 128, "bf16", 256), (33, 130, 1856, "bf16", 9), (40, 700, 64, "bf16", 1)]


@pytest.mark.parametrize("tokens,vocab,width,dtype,k", SCORES)
def test_scores_look_for_their_entries(loss, tokens, vocab, width, dtype, k):  # noqa: F811
    case = Case(tokens, vocab, width, dtype, k=k, left_out=0.1 * (tokens > 1), temperature=0.8)
    gen = torch.Generator().manual_seed(k)
    case.ids[torch.rand(tokens, k, generator=gen) < 0.2] = vocab                     # outside the vocabulary, by one
    case.ids[torch.rand(tokens, k, generator=gen) < 0.1] = -2 ** 40
    case.ids[0, 0], case.ids[0, -1] = vocab - 1, vocab - 1                           # the last word, twice where there are several
    case.reference().run(loss, dh=False, dweight=False).check()


@pytest.mark.parametrize("tokens,dh", [(5, False), (40, False), (40, True), (300, True)])
@pytest.mark.parametrize("k", [1, 6])
def test_entries_in_a_wider_matrix(loss, tokens, dh, k):  # noqa: F811
    case = Case(tokens, 700, 64, "bf16", k=k).reference()
    case.describe(loss, dh=dh, dweight=dh)
    ids, logits = torch.full((tokens, k + 5), -7, device="cuda"), torch.full((tokens, k + 3), float("nan"), device="cuda")
    ids[:, 2:2 + k], logits[:, 3:] = case.ids.cuda(), case.logits.cuda()
    p = loss.make_distill(case.gpu["h"], case.gpu["weight"], ids[:, 2:2 + k], logits[:, 3:], dloss=case.gpu["dloss"], **case.out)
    assert loss.tsenor_distill_workspace_bytes(p) == case.work.numel()
    loss.tsenor_distill(p, case.work)
    torch.cuda.synchronize()
    case.check()


@pytest.mark.parametrize("tokens,vocab,width,dtype,gradients", [(1 << 24, 5, 8, "bf16", True), (1 << 24, 5, 8, "f32", False), (540000, 7, 2048, "bf16", True),
                                                                 (200000, 7, 2048, "f32", True)])
def test_many_tokens_of_few_words(loss, tokens, vocab, width, dtype, gradients):  # noqa: F811
    """As many tokens as there may be, more than the threads of one launch are for; and more hidden states than are copied at a time."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    h = torch.rand(tokens, width, device="cuda", generator=gen).to(DTYPES[dtype])
    weight = (torch.randn(vocab, width, device="cuda", generator=gen) * (8 / width) ** 0.5).to(DTYPES[dtype])
    targets = torch.randint(-1, 2, (tokens,), device="cuda", generator=gen)         # two of the words, and a third left out
    out = {"loss": torch.full((tokens,), float("nan"), device="cuda"), "lse": torch.full((tokens,), float("nan"), device="cuda")}
    if gradients:
        out["dh"], out["dweight"] = torch.full_like(h, float("nan")), torch.full_like(weight, float("nan"))
    p = loss.make_cross_entropy(h, weight, targets, **out)
    loss.tsenor_cross_entropy(p, torch.empty(loss.tsenor_cross_entropy_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    counts, x, w = targets >= 0, h.double(), weight.double()
    z = x @ w.t()
    lse = torch.logsumexp(z, 1)
    off = (width + 24) * U * (1 + (x @ w.t().abs()).amax(1))                         # a logit of `width` products, and a sum of a few exponentials
    assert ((out["lse"].double() - lse)[counts].abs() <= off[counts]).all()
    assert ((out["loss"].double() - (lse - z.gather(1, targets.clamp(min=0)[:, None])[:, 0]))[counts].abs() <= 2 * off[counts]).all()
    assert not out["lse"][~counts].any() and not out["loss"][~counts].any()
    if gradients:
        g = (z - lse[:, None]).exp().scatter_add_(1, targets.clamp(min=0)[:, None], torch.full((tokens, 1), -1.0, dtype=torch.float64, device="cuda"))
        g[~counts] = 0.0
        # logits, fp16, bf16, and the result's rounding; dweight: at most 2^24 additions shared by 128 workgroups
        rough = 2 * float(off.max()) + 64 * U + (1.01 * (2.0 ** -11 + 2.0 ** -8) if dtype == "bf16" else 0.0)
        step = HALF_STEP[dtype]
        want = g @ w
        assert ((out["dh"].double() - want).abs() <= rough * (g.abs() @ w.abs()) + step * want.abs() + 1e-30).all()
        want, sizes = g.t() @ x, g.t().abs() @ x.abs()
        assert ((out["dweight"].double() - want).abs() <= (rough + 2 ** 17 * U) * sizes + step * want.abs()).all()
        assert (want.abs() > 0.1 * sizes).all(1).any()                               # (of the inputs: what a bound of sizes says something of)
