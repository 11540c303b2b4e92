"""The losses (tsenor_loss.h) against plain 64-bit implementations on the CPU."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def loss():
    from paper_2505_23949_amd import loss as module

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return module


def on_gpu(x, ld=None, offset=0):
    """x on the GPU; with ld, as a column range of a wider matrix filled with NaN."""
    if ld is None:
        return x.cuda()
    wide = torch.full((x.shape[0], ld), math.nan, dtype=x.dtype)
    wide[:, offset:offset + x.shape[1]] = x
    return wide.cuda()[:, offset:offset + x.shape[1]]


class Case:
    """Inputs of a call (on the CPU, in the call's types), and what it has to give in 64 bits with how far off that may be."""

    def __init__(self, tokens, vocab, width, dtype="bf16", k=0, temperature=1.0, left_out=0.0, dloss=True, spread=2.0, seed=0, teacher=torch.float32):
        gen = torch.Generator().manual_seed(1000 * seed + tokens + 7 * vocab + 13 * width + k)
        self.tokens, self.vocab, self.width, self.dtype, self.k, self.temperature = tokens, vocab, width, dtype, k, temperature
        self.h = torch.randn(tokens, width, generator=gen).to(DTYPES[dtype])
        self.weight = (spread / max(width, 1) ** 0.5 * torch.randn(vocab, width, generator=gen)).to(DTYPES[dtype])
        out = torch.rand(tokens, generator=gen) < left_out
        if k:
            self.ids = torch.stack([torch.randperm(vocab, generator=gen)[:k] for _ in range(tokens)]) if tokens else torch.zeros(0, k, dtype=torch.int64)
            self.logits = (3.0 * torch.randn(tokens, k, generator=gen)).to(teacher)
            self.ids[out] = -1
        else:
            self.targets = torch.randint(0, vocab, (tokens,), generator=gen)
            self.targets[out] = -100
        self.dloss = torch.randn(tokens, generator=gen) if dloss else None

    def reference(self, device="cpu"):
        """On the GPU (in torch's 64-bit operations) where the CPU would take seconds."""
        if device != "cpu":
            there = Case.__new__(Case)
            there.__dict__.update({k: v.to(device) if isinstance(v, torch.Tensor) else v for k, v in self.__dict__.items()})
            with torch.device(device):
                there.reference()
            self.want, self.off = ({k: v.cpu() for k, v in d.items()} for d in (there.want, there.off))
            return self
        h, w, inverse = self.h.double(), self.weight.double(), 1.0 / self.temperature
        z = (h @ w.t()) * inverse
        lse = torch.logsumexp(z, 1)
        if self.k:
            valid = (self.ids >= 0) & (self.ids < self.vocab)
            ids = torch.where(valid, self.ids, 0)
            u = torch.where(valid, self.logits.double() * inverse, -math.inf)
            counts = (u != -math.inf).any(1)
            q = torch.where(counts[:, None], torch.softmax(u, 1), 0.0)
        else:
            valid = ((self.targets >= 0) & (self.targets < self.vocab))[:, None]
            ids, counts, q = torch.where(valid, self.targets[:, None], 0), valid[:, 0], valid.double()
        log_q = torch.where(q > 0, q.log(), 0.0)
        terms = torch.where(q > 0, q * (log_q - z.gather(1, ids) + lse[:, None]), 0.0)
        weight = (torch.ones(self.tokens, dtype=torch.float64) if self.dloss is None else self.dloss.double()) * inverse
        p = (z - lse[:, None]).exp()
        onto = torch.zeros_like(p).scatter_add_(1, ids, q)
        g = torch.where(counts[:, None], (p - onto) * weight[:, None], 0.0)
        self.want = {"loss": torch.where(counts, terms.sum(1), 0.0), "lse": torch.where(counts, lse, 0.0), "dh": g @ w, "dweight": g.t() @ h}

        # A logit: products and sums of `width` terms and the scaling, any order: width + 2 roundings of the sum of sizes.
        dz = (self.width + 2) * U * (h.abs() @ w.abs().t()) * inverse
        dz_most = dz.amax(1) if self.vocab else torch.zeros(self.tokens, dtype=torch.float64)
        # A sum of exponentials: each off by its argument's rounding (of at most the range of z, twice) and 4 last places, sums over at most
        # 64 + 16 + vocab / 64 terms one behind the other.
        far = 2.0 * (z.amax(1) - z.amin(1)) * U if self.vocab else 0.0
        of_sum = far + (4 + 80 + self.vocab / 64) * U
        off_lse = dz_most + of_sum + 4 * U * lse.abs()
        size = (z.abs() * onto).sum(1) + (q * log_q.abs()).sum(1) + lse.abs()
        # (of the teacher's: its own logits, of at most 8 entries behind each other in a lane, their exponentials and logarithms)
        of_q = (32 + 4 * self.k + 4 * torch.where(q > 0, log_q, 0.0).abs().amax(1)) * U if self.k else 0.0
        off_loss = 2 * dz_most + off_lse + 16 * U * size + (of_q * (size + 1.0) if self.k else 0.0)
        # the gradient of a logit: that of its probability, the roundings of subtraction and scaling; bf16: exponentials kept in
        # fp16 (2^-11, steps of 2^-24 of 2^15 of the largest of a tile at the smallest), dz in bf16
        of_p = (dz_most + off_lse + far + 8 * U)[:, None] * p
        off_g = weight.abs()[:, None] * (of_p + 4 * U * (p + onto) + (of_q[:, None] * onto if self.k else 0.0))
        if self.dtype == "bf16":
            off_g = off_g + 2.0 ** -11 * weight.abs()[:, None] * (p + 2.0 ** -28 * p.amax(1, keepdim=True)) + 2.0 ** -8 * g.abs() * 1.01
        off_g = torch.where(counts[:, None], off_g, 0.0)
        step = HALF_STEP[self.dtype]
        self.off = {"loss": torch.where(counts, off_loss, 0.0), "lse": torch.where(counts, off_lse, 0.0),
                    "dh": off_g @ w.abs() + (self.vocab + 2) * U * (g.abs() @ w.abs()) + step * self.want["dh"].abs() + 1e-37,
                    "dweight": off_g.t() @ h.abs() + (self.tokens + 2) * U * (g.abs().t() @ h.abs()) + step * self.want["dweight"].abs() + 1e-37}
        return self

    def describe(self, loss, *, dh=True, dweight=True, lse=True, ld=0, offset=0):
        self.gpu = {"h": on_gpu(self.h, self.width + ld if ld else None, offset), "weight": on_gpu(self.weight, self.width + ld if ld else None, offset)}
        self.out = {"loss": torch.full((self.tokens,), math.nan, device="cuda")}
        if lse:
            self.out["lse"] = torch.full((self.tokens,), math.nan, device="cuda")
        if dh:
            self.out["dh"] = torch.full((self.tokens, self.width), math.nan, dtype=DTYPES[self.dtype], device="cuda")
        if dweight:
            self.out["dweight"] = torch.full((self.vocab, self.width), math.nan, dtype=DTYPES[self.dtype], device="cuda")
        dloss = None if self.dloss is None else self.dloss.cuda()
        if self.k:
            self.gpu.update(ids=self.ids.cuda(), logits=self.logits.cuda(), dloss=dloss)
            p = loss.make_distill(self.gpu["h"], self.gpu["weight"], self.gpu["ids"], self.gpu["logits"], temperature=self.temperature, dloss=dloss, **self.out)
            size, self.call = loss.tsenor_distill_workspace_bytes(p), loss.tsenor_distill
        else:
            self.gpu.update(targets=self.targets.cuda(), dloss=dloss)
            p = loss.make_cross_entropy(self.gpu["h"], self.gpu["weight"], self.gpu["targets"], dloss=dloss, **self.out)
            size, self.call = loss.tsenor_cross_entropy_workspace_bytes(p), loss.tsenor_cross_entropy
        assert size > 0
        self.problem, self.work = p, torch.full((size,), 255, dtype=torch.uint8, device="cuda")  # (NaN, whatever type it is read as)
        return self

    def run(self, loss, **kw):
        self.describe(loss, **kw)
        self.call(self.problem, self.work)
        torch.cuda.synchronize()
        return self

    def check(self):
        for name, got in self.out.items():
            got, want, off = got.double().cpu(), self.want[name], self.off[name]
            err = (got - want).abs()
            assert (err <= off).all(), (name, float((err / off).nan_to_num(math.inf).max()), int((~(err <= off)).sum()))
        if self.dtype == "bf16":
            # Roundings of either sign add up like a walk: bf16 is off by 2^-9 of a value on average at the most, and there are three (fp16's
            # counts as one).
            for name in ("dh", "dweight"):
                if name in self.out and self.want[name].numel() > 100:
                    err = (self.out[name].double().cpu() - self.want[name]).norm()
                    assert err <= 3 * 2.0 ** -9 * self.want[name].norm() + 1e-30, name


# ---- values ---------------------------------------------------------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 5, 7), (2, 64, 64), (3, 129, 100), (16, 1000, 72), (17, 257, 256), (64, 128, 128), (65, 300, 513), (130, 1029, 96),
         (257, 515, 320), (300, 2048, 64), (9, 4099, 129),
         (70, 700, 328), (2, 534, 1096), (2049, 300, 40), (71, 200, 1200), (40, 300, 1500), (20, 130, 3008)]


# (tokens, vocab, width, dh, dweight) of calls that take the larger tiles, shared sums and the like; PICKED: with so many entries that their rows of
# the head are not read again
LARGER = [(137, 34211, 64, 0, 0), (66, 17572, 64, 1, 1), (18, 34795, 64, 0, 0), (132, 17148, 272, 0, 0), (18, 130, 1856, 1, 0), (7377, 133, 1040, 1, 0),
          (6873, 141, 520, 1, 1), (5971, 139, 264, 1, 0), (5648, 259, 672, 1, 1), (17, 130, 64, 1, 0), (898, 7219, 4288, 1, 0), (262, 9910, 4120, 1, 0),
          (2794, 3762, 136, 1, 0), (162, 6137, 5384, 1, 0), (16, 1220, 64, 1, 0), (17, 33043, 144, 1, 1), (16, 17269, 144, 1, 1), (2178, 277, 1840, 1, 1),
          (579, 1819, 1272, 1, 1), (265, 37543, 64, 1, 1), (7147, 654, 5384, 0, 1), (6797, 336, 5408, 0, 1), (4718, 130, 800, 0, 1), (3831, 467, 1344, 0, 1),
          (6635, 136, 5384, 0, 1), (19, 52402, 1192, 1, 1), (67, 35502, 1968, 0, 1), (1376, 32990, 144, 1, 1), (4005, 2790, 3000, 0, 1),
          (18, 1083, 1888, 1, 1), (1, 129, 64, 0, 1), (1, 18232, 64, 0, 1), (65, 39796, 944, 0, 1), (1632, 33074, 144, 0, 1), (403, 8072, 5424, 1, 0),
          (144, 38235, 64, 1, 1), (3021, 7272, 1168, 0, 1)]
PICKED = [(512, 2000, 1024, "bf16", 64, 0.0), (700, 1031, 960, "bf16", 130, 0.2), (300, 1500, 1000, "f32", 100, 0.1), (2100, 4099, 512, "bf16", 256, 0.0)]


# up to 16 tokens, whose dh is made from the head as it stands: words by one workgroup and by many, rows of many blocks of columns, more words
# than stand in LDS at a time
FEW = [(1, 30, 12), (4, 33, 515), (5, 31, 1029), (16, 700, 1003), (13, 3001, 1203), (3, 901, 5083), (2, 70001, 77), (15, 70003, 133), (7, 513, 9), (1, 1025, 3), (14, 1601, 32769)]


@pytest.mark.parametrize("left_out", [0.0, 0.5])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", FEW)
def test_few_tokens(loss, tokens, vocab, width, dtype, left_out):
    for k, dweight in ((0, True), (3, False)):
        Case(tokens, vocab, width, dtype, k=k, left_out=left_out).reference("cuda").run(loss, dweight=dweight).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [64, 515, 1208])
def test_few_tokens_with_a_head_in_a_wider_matrix(loss, width, dtype):
    """Rows that begin at any element, NaN between them."""
    Case(9, 800, width, dtype).reference("cuda").run(loss, ld=3, offset=1).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width,dh,dweight", LARGER)
def test_larger_calls(loss, tokens, vocab, width, dh, dweight, dtype):
    Case(tokens, vocab, width, dtype, left_out=0.1).reference("cuda").run(loss, dh=bool(dh), dweight=bool(dweight)).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", SIZES)
def test_cross_entropy(loss, tokens, vocab, width, dtype):
    Case(tokens, vocab, width, dtype).reference().run(loss).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width", SIZES)
def test_distill(loss, tokens, vocab, width, dtype):
    for k, temperature in ((1, 1.0), (min(vocab, 5), 2.0), (min(vocab, 70), 0.7)):
        Case(tokens, vocab, width, dtype, k=k, temperature=temperature).reference().run(loss).check()


@pytest.mark.parametrize("tokens,vocab,width,dtype,k,left_out", PICKED)
def test_entries_picked_from_the_tiles(loss, tokens, vocab, width, dtype, k, left_out):
    """So many entries that their rows of the head are not read again."""
    case = Case(tokens, vocab, width, dtype, k=k, left_out=left_out, temperature=1.5)
    case.ids[0, :8] = torch.tensor([vocab - 1, 0, vocab - 1, 127, 128, 63, 64, 0]) % vocab  # ends, the same word twice
    case.ids[1, 5:] = -1
    case.ids[2, ::2] = vocab + 3
    case.ids[3, :] = 77
    case.reference().run(loss).check()


@pytest.mark.parametrize("k", [255, 256])
def test_most_entries(loss, k):
    Case(33, 600, 64, "bf16", k=k, temperature=3.0).reference().run(loss).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k", [0, 6])
@pytest.mark.parametrize("ld,offset", [(8, 0), (8, 8), (3, 1), (64, 16), (5, 5)])
def test_strides(loss, dtype, k, ld, offset):
    for width in (128, 72):
        Case(37, 260, width, dtype, k=k).reference().run(loss, ld=ld, offset=offset).check()


@pytest.mark.parametrize("k", [0, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left_out", [0.02, 0.5, 0.97])
def test_tokens_left_out(loss, dtype, k, left_out):
    for tokens in (5, 200, 9001 if dtype == "f32" and k == 0 else 513):
        case = Case(tokens, 140, 64, dtype, k=k, left_out=left_out).reference()
        # hidden states of tokens that are left out are not looked at
        out = case.want["loss"] == 0
        case.h[out] = math.nan
        case.run(loss).check()
        for name in ("loss", "lse", "dh"):
            assert not case.out[name].cpu()[out].any(), name


@pytest.mark.parametrize("k", [0, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_token_counts(loss, dtype, k):
    # (with the larger vocabulary, workgroups share the sums of dh)
    for vocab in (200, 4099):
        case = Case(70, vocab, 64, dtype, k=k, left_out=1.1).run(loss)
        for name, got in case.out.items():
            assert not got.cpu().any(), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_targets_at_and_outside_the_ends(loss, dtype):
    case = Case(9, 100, 64, dtype)
    case.targets = torch.tensor([0, 99, 100, -1, -100, 2 ** 40, -2 ** 62, 50, 2 ** 32 + 3])
    case.reference().run(loss).check()
    assert (case.out["loss"].cpu() != 0).tolist() == [True, True] + [False] * 5 + [True, False]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_entries_that_take_no_part(loss, dtype):
    case = Case(8, 90, 64, dtype, k=7)
    case.ids[0, 3:] = -1                       # padding
    case.ids[1, 0] = 90                        # outside the vocabulary
    case.ids[2, 2] = 2 ** 33
    case.logits[3, 4] = -math.inf              # a word that the teacher rules out
    case.logits[4, :] = -math.inf              # all of them: left out
    case.ids[5, :] = -5
    case.ids[6, 1:] = case.ids[6, 0]           # the same word in all entries
    case.ids[7, 4] = case.ids[7, 2]
    case.logits[0, 4] = math.nan               # not looked at
    case.reference().run(loss).check()
    assert (case.out["loss"].cpu()[[4, 5]] == 0).all()


@pytest.mark.parametrize("teacher", [torch.float32, torch.bfloat16])
def test_teachers_types(loss, teacher):
    Case(20, 300, 64, "bf16", k=9, teacher=teacher).reference().run(loss).check()


@pytest.mark.parametrize("wanted", [dict(dh=False, dweight=False, lse=False), dict(dh=False, dweight=False), dict(dweight=False), dict(dh=False), dict(lse=False)])
@pytest.mark.parametrize("k", [0, 5])
@pytest.mark.parametrize("tokens", [1, 7, 40, 300])
def test_outputs_that_are_wanted(loss, wanted, k, tokens):
    Case(tokens, 700, 192, "bf16", k=k, left_out=0.1 * (tokens > 1)).reference().run(loss, **wanted).check()


@pytest.mark.parametrize("k", [0, 4])
def test_without_weights_of_the_losses(loss, k):
    Case(50, 333, 64, "f32", k=k, dloss=False).reference().run(loss).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spread", [0.0, 40.0, 1000.0])
def test_flat_and_peaked(loss, dtype, spread):
    """Logits that are all the same, and thousands apart: exponentials that leave single precision are 0."""
    Case(40, 700, 64, dtype, spread=spread).reference().run(loss).check()
    Case(40, 700, 64, dtype, k=8, spread=spread).reference().run(loss).check()


def test_learned_targets(loss):
    """Probabilities near 1: 1 - p comes from single precision, not from what dz is kept in."""
    case = Case(64, 512, 64, "bf16")
    case.weight = (8.0 * torch.eye(512, 64)[torch.randperm(512, generator=torch.Generator().manual_seed(1))]).bfloat16()
    rows = torch.nonzero(case.weight.float().abs().sum(1))[:, 0]
    case.targets = rows[torch.arange(64) % len(rows)]
    case.h = (2.0 * case.weight[case.targets].float()).bfloat16()
    case.reference().run(loss).check()
    assert float(case.out["loss"].max()) < 1e-3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k", [0, 3])
def test_nan_stays_with_its_token(loss, dtype, k):
    case = Case(6, 150, 64, dtype, k=k)
    case.h[2, 5], case.h[4, 0] = math.nan, math.inf
    case.run(loss, dweight=False)
    got = case.out["loss"].cpu()
    assert torch.isnan(got).tolist() == [False, False, True, False, True, False]
    dh = case.out["dh"].float().cpu()
    assert torch.isnan(dh).all(1).tolist() == [False, False, True, False, True, False]
    clean = Case(6, 150, 64, dtype, k=k).reference()
    keep = [0, 1, 3, 5]
    assert ((dh.double()[keep] - clean.want["dh"][keep]).abs() <= clean.off["dh"][keep]).all()
    assert ((got.double()[keep] - clean.want["loss"][keep]).abs() <= clean.off["loss"][keep]).all()


def test_nothing_to_do(loss):
    for tokens, vocab, width, k in ((0, 100, 64, 0), (0, 100, 64, 3), (5, 100, 0, 0), (5, 100, 0, 2), (0, 0, 0, 0)):
        case = Case(tokens, max(vocab, 1), width, "bf16", k=k).reference()
        case.run(loss)
        case.check()
        if tokens == 0:
            assert not case.out["dweight"].cpu().any()
    # no vocabulary: no target is in it
    h, weight, targets = torch.ones(4, 64, device="cuda"), torch.zeros(0, 64, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    out, dh = torch.ones(4, device="cuda"), torch.ones(4, 64, device="cuda")
    p = loss.make_cross_entropy(h, weight, targets, loss=out, dh=dh)
    loss.tsenor_cross_entropy(p, torch.empty(loss.tsenor_cross_entropy_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    assert not out.any() and not dh.any()


@pytest.mark.parametrize("k", [0, 5])
@pytest.mark.parametrize("far", [False, True])
def test_dh_alone_of_many_logits(loss, k, far):
    """Exponentials counted from a row's own entries; `far`: entries that the largest logit is hundreds above, for which that does not do."""
    tokens = 538
    case = Case(tokens, 40884, 72, "bf16", k=k, left_out=0.05, temperature=1.3 if k else 1.0)
    if far:
        # word 7 is worth 300 to token 3 and its like, whose entries are none of it
        case.h[3::31, 0] = 40.0
        case.weight[7, 0] = 8.0
        if k:
            case.ids[:, 0] = torch.where(case.ids[:, 0] == 7, 8, case.ids[:, 0])
        else:
            case.targets[case.targets == 7] = 8
    case.reference("cuda").run(loss, dweight=False).check()
    if far:
        assert float(case.out["loss"].max()) > 150
    case.h[10, 3] = math.nan
    out = case.out["dh"].clone()
    case.run(loss, dweight=False)
    keep = torch.arange(tokens) != 10
    assert torch.isnan(case.out["loss"].cpu()[10]) == (case.want["loss"][10] != 0)
    assert torch.isfinite(case.out["dh"].float().cpu()[keep]).all()
    assert torch.equal(case.out["dh"].cpu()[keep], out.cpu()[keep])


# ---- gradients against differences -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("k,temperature", [(0, 1.0), (6, 1.5)])
def test_gradients_against_differences(loss, k, temperature):
    """(L(x + e d) - L(x - e d)) / 2e along random directions, L = sum(dloss loss) from the kernels' own losses."""
    case = Case(24, 200, 64, "f32", k=k, temperature=temperature).reference().run(loss)
    grad = {"h": case.out["dh"].double().cpu(), "weight": case.out["dweight"].double().cpu()}
    gen = torch.Generator().manual_seed(5)
    e = 2.0 ** -7
    for name in ("h", "weight"):
        at = getattr(case, name).clone()
        d = torch.randn(at.shape, generator=gen)
        d = (d / (d @ (case.weight if name == "h" else case.h).t()).abs().max()).float()  # logits change by 1 at most
        value = []
        for sign in (1, -1):
            setattr(case, name, at + sign * e * d)
            case.run(loss, dh=False, dweight=False)
            value.append(float((case.dloss.double() * case.out["loss"].double().cpu()).sum()))
        setattr(case, name, at)
        got, want = (value[0] - value[1]) / (2 * e), float((grad[name] * d.double()).sum())
        # losses are off by `off` each, x + e d by a last place of x, which changes a logit by 2^-24 of the sum of its sizes (part of `off`);
        # the third derivative of a loss along changes of at most 1 / temperature is at most 4 of those cubed
        scale = case.dloss.double().abs()
        bound = float((scale * 4 * case.off["loss"]).sum()) / e + e * e * 4 / 6 * float(scale.sum()) + float((case.off["dh" if name == "h" else "dweight"] * d.abs().double()).sum())
        assert abs(got - want) <= bound, (name, got, want, bound)
        assert bound < 0.1 * grad[name].norm() * d.double().norm()


# ---- how calls are made ------------------------------------------------------------------------------------------------------

def test_rows_of_one_call_are_those_of_several(loss):
    """What a token gets does not depend on the tokens beside it (losses and dh, bit by bit at the same kernels)."""
    whole = Case(512, 700, 128, "bf16", k=5).run(loss)
    part = Case(512, 700, 128, "bf16", k=5)
    order = torch.randperm(512, generator=torch.Generator().manual_seed(3))
    part.h, part.ids, part.logits, part.dloss = part.h[order], part.ids[order], part.logits[order], part.dloss[order]
    part.run(loss)
    for name in ("loss", "lse", "dh"):
        assert torch.equal(part.out[name].cpu(), whole.out[name].cpu()[order]), name


def test_repeats_give_the_same_bits(loss):
    case = Case(300, 3000, 256, "bf16", left_out=0.2).run(loss)
    first = {name: t.clone() for name, t in case.out.items()}
    for _ in range(3):
        case.work.random_(0, 255)
        case.call(case.problem, case.work)
        torch.cuda.synchronize()
        for name, t in case.out.items():
            assert torch.equal(t, first[name]), name


@pytest.mark.parametrize("tokens", [1, 40, 200])
@pytest.mark.parametrize("k", [0, 4])
def test_captured_and_replayed(loss, tokens, k):
    """Two captured calls, replayed in turn with eager ones, each with a workspace of its own; inputs change between."""
    cases = [Case(tokens, 500, 128, "bf16", k=k, seed=s, left_out=0.3 * (tokens > 1)).run(loss) for s in (1, 2)]
    graphs = []
    for case in cases:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            case.call(case.problem, case.work)
        graphs.append(graph)
    for turn in range(4):
        want = []
        for case in cases:
            fresh = Case(tokens, 500, 128, "bf16", k=k, seed=10 + turn, left_out=0.2 * (tokens > 1)).run(loss)
            for name, t in fresh.gpu.items():
                if t is not None:
                    case.gpu[name].copy_(t)
            want.append(fresh.out)
            for t in case.out.values():
                t.fill_(7.0)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for case, out in zip(cases, want):
            for name, t in case.out.items():
                assert torch.equal(t, out[name]), (turn, name)


def test_streams(loss):
    """Two calls at once, on streams of their own."""
    cases = [Case(200, 1500, 256, "bf16", k=k).reference().describe(loss) for k in (0, 5)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        for case, stream in zip(cases, streams):
            case.call(case.problem, case.work, stream=stream)
    torch.cuda.synchronize()
    for case in cases:
        case.check()


def test_pieces(loss):
    """More logits than are kept at a time: the second piece's gradients of the head are added to the first one's."""
    tokens, vocab, width = 9000, 131072, 64
    gen = torch.Generator(device="cuda").manual_seed(0)
    h = torch.randn(tokens, width, device="cuda", generator=gen).bfloat16()
    weight = (0.3 * torch.randn(vocab, width, device="cuda", generator=gen)).bfloat16()
    targets = torch.randint(-vocab // 4, vocab, (tokens,), device="cuda", generator=gen)
    scale = torch.rand(tokens, device="cuda", generator=gen)

    def call(rows, dtype=torch.bfloat16):
        n = h[rows].shape[0]
        out = {"loss": torch.empty(n, device="cuda"), "dh": torch.empty(n, width, dtype=dtype, device="cuda"),
               "dweight": torch.empty(vocab, width, dtype=dtype, device="cuda")}
        inputs = h[rows].to(dtype), weight.to(dtype), targets[rows]
        p = loss.make_cross_entropy(*inputs, dloss=scale[rows], **out)
        size = loss.tsenor_cross_entropy_workspace_bytes(p)
        assert size < 2 ** 32
        loss.tsenor_cross_entropy(p, torch.empty(size, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        return out

    # a tile of logits of a token is the same whatever piece it is in; parts of the head's gradient are rounded to bf16 here, and once there
    for dtype, off in ((torch.bfloat16, 2.0 ** -8), (torch.float32, 2.0 ** -16)):
        whole, parts = call(slice(None), dtype), [call(slice(0, 3000), dtype), call(slice(3000, 6000), dtype), call(slice(6000, None), dtype)]
        torch.cuda.synchronize()
        assert torch.equal(whole["loss"], torch.cat([p["loss"] for p in parts]))
        assert (whole["dh"].float() - torch.cat([p["dh"].float() for p in parts])).norm() <= off * whole["dh"].float().norm()
        want = sum(p["dweight"].float() for p in parts)
        assert (whole["dweight"].float() - want).norm() <= 2 * off * want.norm()
        assert whole["dweight"].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width,k", [(40, 300, 64, 0), (40, 300, 64, 9), (1400, 515, 136, 0), (10, 129, 72, 3), (300, 70000, 64, 2)])
def test_weights_and_teachers_that_are_no_numbers(loss, tokens, vocab, width, k, dtype):
    """An infinite or NaN weight, or a teacher's NaN, is its own token's: losses and dh of the others are what they are without it."""
    case = Case(tokens, vocab, width, dtype, k=k)
    case.dloss[2], case.dloss[4] = 0.0, 0.0
    case.reference("cuda")
    case.dloss[2], case.dloss[4] = math.inf, math.nan
    if k:
        case.logits[6, 1] = math.nan
    out = case.run(loss, dweight=False).out
    got = {name: v.double().cpu() for name, v in out.items()}
    assert not got["dh"][[2, 4]].isfinite().any()
    rest = torch.ones(tokens, dtype=torch.bool)
    if k:
        rest[6] = False
        assert got["loss"][6].isnan() and got["dh"][6].isnan().all()
    assert ((got["loss"] - case.want["loss"]).abs() <= case.off["loss"])[rest].all()  # (a weight does not touch the loss)
    rest[[2, 4]] = False
    assert ((got["dh"] - case.want["dh"]).abs() <= case.off["dh"])[rest].all()
