"""Distillation at the ends of the temperature's range, with logits that are exact in single precision."""
import pytest
import torch

from test_gpu_loss import DTYPES, HALF_STEP, U, Case, loss  # noqa: F401  (loss: a fixture)

pytestmark = pytest.mark.gpu

# few tokens, tiles, large tiles, exponentials counted from one number for a row; scores in place
CALLS = [(7, 300, 64, True, True), (100, 300, 64, True, True), (265, 37543, 64, True, True), (538, 40884, 64, True, False), (40, 300, 64, False, False)]


@pytest.mark.parametrize("temperature", [2.0 ** -20, 2.0 ** -10, 2.0 ** 20])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,width,dh,dweight", CALLS)
def test_ends_of_the_range(loss, tokens, vocab, width, dh, dweight, dtype, temperature):  # noqa: F811
    k, gen = 3, torch.Generator().manual_seed(tokens)
    case = Case(tokens, vocab, width, dtype, k=k, temperature=temperature)
    values = torch.tensor([-1.0, -0.5, 0.0, 0.5, 1.0])
    case.h = (3 * values[torch.randint(0, 5, (tokens, width), generator=gen)]).to(DTYPES[dtype])     # logits are multiples of 3/4 of up to 192
    case.weight = values[torch.randint(0, 5, (vocab, width), generator=gen)].to(DTYPES[dtype])
    case.logits = torch.randint(-2, 3, (tokens, k), generator=gen).float()
    z = case.h.double() @ case.weight.double().t()
    case.ids[:, 0] = z.argmax(1)                                                                     # the word that is learned, and two others
    case.ids[:, 1:] = torch.where(case.ids[:, 1:] == case.ids[:, :1], (case.ids[:, :1] + 1) % vocab, case.ids[:, 1:])
    case.run(loss, dh=dh, dweight=dweight)

    log_q = torch.log_softmax(case.logits.double() / temperature, 1)
    q, top = log_q.exp(), z.amax(1, keepdim=True)
    down = (top - z) / temperature                                                                   # how far below the largest, over the temperature
    e = (-down).exp()
    log_total = e.sum(1, keepdim=True).log()
    terms = torch.where(q > 0, q * (log_q + down.gather(1, case.ids) + log_total), 0.0)
    weight = case.dloss.double()[:, None] / temperature
    p = e / e.sum(1, keepdim=True)
    onto = torch.zeros_like(p).scatter_add_(1, case.ids, q)
    g = (p - onto) * weight
    want = {"loss": terms.sum(1), "lse": (top / temperature + log_total)[:, 0], "dh": g @ case.weight.double(), "dweight": g.t() @ case.h.double()}
    # of p: its exponential's argument (a difference that is exact, by a number and a scale that are rounded), 15 added to it, the exponential, the
    # sum of all (each addition rounds it) and the division; of q the same with k of them
    of_p = (2 * down + 16 + 4 + 84 + vocab / 64 + 8) * U
    u = (case.logits.double().amax(1, keepdim=True) - case.logits.double()) / temperature
    of_q = (2 * u + 32 + 4 * k) * U
    of_log = (84 + vocab / 64 + 8) * U
    size = q * (2 * u + log_q.abs() + 3 * down.gather(1, case.ids) + log_total)
    off = {"loss": torch.where(q > 0, of_q * q * (log_q + down.gather(1, case.ids) + log_total).abs() + 8 * U * size + of_log * q, 0.0).sum(1) + 8 * U * want["loss"].abs(),
           "lse": of_log + 4 * U * want["lse"].abs()}
    of_g = weight.abs() * (of_p * p + 4 * U * (p + onto) + torch.zeros_like(p).scatter_add_(1, case.ids, of_q * q))
    if dtype == "bf16":
        of_g = of_g + 1.01 * (2.0 ** -11 * p + 2.0 ** -40) * weight.abs() + 1.01 * 2.0 ** -8 * g.abs()
    step = HALF_STEP[dtype]
    off["dh"] = of_g @ case.weight.double().abs() + (vocab + 2) * U * (g.abs() @ case.weight.double().abs()) + step * want["dh"].abs() + 1e-37
    off["dweight"] = of_g.t() @ case.h.double().abs() + (tokens + 2) * U * (g.abs().t() @ case.h.double().abs()) + step * want["dweight"].abs() + 1e-37
    for name, got in case.out.items():
        err = (got.double().cpu() - want[name]).abs()
        assert (err <= off[name]).all(), (name, float((err / off[name]).nan_to_num(torch.inf).max()), int((~(err <= off[name])).sum()))
