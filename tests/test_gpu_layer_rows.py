"""The norm's gradients where a workgroup has many rows, in the places of its inputs, and with rows that have no norm: against 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
EPS = 1e-5


@pytest.fixture(scope="module")
def layer():
    from paper_2505_23949_amd import layer as module

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return module


def backward(layer, h, gain, dy, dsum, dh=None):
    dh = torch.empty_like(h) if dh is None else dh
    dgain = torch.empty(h.shape[1], device="cuda")
    p = layer.make_norm_backward(h, gain, EPS, dy, dh=dh, dgain=dgain, dsum=dsum)
    layer.tsenor_norm_backward(p, torch.empty(layer.tsenor_norm_backward_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255))
    return dh, dgain


# More rows than workgroups (2^20 / cols of them, 256 at least; 1024 / (cols / 2048) above 16384 columns), so that each takes several, an
# odd number some of them; every width of workgroup, rows that begin and end anywhere.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(5003, 300), (3001, 1000), (1031, 1500), (1031, 2048), (1031, 4093), (777, 8190), (777, 16380), (701, 16500)])
def test_workgroups_of_many_rows(layer, rows, cols, dtype):
    gen = torch.Generator("cuda").manual_seed(rows + cols)

    def rand(*shape):
        return torch.randn(*shape, generator=gen, device="cuda").to(DTYPES[dtype])

    h, dy, past = rand(rows, cols), rand(rows, cols), rand(rows, cols)
    h *= 1 + torch.arange(rows, device="cuda")[:, None] % 7                 # (rows of other sizes: a row taken for another shows)
    gain = (1 + 0.3 * rand(cols)).float()
    x, d, g = h.double(), dy.double(), gain.double()
    c = 1.0 / torch.sqrt(x.square().mean(1, keepdim=True) + EPS)
    a = g * d
    along = (a * x).mean(1, keepdim=True)
    terms = c * a.abs() + x.abs() * c ** 3 * (a * x).abs().mean(1, keepdim=True)
    # an addition or product is 2^-24 off: cols / 512 + 40 of them in a row's sums and results, rows / 16 + 60 in a column's
    near = 2.0 ** -24 * (cols / 512 + 41) * terms
    sizes = (d * x * c).abs().sum(0)
    for dsum in (None, past):
        dh, dgain = backward(layer, h, gain, dy, dsum)
        want = c * a - x * c ** 3 * along + (0.0 if dsum is None else dsum.double())
        assert ((dh.double() - want).abs() <= near + HALF_ULP[dtype] * want.abs() * 1.01 + 1e-38).all()
        assert ((dgain.double() - (d * x * c).sum(0)).abs() <= 2.0 ** -24 * (rows / 16 + cols / 512 + 60) * sizes).all()
        # in the place of dy, and of dsum: the same bits
        place = dy.clone()
        again, again_gain = backward(layer, h, gain, place, dsum, dh=place)
        assert torch.equal(again, dh) and torch.equal(again_gain, dgain)
        if dsum is not None:
            place = dsum.clone()
            again, again_gain = backward(layer, h, gain, dy, place, dh=place)
            assert torch.equal(again, dh) and torch.equal(again_gain, dgain)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [200, 700, 4096, 9000, 17000])
def test_gradients_of_rows_without_a_norm(layer, cols, dtype):
    gen = torch.Generator("cuda").manual_seed(cols)
    rows = 9
    h, dy = (torch.randn(rows, cols, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    gain = torch.ones(cols, device="cuda")
    clean, clean_gain = backward(layer, h, gain, dy, None)
    h[2] = 0.0                                                              # c = eps^-1/2, and no second term
    with_zero, zero_gain = backward(layer, h, gain, dy, None)
    want = dy[2].double() / math.sqrt(EPS)
    assert ((with_zero[2].double() - want).abs() <= (HALF_ULP[dtype] * 1.01 + 2.0 ** -22) * want.abs()).all()
    others = [k for k in range(rows) if k != 2]
    assert torch.equal(with_zero[others], clean[others]) and torch.isfinite(zero_gain).all()
    # NaN: the row's gradients are, and every column's sum over the rows; infinity: its c is 0, so only its own column's
    for value, bad_columns in ((math.nan, cols), (math.inf, 1)):
        one = h.clone()
        one[5, 7] = value
        got, got_gain = backward(layer, one, gain, dy, None)
        others = [k for k in range(rows) if k != 5]
        assert torch.isnan(got[5]).all() and torch.equal(got[others], with_zero[others])
        assert int(torch.isnan(got_gain).sum()) == bad_columns and bool(torch.isnan(got_gain[7]))
    # a gradient that is not finite stays in its row and, in dgain, in its column
    for value in (math.nan, math.inf):
        one = dy.clone()
        one[5, 7] = value
        got, got_gain = backward(layer, h, gain, one, None)
        assert not torch.isfinite(got[5]).any() and torch.equal(got[others], with_zero[others])
        assert not torch.isfinite(got_gain[7]) and torch.isfinite(got_gain).sum() == cols - 1
