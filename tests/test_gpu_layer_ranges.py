"""The layer operators where intermediate results could leave the range of single precision though the formula's do not, and with more
tensors than a launch of clipping takes: against 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def layer():
    from paper_2505_23949_amd import layer as module

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return module


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, dtype=torch.float64)


# ---- norm ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size,eps", [(1e15, 1e-5), (1e17, 1e-5), (1e-14, 0.0), (1e-17, 0.0)])
@pytest.mark.parametrize("rows,cols", [(5, 300), (3, 4096), (2, 16000), (3, 17000)])
def test_norm_backward_of_large_and_small_rows(layer, rows, cols, size, eps, dtype):
    gen = torch.Generator().manual_seed(rows + cols)
    unit = rand(gen, rows, cols)
    h = (size * unit).to(DTYPES[dtype]).cuda()
    dy = (unit + 0.5 * rand(gen, rows, cols)).to(DTYPES[dtype]).cuda()      # (along h, so that the second term is as large as the first)
    gain = (1 + 0.3 * rand(gen, cols)).float().cuda()
    dh, dgain = torch.empty_like(h), torch.empty(cols, device="cuda")
    p = layer.make_norm_backward(h, gain, eps, dy, dh=dh, dgain=dgain)
    layer.tsenor_norm_backward(p, torch.empty(layer.tsenor_norm_backward_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    x, g, d = h.cpu().double(), gain.cpu().double(), dy.cpu().double()
    c = 1.0 / torch.sqrt(x.square().mean(1, keepdim=True) + eps)
    a = g * d
    want = c * a - x * c ** 3 * (a * x).mean(1, keepdim=True)
    # rounding errors as at any other size: 2^-24 of the sizes of the terms for each of the additions in a row and the few products
    terms = c * a.abs() + x.abs() * c ** 3 * (a * x).abs().mean(1, keepdim=True)
    near = 2.0 ** -24 * (cols / 512 + 41) * terms
    assert ((dh.cpu().double() - want).abs() <= near + HALF_ULP[dtype] * want.abs() * 1.01).all()
    sizes = (d * x * c).abs().sum(0)
    assert ((dgain.cpu().double() - (d * x * c).sum(0)).abs() <= 2.0 ** -24 * (rows / 16 + cols / 512 + 60) * sizes).all()


@pytest.mark.parametrize("size,gain_size,eps", [(1e18, 1e26, 1e-5), (1e-17, 1e-25, 0.0)])
@pytest.mark.parametrize("rows,cols", [(4, 200), (2, 5000), (2, 17000)])
def test_norm_of_large_and_small_rows_and_gains(layer, rows, cols, size, gain_size, eps):
    gen = torch.Generator().manual_seed(cols)
    size = size / math.sqrt(cols)                            # (the sum of squares stays in range)
    x = (size * rand(gen, rows, cols)).float().cuda()
    gain = (gain_size * (1 + 0.3 * rand(gen, cols))).float().cuda()
    y, q = torch.empty_like(x), layer.empty_scaled(rows, cols, "cuda")
    layer.tsenor_norm(layer.make_norm(x, gain, eps, y_out=y, out=q))
    h = x.cpu().double()
    want = h / torch.sqrt(h.square().mean(1, keepdim=True) + eps) * gain.cpu().double()
    near = 2.0 ** -24 * (cols / 512 + 32) * want.abs()
    assert ((y.cpu().double() - want).abs() <= near + HALF_ULP["f32"] * want.abs() * 1.01).all()


# ---- clipping -----------------------------------------------------------------------------------------------------------

def clip(layer, grads, largest):
    norm = torch.empty(2, device="cuda")
    p = layer.make_clip(grads, largest, norm_out=norm)
    layer.tsenor_clip(p, torch.empty(layer.tsenor_clip_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255))
    return norm.cpu().double()


def test_a_norm_beyond_single_precision_leaves_the_gradients(layer):
    # finite in double, infinite where it is reported: the caller is told to drop the step, and finds the gradients as they were
    g = torch.full((5,), 3e38, device="cuda")
    kept = g.clone()
    assert clip(layer, [g], 1.0).tolist() == [math.inf, 1.0] and torch.equal(g, kept)


def test_factors_below_the_normal_numbers(layer):
    # the factor is 5e-43 (357 steps of the smallest number), the results 5e-5: as exact as any others
    for dtype in ("f32", "bf16"):
        g = (1e38 * torch.tensor([1.0, -1.1, 0.9, 0.7])).to(DTYPES[dtype]).cuda()
        wide = g.cpu().double()
        norm = float(wide.norm())
        got = clip(layer, [g], 1e-4)
        assert abs(got[0] - norm) <= 1e-7 * norm and abs(got[1] - 1e-4 / norm) <= 2.0 ** -149
        want = wide * (1e-4 / norm)
        assert ((g.cpu().double() - want).abs() <= (HALF_ULP[dtype] * 1.01 + 2.0 ** -23) * want.abs()).all()


def test_clip_of_many_tensors_in_launches_of_all_sizes(layer):
    # launches of few and of many chunks in turn, so that the later ones add to the sums of some workgroups and begin those of others
    gen = torch.Generator("cuda").manual_seed(2)
    sizes = [7] * 250 + [5_000_000, 4097] + [3] * 500 + [9_000_001] * 2 + [64] * 181 + [4096] * 1000
    grads = [torch.randn(n, device="cuda", generator=gen).to(torch.bfloat16 if k % 3 else torch.float32) for k, n in enumerate(sizes)]
    before = [g.clone() for g in grads]
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    got = clip(layer, grads, 0.25 * norm)
    assert abs(got[0] - norm) <= 1e-7 * norm and abs(got[1] - 0.25) <= 1e-7
    factor = float(got[1])
    for g, b in zip(grads, before):
        assert torch.equal(g, (b.float() * factor).to(g.dtype))
    # the same bits again
    again = [b.clone() for b in before]
    assert torch.equal(clip(layer, again, 0.25 * norm), got)
