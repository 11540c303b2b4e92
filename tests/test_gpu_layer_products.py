"""Products of small whole numbers, which single precision sums exactly, through every kernel that tsenor_product chooses from; and how far
the sums of ordinary operands are off."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

# rows of a, rows of b, columns, and the kernels that they are given to, launch by launch ("+": workgroups share the columns of a tile).
# Rows and columns are ragged in every kernel, and its blocks of 128 columns fewer than its buffers, as many, and many more.
PRODUCTS = [
    (1, 300, 4100, ("few",)), (3, 300, 1500, ("few",)), (7, 5000, 9100, ("few",)), (12, 4090, 4100, ("few",)), (13, 70, 2100, ("few",)),
    (16, 1000, 8200, ("few",)),
    (9, 131, 171, ("small",)), (999, 2003, 5000, ("small",)), (40, 300, 4100, ("small+",)), (17, 66, 990, ("small+",)),
    (8450, 133, 100, ("tile",)), (8450, 133, 300, ("tile",)), (8930, 133, 621, ("tile",)), (1001, 3001, 3000, ("tile",)),
    (1027, 2050, 14300, ("tile",)),
    (260, 11287, 121, ("pairs",)), (11110, 264, 491, ("pairs",)), (2327, 6543, 1413, ("pairs",)),
    (1999, 4093, 2500, ("wide",)), (1999, 4093, 14331, ("wide",)),
    (1155, 12783, 122, ("large",)), (9883, 1434, 205, ("large",)), (1000, 16001, 2001, ("large",)),
    (4096, 14331, 4096, ("large", "wide")), (14331, 4093, 2500, ("large", "wide")), (4097, 8200, 9000, ("large", "tile")),
    (8200, 4097, 9000, ("large", "tile")), (5001, 5003, 3900, ("large", "pairs")), (4200, 4300, 4000, ("large", "small")),
]


@pytest.fixture(scope="module")
def layer():
    from paper_2505_23949_amd import layer as module

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return module


def scaled_from(layer, x, square=False):
    q = layer.empty_scaled(*x.shape, "cuda")
    layer.tsenor_quantize(layer.make_quantize(x, out=q, square=square))
    return q


def product(layer, a, b, out, mask=None):
    p = layer.make_product(a, b, out=out, mask=mask)
    work = torch.empty(layer.tsenor_product_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)
    layer.tsenor_product(p, work)
    return out


@pytest.mark.parametrize("m,n,k,kinds", PRODUCTS)
def test_small_whole_numbers_through_every_kernel(layer, m, n, k, kinds):
    gen = torch.Generator("cuda").manual_seed(m + n + k)
    a = torch.randint(-4, 5, (m, k), generator=gen, device="cuda").float()
    b = torch.randint(-4, 5, (n, k), generator=gen, device="cuda").float() * 0.5
    a *= torch.exp2(torch.randint(-1, 2, (m, 1), generator=gen, device="cuda").float())   # scales that differ from row to row
    b *= torch.exp2(torch.randint(-1, 2, (n, 1), generator=gen, device="cuda").float())
    # (halves times quarters of whole numbers, at most 8 * 4 each: sums of 2^14 are below 2^19, in eighths 2^22: exact in single precision)
    want = (a @ b.t()).bfloat16()
    qa, qb = scaled_from(layer, a), scaled_from(layer, b)
    got = product(layer, qa, qb, torch.empty(m, n, dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(got, want)
    mask = (torch.rand(m, n, generator=gen, device="cuda") > 0.25).to(torch.uint8)
    wide = torch.full((m, n + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    product(layer, qa, qb, wide[:, 3:3 + n], mask)
    assert torch.equal(wide[:, 3:3 + n], torch.where(mask != 0, want, torch.zeros_like(want)))
    assert (wide[:, :3] == 7).all() and (wide[:, 3 + n:] == 7).all()


@pytest.mark.parametrize("m,n,k", [(5, 4096, 4096), (48, 4096, 2500), (600, 1500, 8192), (1999, 4093, 2500), (1000, 16001, 500)])
def test_sums_of_ordinary_operands(layer, m, n, k):
    # The header: results of normal operands are 1.6e-5 (of their rms R) off before they are rounded.  That moves a result over the middle
    # between two bf16 values, s <= 2^-7 |v| apart, with probability |error| / s, which costs s^2: on average |error| s <=
    # 1.3e-5 R * 2^-7 * 0.8 R = 8.1e-8 R^2, 2.8e-4 R.  An error of twice the size is 4e-4.
    gen = torch.Generator("cuda").manual_seed(m + n + k)
    qa = scaled_from(layer, torch.randn(m, k, generator=gen, device="cuda"))
    qb = scaled_from(layer, torch.randn(n, k, generator=gen, device="cuda"), square=True)
    got = product(layer, qa, qb, torch.empty(m, n, dtype=torch.bfloat16, device="cuda"))
    exact = qa.dequantize().double() @ qb.dequantize().double().t()
    size = float(exact.norm())
    assert float((got.double() - exact.bfloat16().double()).norm()) <= 4e-4 * size
    # and a result is the nearest bf16 value or, where the sum's error took it over the middle, one that much farther: 2^-8 of it and 40 rms errors
    assert float(((got.double() - exact).abs() - 2.0 ** -8 * exact.abs()).max()) <= 40 * 1.6e-5 * size / math.sqrt(m * n)
    # the same bits again
    assert torch.equal(product(layer, qa, qb, torch.empty_like(got)), got)
