"""The layer operators (tsenor_layer.h) against plain 64-bit implementations on the CPU."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # of 24 and 8 bits
EPS = 1e-5


@pytest.fixture(scope="module")
def layer():
    from paper_2505_23949_amd import layer as module

    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return module


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, dtype=torch.float64)


def on_gpu(x, dtype, ld=None, offset=0):
    """x as a GPU tensor of `dtype`; with ld, as a column range of a wider matrix filled with NaN."""
    x = x.to(DTYPES[dtype])
    if ld is None:
        return x.cuda()
    wide = torch.full((x.shape[0], ld), math.nan, dtype=x.dtype)
    wide[:, offset:offset + x.shape[1]] = x
    return wide.cuda()[:, offset:offset + x.shape[1]]


# ---- the 8-bit format in 64 bits ----------------------------------------------------------------------------------------

def nearest_8bit(v):
    """v (double) to the nearest e4m3 value, ties to even; NaN for what is not finite."""
    size = v.abs()
    exponent = torch.floor(torch.log2(torch.clamp(size, min=2.0 ** -6)))
    step = torch.exp2(exponent - 3)
    q = torch.copysign(torch.round(size / step) * step, v)
    return torch.where(torch.isfinite(v), q, torch.full_like(v, math.nan))


def reference_scales(x, square):
    """(blocks, rows) exponents of the scales of x (double)."""
    rows, cols = x.shape
    out = torch.zeros(-(-cols // 128), rows, dtype=torch.float64)
    for r0 in range(0, rows, 128 if square else 1):
        for k in range(out.shape[0]):
            part = x[r0:r0 + (128 if square else 1), k * 128:(k + 1) * 128]
            largest = part[torch.isfinite(part)].abs().max().item() if torch.isfinite(part).any() else 0.0
            e = 0
            if largest > 0:
                e = max(-126, math.frexp(largest / 448.0)[1])
                if e > -126 and largest <= 448.0 * 2.0 ** (e - 1):
                    e -= 1
            out[k, r0:r0 + (128 if square else 1)] = e
    return out


def parts(q):
    """(values of the columns as doubles, padding, exponents of the scales) of a ScaledMatrix."""
    wide = q.values.float().cpu().double()
    return wide[:, :q.cols], wide[:, q.cols:-(-q.cols // 128) * 128], q.scales[:, :q.rows].view(torch.uint8).cpu().double() - 127


def check_quantized(q, x, square):
    values, padding, exponents = parts(q)
    want = reference_scales(x, square)
    assert torch.equal(exponents, want)
    expected = nearest_8bit(x * torch.exp2(-want.t().repeat_interleave(128, 1)[:, :x.shape[1]]))
    assert torch.equal(torch.isnan(values), torch.isnan(expected))
    assert torch.equal(values.nan_to_num(), expected.nan_to_num())
    assert torch.equal(padding, torch.zeros_like(padding))


# ---- quantisation -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("rows,cols,ld", [(1, 1, None), (1, 128, None), (3, 129, None), (127, 5, 9), (128, 128, None), (130, 257, 264),
                                          (257, 640, None), (64, 1000, 1003)])
def test_quantize(layer, dtype, square, rows, cols, ld):
    gen = torch.Generator().manual_seed(rows * 1000 + cols)
    x = rand(gen, rows, cols) * torch.exp2(6 * rand(gen, rows, 1)) * torch.exp2(3 * rand(gen, 1, cols))
    x[rand(gen, rows, cols) > 1.5] = 0.0
    g = on_gpu(x, dtype, ld, 1 if ld and ld % 8 else 0)
    mask = (rand(gen, rows, cols) > 0).to(torch.uint8)
    for m in (None, mask):
        q, qt = layer.empty_scaled(rows, cols, "cuda"), layer.empty_scaled(cols, rows, "cuda")
        layer.tsenor_quantize(layer.make_quantize(g, out=q, out_t=qt, mask=None if m is None else m.cuda(), square=square))
        stored = g.cpu().double() if m is None else torch.where(m != 0, g.cpu().double(), 0.0)
        check_quantized(q, stored, square)
        check_quantized(qt, stored.t(), square)
        # either alone gives the same bytes
        for way, whole in (("out", q), ("out_t", qt)):
            one = layer.empty_scaled(whole.rows, whole.cols, "cuda")
            layer.tsenor_quantize(layer.make_quantize(g, **{way: one}, mask=None if m is None else m.cuda(), square=square))
            assert all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(parts(one), parts(whole)))


@pytest.mark.parametrize("square", [False, True])
def test_quantize_of_values_at_the_ends(layer, square):
    gen = torch.Generator().manual_seed(5)
    x = rand(gen, 140, 300)
    x[0, :128] = 0.0                                    # a block without a value
    x[1, :128] = math.inf                               # one without a finite value
    x[2, 3], x[2, 130], x[3, 200] = math.nan, -math.inf, math.inf
    x[4, 0] = 448.0 * 2.0 ** 5                          # a maximum that fits exactly, and ones just above
    x[5, 0] = 448.0 * 2.0 ** 5 * (1 + 2.0 ** -23)
    x[6, 0] = 3.4e38
    x[7, :128] = 2.0 ** -149 * torch.arange(128)        # subnormal singles
    x[8, :128] = 2.0 ** -126
    x[9, :128] = torch.arange(128) + 0.5                # ties
    x[10, 0] = -448.0
    x[11, :128] = -0.0
    g = on_gpu(x, "f32")
    x = g.cpu().double()
    for m in (None, (torch.isfinite(x) & (rand(gen, 140, 300) > -1)).to(torch.uint8)):
        q, qt = layer.empty_scaled(140, 300, "cuda"), layer.empty_scaled(300, 140, "cuda")
        layer.tsenor_quantize(layer.make_quantize(g, out=q, out_t=qt, mask=None if m is None else m.cuda(), square=square))
        stored = x if m is None else torch.where(m != 0, x, 0.0)
        check_quantized(q, stored, square)
        check_quantized(qt, stored.t(), square)
    # a mask that leaves nothing
    q = layer.empty_scaled(140, 300, "cuda")
    layer.tsenor_quantize(layer.make_quantize(g, out=q, mask=torch.zeros(140, 300, dtype=torch.uint8, device="cuda"), square=square))
    values, _, exponents = parts(q)
    assert not values.any() and not exponents.any()


# ---- norm ---------------------------------------------------------------------------------------------------------------

SHAPES = [(1, 1), (5, 7), (3, 128), (9, 500), (2, 513), (7, 1000), (4, 2048), (3, 2500), (2, 4096), (3, 5001), (2, 8192), (2, 16384), (3, 16385),
          (1, 40000), (33, 300)]


@pytest.mark.parametrize("dtype,gain_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm(layer, dtype, gain_dtype, rows, cols):
    gen = torch.Generator().manual_seed(rows + cols)
    odd = cols % 2 == 1                                     # rows that begin anywhere
    x = on_gpu(rand(gen, rows, cols) * 3, dtype, cols + 3 if odd else None, 1)
    r = on_gpu(rand(gen, rows, cols), dtype, cols + 8 if odd else None, 8)
    gain = on_gpu(1 + 0.3 * rand(gen, cols), gain_dtype)
    for residual in (None, r):
        q = layer.empty_scaled(rows, cols, "cuda")
        total, y = torch.empty(rows, cols, dtype=x.dtype, device="cuda"), torch.empty(rows, cols, dtype=x.dtype, device="cuda")
        layer.tsenor_norm(layer.make_norm(x, gain, EPS, residual=residual, out=q, sum_out=total, y_out=y))
        h = x.cpu().float() if residual is None else x.cpu().float() + r.cpu().float()
        assert torch.equal(total.cpu(), h.to(x.dtype))
        h = total.cpu().double()
        want = h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS) * gain.cpu().double()
        # the sum of squares: at most cols / threads / 8 + 20 additions in a row, each 2^-24; root, quotient and products: 6
        near = 2.0 ** -24 * (cols / 512 + 32) * want.abs()
        assert ((y.cpu().double() - want).abs() <= near + HALF_ULP[dtype] * want.abs() * 1.01 + 1e-38).all()
        values, padding, exponents = parts(q)
        scale = torch.exp2(exponents).t().repeat_interleave(128, 1)[:, :cols]
        # the nearest 8-bit value: 2^-4 of the value away at most, or half a step of the smallest, 2^-10
        assert ((values * scale - want).abs() <= near * 1.1 + torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * scale)).all()
        for k in range(exponents.shape[0]):
            largest = want[:, k * 128:(k + 1) * 128].abs().amax(1)
            s = torch.exp2(exponents[k])
            assert (largest <= 448 * s * (1 + 1e-5)).all() and ((largest > 224 * s * (1 - 1e-5)) | (largest == 0)).all()
        assert not padding.any()
        # each output alone: the same bits; the sum in the residual's place
        alone = layer.empty_scaled(rows, cols, "cuda")
        layer.tsenor_norm(layer.make_norm(x, gain, EPS, residual=residual, out=alone))
        assert all(torch.equal(a, b) for a, b in zip(parts(alone), parts(q)))
        if residual is not None:
            place = residual.contiguous().clone()
            only = torch.empty_like(y)
            layer.tsenor_norm(layer.make_norm(x, gain, EPS, residual=place, sum_out=place, y_out=only))
            assert torch.equal(place, total) and torch.equal(only, y)


def test_norm_of_rows_without_a_norm(layer):
    x = torch.randn(6, 700, device="cuda")
    x[0] = 0.0
    x[1, 5] = math.nan
    x[2, 5] = math.inf
    x[3] *= 1e-30
    gain = torch.ones(700, device="cuda")
    q, y = layer.empty_scaled(6, 700, "cuda"), torch.empty_like(x)
    layer.tsenor_norm(layer.make_norm(x, gain, EPS, out=q, y_out=y))
    values, _, exponents = parts(q)
    assert not y[0].any() and not values[0].any() and not exponents[:, 0].any()
    assert torch.isnan(y[1]).all() and torch.isnan(values[1]).all() and not exponents[:, 1].any()
    assert torch.isnan(y[2, 5]) and (y[2].nan_to_num() == 0).all()
    assert torch.isfinite(y[3:]).all() and torch.isfinite(values[3:]).all()
    # no eps and no values: 0 / 0
    layer.tsenor_norm(layer.make_norm(x, gain, 0.0, y_out=y))
    assert torch.isnan(y[0]).all()


def norm_gradients(h, gain, dy, dsum):
    c = 1.0 / torch.sqrt(h.square().mean(1, keepdim=True) + EPS)
    a = gain * dy
    dh = c * a - h * c ** 3 * (a * h).mean(1, keepdim=True)
    return (dh if dsum is None else dh + dsum), (dy * h * c).sum(0)


def test_the_formula_of_the_gradients_against_differences():
    gen = torch.Generator().manual_seed(1)
    h, gain, dy, dsum = rand(gen, 4, 9), 1 + 0.3 * rand(gen, 9), rand(gen, 4, 9), rand(gen, 4, 9)

    def loss(h, gain):
        return float((h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS) * gain * dy).sum() + (h * dsum).sum())

    dh, dgain = norm_gradients(h, gain, dy, dsum)
    step = 1e-6
    for i in range(4):
        for j in range(9):
            d = torch.zeros_like(h)
            d[i, j] = step
            assert abs((loss(h + d, gain) - loss(h - d, gain)) / (2 * step) - dh[i, j]) < 1e-8
    for j in range(9):
        d = torch.zeros_like(gain)
        d[j] = step
        assert abs((loss(h, gain + d) - loss(h, gain - d)) / (2 * step) - dgain[j]) < 1e-8


@pytest.mark.parametrize("dtype,gain_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,cols", SHAPES + [(700, 260), (1025, 600), (600, 17000)])
def test_norm_backward(layer, dtype, gain_dtype, rows, cols):
    gen = torch.Generator().manual_seed(rows * 3 + cols)
    odd = cols % 2 == 1
    h = on_gpu(rand(gen, rows, cols) * 3, dtype, cols + 3 if odd else None, 1)
    dy = on_gpu(rand(gen, rows, cols), dtype, cols + 5 if odd else None, 2)
    past = on_gpu(rand(gen, rows, cols), dtype, cols + 8 if odd else None, 8)
    gain = on_gpu(1 + 0.3 * rand(gen, cols), gain_dtype)
    wide = [t.cpu().double() for t in (h, gain, dy)]
    for dsum in (None, past):
        dh, dgain = torch.empty(rows, cols, dtype=h.dtype, device="cuda"), torch.empty(cols, device="cuda")
        p = layer.make_norm_backward(h, gain, EPS, dy, dh=dh, dgain=dgain, dsum=dsum)
        work = torch.empty(layer.tsenor_norm_backward_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)
        layer.tsenor_norm_backward(p, work)
        want, want_gain = norm_gradients(*wide, None if dsum is None else dsum.cpu().double())
        c = 1.0 / torch.sqrt(wide[0].square().mean(1, keepdim=True) + EPS)
        # sums over the row as above, of terms that may cancel: 2^-24 of the sum of their sizes
        terms = c * (wide[1] * wide[2]).abs() + wide[0].abs() * c ** 3 * (wide[1] * wide[2] * wide[0]).abs().mean(1, keepdim=True)
        near = 2.0 ** -24 * (cols / 512 + 40) * terms
        assert ((dh.cpu().double() - want).abs() <= near + HALF_ULP[dtype] * want.abs() * 1.01 + 2.0 ** -24 * terms + 1e-38).all()
        sizes = (wide[2] * wide[0] * c).abs().sum(0)
        assert ((dgain.cpu().double() - want_gain).abs() <= 2.0 ** -24 * (rows / 16 + cols / 512 + 60) * sizes + 1e-38).all()
        # again, and in dy's place: the same bits
        again, place = torch.empty_like(dgain), dy.contiguous().clone()
        p = layer.make_norm_backward(h, gain, EPS, place, dh=place, dgain=again, dsum=dsum)
        layer.tsenor_norm_backward(p, work)
        assert torch.equal(place, dh) and torch.equal(again, dgain)


# ---- product ------------------------------------------------------------------------------------------------------------

def scaled_from(layer, x, square=False):
    q = layer.empty_scaled(*x.shape, "cuda")
    layer.tsenor_quantize(layer.make_quantize(x.float().cuda(), out=q, square=square))
    return q


def product(layer, a, b, out, mask=None):
    p = layer.make_product(a, b, out=out, mask=mask)
    work = torch.empty(layer.tsenor_product_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)
    layer.tsenor_product(p, work)
    return out


PRODUCTS = [(1, 1, 1), (1, 130, 128), (2, 16, 129), (16, 100, 256), (17, 513, 384), (1, 4096, 512), (33, 260, 1000), (48, 300, 2200), (64, 64, 64),
            (65, 70, 140), (100, 129, 640), (127, 255, 1024), (129, 128, 100), (200, 520, 3500), (256, 256, 256), (257, 300, 500), (300, 1000, 130),
            (520, 260, 2049), (1000, 770, 384), (128, 200, 9000), (12, 5000, 260), (2000, 4001, 300), (4000, 4010, 260)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product_of_small_whole_numbers(layer, m, n, k):
    # products and sums that single precision holds exactly: only the rounding to bf16 is left, and that is known
    gen = torch.Generator().manual_seed(m + n + k)
    a = torch.randint(-4, 5, (m, k), generator=gen).double() * torch.exp2(torch.randint(-1, 2, (m, 1), generator=gen).double())
    b = torch.randint(-4, 5, (n, k), generator=gen).double() * torch.exp2(torch.randint(-1, 2, (n, 1), generator=gen).double())
    want = a @ b.t()
    qa, qb = scaled_from(layer, a), scaled_from(layer, b)
    got = product(layer, qa, qb, torch.empty(m, n, dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(got.cpu(), want.to(torch.bfloat16))
    # a mask, into a column range of a wider matrix that begins anywhere
    mask = (torch.rand(m, n, generator=gen) > 0.5).to(torch.uint8)
    wide = torch.full((m, n + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    product(layer, qa, qb, wide[:, 3:3 + n], mask.cuda())
    assert torch.equal(wide[:, 3:3 + n].cpu(), torch.where(mask != 0, want, 0.0).to(torch.bfloat16))
    assert (wide[:, :3] == 7).all() and (wide[:, 3 + n:] == 7).all()


@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(layer, m, n, k, square):
    gen = torch.Generator().manual_seed(m * 7 + n + k)
    qa = scaled_from(layer, rand(gen, m, k) * torch.exp2(2 * rand(gen, 1, k)))
    qb = scaled_from(layer, rand(gen, n, k) * torch.exp2(2 * rand(gen, n, 1)), square)
    a, b = qa.dequantize().cpu().double(), qb.dequantize().cpu().double()
    want, sizes = a @ b.t(), a.abs() @ b.abs().t()
    got = product(layer, qa, qb, torch.empty(m, n, dtype=torch.bfloat16, device="cuda")).cpu().double()
    # the products of a group keep 16 bits below the largest of them; 2^-12 of all sizes is far more than that loses
    assert ((got - want).abs() <= HALF_ULP["bf16"] * 1.01 * want.abs() + 2.0 ** -12 * sizes).all()
    assert (got - want).norm() <= 2.5e-3 * want.norm() + 2.0 ** -14 * sizes.norm()


# enough tiles that the last round of them is left to a launch of its own, by rows of a or of b
@pytest.mark.parametrize("m,n,k", [(4096, 14336, 640), (9001, 4100, 2500), (4100, 9001, 2500), (5001, 5003, 3900), (4200, 4300, 4000)])
def test_large_product_of_small_whole_numbers(layer, m, n, k):
    gen = torch.Generator("cuda").manual_seed(m + n + k)
    a = torch.randint(-4, 5, (m, k), generator=gen, device="cuda").float()
    b = torch.randint(-4, 5, (n, k), generator=gen, device="cuda").float() * 0.5
    qa, qb = scaled_from(layer, a), scaled_from(layer, b)
    mask = (torch.rand(m, n, generator=gen, device="cuda") > 0.25).to(torch.uint8)
    wide = torch.full((m, n + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    product(layer, qa, qb, wide[:, 3:3 + n], mask)
    want = (a @ b.t()).bfloat16() * mask                 # (halves of whole numbers below 2^18: sums in single precision are exact)
    assert torch.equal(wide[:, 3:3 + n], want)
    assert (wide[:, :3] == 7).all() and (wide[:, 3 + n:] == 7).all()


def test_product_without_columns_is_zero(layer):
    a, b = layer.empty_scaled(5, 0, "cuda"), layer.empty_scaled(9, 0, "cuda")
    assert not product(layer, a, b, torch.full((5, 9), 3.0, dtype=torch.bfloat16, device="cuda")).any()


def test_large_product_without_columns_is_zero(layer):
    a, b = layer.empty_scaled(300, 0, "cuda"), layer.empty_scaled(500, 0, "cuda")
    wide = torch.full((300, 503), 3.0, dtype=torch.bfloat16, device="cuda")
    product(layer, a, b, wide[:, 2:502])
    assert not wide[:, 2:502].any() and (wide[:, :2] == 3).all() and (wide[:, 502:] == 3).all()


def test_product_keeps_infinite_and_undefined_rows_apart(layer):
    gen = torch.Generator().manual_seed(3)
    x = rand(gen, 70, 300)
    x[3, 5], x[40, 299] = math.nan, math.inf
    qa, qb = scaled_from(layer, x), scaled_from(layer, rand(gen, 90, 300))
    got = product(layer, qa, qb, torch.empty(70, 90, dtype=torch.bfloat16, device="cuda"))
    bad = torch.isnan(got).all(1)
    assert bad.nonzero().flatten().tolist() == [3, 40] and torch.isfinite(got[~bad]).all()
    # dropped by the mask they are 0
    mask = torch.ones(70, 90, dtype=torch.uint8, device="cuda")
    mask[3], mask[40] = 0, 0
    got = product(layer, qa, qb, got, mask)
    assert torch.isfinite(got).all() and not got[3].any() and not got[40].any()


# ---- gradient clipping ----------------------------------------------------------------------------------------------------

def clip(layer, grads, largest, out=None):
    norm = torch.empty(2, device="cuda")
    p = layer.make_clip(grads, largest, out=out, norm_out=norm)
    work = torch.empty(layer.tsenor_clip_workspace_bytes(p), dtype=torch.uint8, device="cuda").fill_(255)
    layer.tsenor_clip(p, work)
    return norm.cpu().double()


@pytest.mark.parametrize("sizes", [(1,), (0, 5, 0), (8192,), (8191, 8193, 3), (100000, 1, 40000, 0, 7), tuple(range(1, 240)), (3_000_001, 9_000_000)])
def test_clip(layer, sizes):
    gen = torch.Generator().manual_seed(len(sizes))
    wide = [rand(gen, n) * 10 for n in sizes]
    grads = []
    for k, g in enumerate(wide):  # types in turn, some of them at odd addresses
        shift = k % 3
        grads.append(torch.cat([torch.zeros(shift, dtype=torch.float64), g]).to(DTYPES["bf16" if k % 2 else "f32"]).cuda()[shift:])
    wide = [g.cpu().double() for g in grads]
    norm = math.sqrt(sum(float(g.square().sum()) for g in wide))
    for largest in (norm * 0.37, norm * 2, math.inf, 0.0):
        factor = largest / norm if norm > largest else 1.0
        out = [torch.full_like(g, 5.0) for g in grads]
        got = clip(layer, grads, largest, out)
        assert abs(got[0] - norm) <= 1e-7 * norm and abs(got[1] - factor) <= 1e-7 * factor
        for g, o in zip(wide, out):
            want = g * float(got[1])
            assert ((o.cpu().double() - want).abs() <= HALF_ULP["f32" if o.dtype == torch.float32 else "bf16"] * 1.01 * want.abs() + 1e-38).all()
        again = [g.clone() for g in grads]
        assert torch.equal(clip(layer, again, largest), got)
        assert all(torch.equal(a, o) for a, o in zip(again, out))


def test_clip_of_norms_that_are_not_finite_and_of_nothing(layer):
    assert clip(layer, [], 1.0).tolist() == [0.0, 1.0]
    assert clip(layer, [torch.empty(0, device="cuda"), torch.zeros(10, device="cuda")], 0.0).tolist() == [0.0, 1.0]
    for bad in (math.nan, math.inf):
        g = torch.randn(10000, device="cuda")
        g[77] = bad
        kept = g.clone()
        got = clip(layer, [g], 1.0)
        assert not math.isfinite(got[0]) and got[1] == 1.0 and torch.equal(g.nan_to_num(), kept.nan_to_num())
    # squares beyond single precision
    g = torch.full((1000,), 1e30, device="cuda")
    got = clip(layer, [g], 1.0)
    assert abs(got[0] / (1e30 * math.sqrt(1000)) - 1) < 1e-6 and abs(float(g.double().norm()) - 1) < 1e-6


# ---- no rows, and offsets beyond 32 bits ------------------------------------------------------------------------------------

def test_matrices_without_rows(layer):
    none, gain = torch.empty(0, 300, device="cuda"), torch.ones(300, device="cuda")
    q, qt = layer.empty_scaled(0, 300, "cuda"), layer.empty_scaled(300, 0, "cuda")
    layer.tsenor_quantize(layer.make_quantize(none, out=q, out_t=qt))
    layer.tsenor_norm(layer.make_norm(none, gain, EPS, residual=none, out=q, sum_out=none.clone(), y_out=none.clone()))
    dgain = torch.full((300,), 7.0, device="cuda")
    p = layer.make_norm_backward(none, gain, EPS, none, dh=none.clone(), dgain=dgain)
    layer.tsenor_norm_backward(p, torch.empty(max(1, layer.tsenor_norm_backward_workspace_bytes(p)), dtype=torch.uint8, device="cuda"))
    assert not dgain.any()
    w = scaled_from(layer, torch.randn(40, 300).double())
    product(layer, q, w, torch.empty(0, 40, dtype=torch.bfloat16, device="cuda"))
    product(layer, w, q, torch.empty(40, 0, dtype=torch.bfloat16, device="cuda"))
    # a weight gradient over no tokens
    got = product(layer, qt, layer.empty_scaled(50, 0, "cuda"), torch.full((300, 50), 3.0, dtype=torch.bfloat16, device="cuda"))
    assert not got.any()
    torch.cuda.synchronize()


def test_rows_far_apart(layer):
    gen = torch.Generator().manual_seed(9)
    ld = 2 ** 30 + 24                                    # three rows: offsets up to 2^32 bytes
    wide = torch.empty(3, ld, dtype=torch.bfloat16, device="cuda")
    x = wide[:, 11:311]
    x.copy_(rand(gen, 3, 300))
    q, qt = layer.empty_scaled(3, 300, "cuda"), layer.empty_scaled(300, 3, "cuda")
    layer.tsenor_quantize(layer.make_quantize(x, out=q, out_t=qt))
    check_quantized(q, x.cpu().double(), False)
    check_quantized(qt, x.cpu().double().t(), False)
    gain, y = torch.ones(300, device="cuda"), torch.empty(3, 300, dtype=torch.bfloat16, device="cuda")
    layer.tsenor_norm(layer.make_norm(x, gain, EPS, y_out=y))
    same = torch.empty_like(y)
    layer.tsenor_norm(layer.make_norm(x.contiguous(), gain, EPS, y_out=same))
    assert torch.equal(y, same)
    for m in (3, 200):                                   # results of one token, and of tiles
        q = scaled_from(layer, rand(gen, m, 300))
        w = scaled_from(layer, rand(gen, 100, 300))
        want = product(layer, q, w, torch.empty(m, 100, dtype=torch.bfloat16, device="cuda"))
        out = torch.empty(3 * ld, dtype=torch.bfloat16, device="cuda").as_strided((m, 100), (3 * ld // m, 1))
        assert torch.equal(product(layer, q, w, out), want)


@pytest.mark.parametrize("rows,cols", [(2 ** 26 + 5, 1), (2 ** 22 + 3, 1030)])
def test_more_rows_than_a_grid_has_threads_for(layer, rows, cols):
    gen = torch.Generator("cuda").manual_seed(rows)
    some = torch.randn(1009, cols, generator=gen, device="cuda").bfloat16()     # a row's number modulo a prime: shifted rows differ
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[:1009], at = some, 1009
    while at < rows:                                     # copies double
        x[at:2 * at] = x[:min(at, rows - at)]
        at *= 2
    whole = rows // 1009 * 1009
    gain = torch.ones(cols, device="cuda")
    y, q = torch.zeros_like(x), layer.empty_scaled(rows, cols, "cuda")
    layer.tsenor_norm(layer.make_norm(x, gain, EPS, y_out=y, out=q))
    want, want_q = torch.empty_like(some), layer.empty_scaled(1009, cols, "cuda")
    layer.tsenor_norm(layer.make_norm(some, gain, EPS, y_out=want, out=want_q))
    assert torch.equal(x[whole - 1009:whole], some)
    for first in (0, 2 ** 21 // 1009 * 1009, whole // 2 // 1009 * 1009, whole - 1009):
        assert torch.equal(y[first:first + 1009], want)
        assert torch.equal(q.values[first:first + 1009].view(torch.uint8), want_q.values.view(torch.uint8))
        assert torch.equal(q.scales.view(torch.uint8)[:, first:first + 1009], want_q.scales.view(torch.uint8)[:, :1009])
    assert torch.equal(y[whole:], want[:rows - whole])


def test_a_gradient_of_more_than_2_to_the_32_elements(layer):
    count = 2 ** 32 + 5000
    g = torch.full((count,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    got = clip(layer, [g], 1.0)
    norm = 2.0 ** -10 * math.sqrt(count)
    assert abs(got[0] - norm) <= 1e-7 * norm and abs(got[1] * norm - 1) <= 1e-6
    first = g[:1].clone()
    assert bool((g == first).all()) and abs(float(first) * 2 ** 10 * norm - 1) <= 2.0 ** -8


# ---- streams and graphs -----------------------------------------------------------------------------------------------------

def test_calls_on_another_stream_and_in_a_graph(layer):
    torch.manual_seed(0)
    x, r, gain = (torch.randn(40, 700, device="cuda").bfloat16() for _ in range(2)), None, torch.ones(700, device="cuda")
    x, r = x
    w = torch.randn(300, 700, device="cuda").bfloat16()
    wq, wt = layer.empty_scaled(300, 700, "cuda"), layer.empty_scaled(700, 300, "cuda")
    q, total, y = layer.empty_scaled(40, 700, "cuda"), torch.empty_like(x), torch.empty(40, 300, dtype=torch.bfloat16, device="cuda")
    dh, dgain = torch.empty_like(x), torch.empty(700, device="cuda")
    clipped, norm = torch.empty_like(dgain), torch.empty(2, device="cuda")
    calls = [(layer.tsenor_quantize, layer.make_quantize(w, out=wq, out_t=wt, square=True), None),
             (layer.tsenor_norm, layer.make_norm(x, gain, EPS, residual=r, out=q, sum_out=total), None),
             (layer.tsenor_product, layer.make_product(q, wq, out=y), layer.tsenor_product_workspace_bytes),
             (layer.tsenor_norm_backward, layer.make_norm_backward(total, gain, EPS, x, dh=dh, dgain=dgain),
              layer.tsenor_norm_backward_workspace_bytes),
             (layer.tsenor_clip, layer.make_clip([dgain], 0.5, out=[clipped], norm_out=norm), layer.tsenor_clip_workspace_bytes)]
    works = [None if size is None else torch.empty(max(256, size(p)), dtype=torch.uint8, device="cuda") for _, p, size in calls]

    def all_calls(stream=None):
        for (call, p, size), work in zip(calls, works):
            call(p, stream=stream) if size is None else call(p, work, stream=stream)

    results = (total, y, dh, dgain, clipped, norm)
    all_calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in results]
    side = torch.cuda.Stream()
    for t in results:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    all_calls(side)
    side.synchronize()
    assert all(torch.equal(t, v) for t, v in zip(results, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_calls()
    for turn in range(3):
        x.mul_(1.5)                              # eager work between the replays
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in results]
        for t in results:
            t.zero_()
        all_calls()
        torch.cuda.synchronize()
        assert all(torch.equal(t, v) for t, v in zip(results, replayed)), turn
