"""CPU-only checks of the layer operators at the edges of what they accept (no launches)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2505_23949_amd import binding

    if not binding.LIB_PATH.exists():
        from paper_2505_23949_amd import build

        build.build()
    return binding.load()


def test_workspace_of_clipping_does_not_grow_with_the_tensors(lib):
    # every workgroup of the second pass adds all sums of the first: as many as the largest launch has workgroups, however many launches
    from paper_2505_23949_amd import layer as l

    def size(count, elements):
        table = (l.tsenor_gradient * count)(*(l.tsenor_gradient(0x1000, 0x1000, elements, 0) for _ in range(count)))
        return lib.tsenor_clip_workspace_bytes(ctypes.byref(l.tsenor_clip_problem(gradients=table, count=count, max_norm=1.0, norm_out=0x1000)))

    for elements in (1, 5000, 1 << 20):
        assert 0 < size(100_000, elements) <= 2048 * 8


def test_rows_too_far_apart_to_address(lib):
    # rows x leading dimension beyond any address: refused, though each of the two is in range
    from paper_2505_23949_amd import binding as b
    from paper_2505_23949_amd import layer as l

    rows, ld = (1 << 30) - 1000, 1 << 40
    out = l.tsenor_scaled(0x10000, 0x20000, rows, 1, 128, -(-rows // 16) * 16)
    far = l.tsenor_scaled(0x10000, 0x20000, rows, 1, ld, -(-rows // 16) * 16)
    small = l.tsenor_scaled(0x10000, 0x20000, 5, 1, 128, 16)
    norm = dict(x=0x1000, gain=0x1000, dtype=0, gain_dtype=0, rows=rows, cols=1, y_out=0x1000)
    back = dict(h=0x1000, gain=0x1000, dy=0x1000, dsum=0x1000, dtype=0, gain_dtype=0, rows=rows, cols=1, dh_out=0x1000, dgain_out=0x1000)
    for name, p in (("tsenor_quantize", l.tsenor_quantize_problem(x=0x1000, dtype=0, rows=rows, cols=1, ld=ld, out=out)),
                    ("tsenor_quantize", l.tsenor_quantize_problem(x=0x1000, dtype=0, rows=rows, cols=1, ld=1, out=far)),
                    ("tsenor_norm", l.tsenor_norm_problem(ld=ld, **norm)),
                    ("tsenor_norm", l.tsenor_norm_problem(ld=1, residual=0x1000, residual_ld=ld, **norm)),
                    ("tsenor_norm_backward", l.tsenor_norm_backward_problem(ld=ld, dy_ld=1, dsum_ld=1, **back)),
                    ("tsenor_norm_backward", l.tsenor_norm_backward_problem(ld=1, dy_ld=ld, dsum_ld=1, **back)),
                    ("tsenor_norm_backward", l.tsenor_norm_backward_problem(ld=1, dy_ld=1, dsum_ld=ld, **back)),
                    ("tsenor_product", l.tsenor_product_problem(a=out, b=small, out=0x1000, out_ld=ld))):
        f = getattr(lib, name)
        scratch = (ctypes.c_void_p(0x100000), 1 << 40) if len(f.argtypes) == 4 else ()
        assert f(ctypes.byref(p), *scratch, None) == b.TSENOR_ERR_SHAPE, name


def test_backward_without_a_training_pass():
    from paper_2505_23949_amd.masked_layer import MaskedLayer

    one = MaskedLayer.__new__(MaskedLayer)
    one._kept = None
    with pytest.raises(RuntimeError, match="training"):
        one.backward(torch.zeros(4, 4))
