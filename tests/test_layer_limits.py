"""CPU-only checks of the layer operators at the edges of what they accept (no launches)."""
import ctypes

import pytest


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
