"""CPU-only: the workspaces of the losses do not grow with the tokens, whatever it is that a token takes most of (no launches)."""
import ctypes

import pytest

from test_loss_boundary import lib, problems  # noqa: F401  (lib: a fixture)

GB = 1 << 30


def size(lib, name, k=None, **kw):  # noqa: F811
    kw.setdefault("h_ld", kw["width"]), kw.setdefault("weight_ld", kw["width"])
    p = problems(**kw)[name]
    if k is not None and name == "tsenor_distill":
        p.k, p.ids_ld, p.logits_ld = k, k, k
    got = getattr(lib, name + "_workspace_bytes")(ctypes.byref(p))
    assert got > 0, kw
    return got


@pytest.mark.parametrize("name", ["tsenor_cross_entropy", "tsenor_distill"])
@pytest.mark.parametrize("gradients", [False, True])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("vocab,width,k", [(256, 8192, 16), (1, 65536, 1), (50257, 64, 16), (300, 64, 256), (64, 4096, 2), (5, 1, 256), (128256, 4096, 128)])
def test_what_a_piece_takes_is_bounded(lib, name, gradients, dtype, vocab, width, k):  # noqa: F811
    """Gradients of logits, hidden states, and sums with entries: up to 2 GiB each (but 256 tokens there are)."""
    more = {} if gradients else dict(dh_out=None, dweight_out=None)
    bits = 10 if dtype == 0 else 2
    row = [(vocab + 63) // 64 * 64 * bits * gradients, (width + 63) // 64 * 64 * (6 if dtype == 0 else 2), (vocab + 63) // 64 * 8 + 8 * k + 4 + (vocab + 63) // 64 * 2 + 2]
    head = (vocab + 63) * (width + 63) * (6 if dtype == 0 else 2) + 4 * vocab * width * gradients      # a copy, and a sum of its gradient
    shared = 256 * 1024 * 1024                                                                          # parts of sums
    for tokens in (1 << 20, 1 << 24):
        most = sum(max(2 * GB, 256 * each) for each in row) + head + shared + 16 * tokens + (1 << 20)
        assert size(lib, name, k, tokens=tokens, vocab=vocab, width=width, dtype=dtype, **more) <= most
