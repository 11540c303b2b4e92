"""CPU-only checks of the losses' boundary: struct layouts, argument validation, workspace sizes (no launches)."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2505_23949_amd import binding

    if not binding.LIB_PATH.exists():
        from paper_2505_23949_amd import build

        build.build()
    return binding.load()


def test_struct_layouts_match_the_header(tmp_path):
    from paper_2505_23949_amd import loss

    prog, want = '#include <stdio.h>\n#include <stddef.h>\n#include "tsenor_loss.h"\nint main(void){\n', []
    for s in (loss.tsenor_head, loss.tsenor_cross_entropy_problem, loss.tsenor_distill_problem):
        prog += f'printf("%zu\\n", sizeof({s.__name__}));\n'
        want.append(ctypes.sizeof(s))
        for name, _ in s._fields_:
            prog += f'printf("%zu\\n", offsetof({s.__name__}, {name}));\n'
            want.append(getattr(s, name).offset)
    prog += 'printf("%d\\n", TSENOR_LOSS_MAX_ENTRIES);\n'
    want.append(loss.TSENOR_LOSS_MAX_ENTRIES)
    source, program = tmp_path / "layout.c", tmp_path / "layout"
    source.write_text(prog + "return 0;}\n")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", program, source], check=True)
    assert [int(x) for x in subprocess.run([program], capture_output=True, text=True, check=True).stdout.split()] == want


def head(**kw):
    from paper_2505_23949_amd import loss as l

    p = l.tsenor_head(h=0x1000, weight=0x2000, dtype=1, tokens=100, vocab=1000, width=256, h_ld=256, weight_ld=256, dloss=0x3000,
                      loss_out=0x4000, lse_out=0x5000, dh_out=0x6000, dweight_out=0x7000)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def problems(**kw):
    """A valid problem of both operators (pointers are never dereferenced: validation happens on the host)."""
    from paper_2505_23949_amd import loss as l

    return {"tsenor_cross_entropy": l.tsenor_cross_entropy_problem(head=head(**kw), targets=0x8000),
            "tsenor_distill": l.tsenor_distill_problem(head=head(**kw), ids=0x8000, logits=0x9000, logits_dtype=0, k=16, ids_ld=16,
                                                       logits_ld=16, temperature=2.0)}


OF_THE_HEAD = [
    (dict(h=None), "NULL"), (dict(weight=None), "NULL"), (dict(loss_out=None), "NULL"), (dict(dtype=2), "UNSUPPORTED"), (dict(dtype=-1), "UNSUPPORTED"),
    (dict(tokens=-1), "SHAPE"), (dict(tokens=(1 << 24) + 1), "SHAPE"), (dict(vocab=-1), "SHAPE"), (dict(vocab=(1 << 21) + 1), "SHAPE"),
    (dict(width=-1), "SHAPE"), (dict(width=(1 << 16) + 1, h_ld=1 << 17, weight_ld=1 << 17), "SHAPE"), (dict(h_ld=255), "SHAPE"),
    (dict(weight_ld=255), "SHAPE"), (dict(h_ld=(1 << 40) + 1), "SHAPE"), (dict(h=0x1001), "ALIGN"), (dict(weight=0x2001), "ALIGN"),
    (dict(dh_out=0x6001), "ALIGN"), (dict(dweight_out=0x7001), "ALIGN"), (dict(dloss=0x3002), "ALIGN"), (dict(loss_out=0x4002), "ALIGN"),
    (dict(lse_out=0x5001), "ALIGN"), (dict(dtype=0, h=0x1002), "ALIGN")]
REFUSED = {
    "tsenor_cross_entropy": [(dict(targets=None), "NULL"), (dict(targets=0x8004), "ALIGN")],
    "tsenor_distill": [
        (dict(ids=None), "NULL"), (dict(logits=None), "NULL"), (dict(k=-1), "SHAPE"), (dict(k=257, ids_ld=300, logits_ld=300), "SHAPE"),
        (dict(ids_ld=15), "SHAPE"), (dict(logits_ld=15), "SHAPE"), (dict(logits_dtype=3), "UNSUPPORTED"), (dict(temperature=0.0), "PARAM"),
        (dict(temperature=-1.0), "PARAM"), (dict(temperature=math.nan), "PARAM"), (dict(temperature=math.inf), "PARAM"),
        (dict(temperature=2.0 ** 21), "PARAM"), (dict(temperature=2.0 ** -21), "PARAM"), (dict(ids=0x8004), "ALIGN"), (dict(logits=0x9002), "ALIGN")],
}


@pytest.mark.parametrize("name", sorted(REFUSED))
def test_refusals(lib, name):
    from paper_2505_23949_amd import binding as b

    call, size = getattr(lib, name), getattr(lib, name + "_workspace_bytes")
    assert call(None, ctypes.c_void_p(0x100000), 1 << 40, None) == b.TSENOR_ERR_NULL and size(None) == 0
    wrong = [(problems(**change)[name], change, status) for change, status in OF_THE_HEAD]
    for change, status in REFUSED[name]:
        p = problems()[name]
        for k, v in change.items():
            setattr(p, k, v)
        wrong.append((p, change, status))
    for p, change, status in wrong:
        assert call(ctypes.byref(p), ctypes.c_void_p(0x100000), 1 << 40, None) == getattr(b, "TSENOR_ERR_" + status), change
        assert size(ctypes.byref(p)) == 0, change
    p = problems()[name]
    need = size(ctypes.byref(p))
    assert need > 0 and need % 256 == 0
    for ws, n in ((0, need), (0x100080, need), (0x100000, need - 1)):
        assert call(ctypes.byref(p), ctypes.c_void_p(ws), n, None) == b.TSENOR_ERR_WORKSPACE


@pytest.mark.parametrize("name", sorted(REFUSED))
def test_workspaces_are_bounded(lib, name):
    """What is kept of the logits does not grow with the tokens past 2 GiB, nor with tokens at all where no gradient is wanted."""
    size = getattr(lib, name + "_workspace_bytes")

    def of(**kw):
        p = problems(**kw)[name]
        got = size(ctypes.byref(p))
        assert got > 0, kw
        return got

    none = dict(dh_out=None, dweight_out=None)
    wide = dict(vocab=1 << 17, width=64, h_ld=64, weight_ld=64)
    assert of(tokens=1 << 20, **wide, dweight_out=None) < 3 << 30
    assert of(tokens=1 << 20, **wide) < 4 << 30
    assert of(tokens=1 << 20, **wide, **none) < 1 << 30
    assert of(tokens=1, **wide, **none) < 1 << 25
    # the largest of everything, still a size
    assert of(tokens=1 << 24, vocab=1 << 21, width=1 << 16, h_ld=1 << 36, weight_ld=1 << 36) > 1 << 37
    assert of(tokens=0) > 0 and of(vocab=0, weight=None) > 0 and of(width=0, h=None, weight=None, h_ld=0, weight_ld=0) > 0


def test_python_checks(lib):
    from paper_2505_23949_amd import loss as l

    h, weight, targets, out = torch.zeros(4, 64), torch.zeros(100, 64), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    ids, logits = torch.zeros(4, 3, dtype=torch.int64), torch.zeros(4, 3)
    with pytest.raises(ValueError, match="one GPU"):
        l.make_cross_entropy(h, weight, targets, loss=out)
    with pytest.raises(ValueError, match="targets"):
        l.make_cross_entropy(h, weight, targets.int(), loss=out)
    with pytest.raises(ValueError, match="targets"):
        l.make_cross_entropy(h, weight, targets[:3], loss=out)
    with pytest.raises(ValueError, match="ids"):
        l.make_distill(h, weight, ids.int(), logits, loss=out)
    with pytest.raises(ValueError, match="ids"):
        l.make_distill(h, weight, ids, logits[:, :2], loss=out)
    with pytest.raises(ValueError, match="overlap"):
        l.make_distill(h, weight, ids[:1].expand(4, 3), logits, loss=out)
    for bad in (dict(h=h.t().contiguous().t()), dict(weight=weight.bfloat16()), dict(weight=weight[:, :32]), dict(h=h.half(), weight=weight.half()),
                dict(loss=out.double()), dict(loss=torch.zeros(8)[::2]), dict(loss=out[:3]), dict(lse=torch.zeros(5)), dict(dloss=out.bfloat16()),
                dict(dh=torch.zeros(4, 65)[:, :64]), dict(dh=torch.zeros(4, 64).bfloat16()), dict(dweight=torch.zeros(99, 64))):
        with pytest.raises((ValueError, TypeError)) as e:
            l._head(**{**dict(h=h, weight=weight, dloss=None, loss=out, lse=None, dh=None, dweight=None), **bad})
        assert "GPU" not in str(e.value), bad
