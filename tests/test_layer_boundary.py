"""CPU-only checks of the layer operators' boundary: struct layouts, argument validation, workspace sizes (no launches)."""
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


def scaled(rows=256, cols=512, **kw):
    from paper_2505_23949_amd import layer

    s = layer.tsenor_scaled(0x10000, 0x20000, rows, cols, -(-cols // 128) * 128, -(-rows // 16) * 16)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def test_struct_layouts_match_the_header(tmp_path):
    from paper_2505_23949_amd import layer

    structs = [layer.tsenor_scaled, layer.tsenor_quantize_problem, layer.tsenor_norm_problem, layer.tsenor_norm_backward_problem,
               layer.tsenor_product_problem, layer.tsenor_gradient, layer.tsenor_clip_problem]
    prog, want = '#include <stdio.h>\n#include <stddef.h>\n#include "tsenor_layer.h"\nint main(void){\n', []
    for s in structs:
        prog += f'printf("%zu\\n", sizeof({s.__name__}));\n'
        want.append(ctypes.sizeof(s))
        for name, _ in s._fields_:
            prog += f'printf("%zu\\n", offsetof({s.__name__}, {name.rstrip("_")}));\n'
            want.append(getattr(s, name).offset)
    source, program = tmp_path / "layout.c", tmp_path / "layout"
    source.write_text(prog + "return 0;}\n")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", program, source], check=True)
    assert [int(x) for x in subprocess.run([program], capture_output=True, text=True, check=True).stdout.split()] == want


def problems():
    """A valid problem of every operator (pointers are never dereferenced: validation happens on the host)."""
    from paper_2505_23949_amd import layer as l

    grads = (l.tsenor_gradient * 2)(l.tsenor_gradient(0x1000, 0x2000, 100, 0), l.tsenor_gradient(0x3000, 0x4000, 50, 1))
    return {
        "tsenor_quantize": l.tsenor_quantize_problem(x=0x1000, dtype=0, rows=256, cols=512, ld=512, out=scaled(), out_t=scaled(512, 256)),
        "tsenor_norm": l.tsenor_norm_problem(x=0x1000, residual=0x2000, gain=0x3000, dtype=1, gain_dtype=0, rows=256, cols=512, ld=512,
                                             residual_ld=512, eps=1e-5, sum_out=0x4000, y_out=0x5000, out=scaled()),
        "tsenor_norm_backward": l.tsenor_norm_backward_problem(h=0x1000, gain=0x2000, dy=0x3000, dsum=0x4000, dtype=0, gain_dtype=0,
                                                               rows=256, cols=512, ld=512, dy_ld=512, dsum_ld=512, eps=0.0,
                                                               dh_out=0x5000, dgain_out=0x6000),
        "tsenor_product": l.tsenor_product_problem(a=scaled(300), b=scaled(256), out=0x1000, out_ld=256),
        "tsenor_clip": l.tsenor_clip_problem(gradients=grads, count=2, max_norm=1.0, norm_out=0x1000),
    }


def with_scaled(field, **kw):
    def change(p):
        s = getattr(p, field)
        for k, v in kw.items():
            setattr(s, k, v)
    return change


def gradient(**kw):
    def change(p):
        for k, v in kw.items():
            setattr(p.gradients[1], k, v)
    return change


REFUSED = {
    "tsenor_quantize": [
        (dict(x=None), "NULL"), (lambda p: (with_scaled("out", values=None)(p), with_scaled("out_t", values=None)(p)), "NULL"),
        (with_scaled("out", scales=None), "NULL"), (dict(dtype=2), "UNSUPPORTED"), (dict(square=2), "UNSUPPORTED"), (dict(rows=-1), "SHAPE"),
        (dict(cols=-1), "SHAPE"), (dict(ld=511), "SHAPE"), (dict(rows=1 << 31), "SHAPE"), (dict(cols=(1 << 24) + 1, ld=1 << 25), "SHAPE"),
        (dict(rows=255), "SHAPE"), (dict(x=0x1002), "ALIGN"), (with_scaled("out", ld=520), "ALIGN"), (with_scaled("out", ld=384), "SHAPE"),
        (with_scaled("out", values=0x10008), "ALIGN"), (with_scaled("out", scale_ld=264), "ALIGN"), (with_scaled("out", scale_ld=240), "SHAPE"),
        (with_scaled("out_t", rows=256, cols=512), "SHAPE"), (with_scaled("out_t", scales=0x20008), "ALIGN")],
    "tsenor_norm": [
        (dict(x=None), "NULL"), (dict(gain=None), "NULL"),
        (lambda p: (with_scaled("out", values=None)(p), setattr(p, "sum_out", None), setattr(p, "y_out", None)), "NULL"),
        (dict(dtype=-1), "UNSUPPORTED"), (dict(gain_dtype=5), "UNSUPPORTED"), (dict(rows=-5), "SHAPE"), (dict(ld=100), "SHAPE"),
        (dict(residual_ld=100), "SHAPE"), (dict(eps=-1.0), "PARAM"), (dict(eps=math.nan), "PARAM"), (dict(eps=math.inf), "PARAM"),
        (dict(eps=1e300), "PARAM"), (dict(x=0x1001), "ALIGN"), (dict(residual=0x2001), "ALIGN"), (dict(sum_out=0x4001), "ALIGN"),
        (dict(y_out=0x5001), "ALIGN"), (dict(gain=0x3002), "ALIGN"), (with_scaled("out", rows=16), "SHAPE"), (with_scaled("out", ld=544), "ALIGN")],
    "tsenor_norm_backward": [
        (dict(h=None), "NULL"), (dict(gain=None), "NULL"), (dict(dy=None), "NULL"), (dict(dh_out=None), "NULL"), (dict(dgain_out=None), "NULL"),
        (dict(dtype=3), "UNSUPPORTED"), (dict(gain_dtype=3), "UNSUPPORTED"), (dict(cols=-1), "SHAPE"), (dict(dy_ld=1), "SHAPE"),
        (dict(dsum_ld=1), "SHAPE"), (dict(ld=1), "SHAPE"), (dict(eps=-1e-9), "PARAM"), (dict(h=0x1002), "ALIGN"), (dict(dh_out=0x5002), "ALIGN"),
        (dict(dgain_out=0x6002), "ALIGN")],
    "tsenor_product": [
        (dict(out=None), "NULL"), (with_scaled("a", values=None), "NULL"), (with_scaled("b", scales=None), "NULL"),
        (with_scaled("a", cols=500), "SHAPE"), (with_scaled("a", rows=-1), "SHAPE"), (with_scaled("b", ld=256), "SHAPE"),
        (with_scaled("b", ld=513), "ALIGN"), (with_scaled("a", values=0x10010 - 8), "ALIGN"), (dict(out_ld=255), "SHAPE"), (dict(out=0x1001), "ALIGN")],
    "tsenor_clip": [
        (dict(norm_out=None), "NULL"), (lambda p: setattr(p, "gradients", None), "NULL"), (dict(count=-1), "SHAPE"),
        (dict(count=(1 << 20) + 1), "SHAPE"), (dict(max_norm=-1.0), "PARAM"), (dict(max_norm=math.nan), "PARAM"), (gradient(in_=None), "NULL"),
        (gradient(out=None), "NULL"), (gradient(count=-1), "SHAPE"), (gradient(count=1 << 41), "SHAPE"), (gradient(dtype=7), "UNSUPPORTED"),
        (gradient(in_=0x3001), "ALIGN"), (gradient(out=0x4001), "ALIGN"), (dict(norm_out=0x1002), "ALIGN")],
}


def call(lib, name, p, ws=0x100000, size=1 << 40):
    f = getattr(lib, name)
    scratch = (ctypes.c_void_p(ws), size) if len(f.argtypes) == 4 else ()
    return f(None if p is None else ctypes.byref(p), *scratch, None)


@pytest.mark.parametrize("name", sorted(REFUSED))
def test_refusals(lib, name):
    from paper_2505_23949_amd import binding as b

    assert call(lib, name, None) == b.TSENOR_ERR_NULL
    for change, status in REFUSED[name]:
        p = problems()[name]
        if callable(change):
            change(p)
        else:
            for k, v in change.items():
                setattr(p, k, v)
        assert call(lib, name, p) == getattr(b, "TSENOR_ERR_" + status), (name, change, status)
        size = getattr(lib, name + "_workspace_bytes", None)
        assert size is None or size(ctypes.byref(p)) == 0, (name, change)


def test_workspaces(lib):
    from paper_2505_23949_amd import binding as b

    for name, p in problems().items():
        size = getattr(lib, name + "_workspace_bytes", None)
        if size is None or size(ctypes.byref(p)) == 0:
            continue
        need = size(ctypes.byref(p))
        assert need % 256 == 0
        for ws, n in ((0, need), (0x100080, need), (0x100000, need - 1)):
            assert call(lib, name, p, ws, n) == b.TSENOR_ERR_WORKSPACE, name
    assert getattr(lib, "tsenor_clip_workspace_bytes")(ctypes.byref(problems()["tsenor_clip"])) > 0
    assert getattr(lib, "tsenor_norm_backward_workspace_bytes")(ctypes.byref(problems()["tsenor_norm_backward"])) > 0
    assert "align" in b.status_string(b.TSENOR_ERR_ALIGN)


def test_matrices_without_elements_need_no_memory(lib):
    from paper_2505_23949_amd import binding as b
    from paper_2505_23949_amd import layer as l

    none = l.tsenor_scaled(None, None, 0, 512, 512, 16)
    assert call(lib, "tsenor_quantize", l.tsenor_quantize_problem(dtype=0, rows=0, cols=512, ld=512)) == b.TSENOR_OK
    assert call(lib, "tsenor_norm", l.tsenor_norm_problem(gain=0x1000, rows=0, cols=512, ld=512, out=none)) == b.TSENOR_OK
    assert call(lib, "tsenor_product", l.tsenor_product_problem(a=none, b=scaled(), out_ld=256)) == b.TSENOR_OK


def test_python_checks():
    from paper_2505_23949_amd import layer as l

    x = torch.zeros(4, 256)
    with pytest.raises(ValueError, match="one GPU"):
        l.make_quantize(x)
    with pytest.raises(ValueError, match="2-D"):
        l.make_quantize(x.t())
    with pytest.raises(ValueError, match="overlap"):
        l.make_quantize(torch.zeros(1, 256).expand(4, 256))
    with pytest.raises(ValueError, match="mask"):
        l.make_quantize(x, mask=torch.zeros(4, 255, dtype=torch.uint8))
    with pytest.raises(ValueError, match="gain"):
        l.make_norm(x, torch.zeros(255), 1e-5)
    with pytest.raises(ValueError, match="residual"):
        l.make_norm(x, torch.zeros(256), 1e-5, residual=x.bfloat16())
    with pytest.raises(ValueError, match="y_out must be contiguous"):
        l.make_norm(x, torch.zeros(256), 1e-5, y_out=torch.zeros(4, 300)[:, :256])
    with pytest.raises(ValueError, match="dgain"):
        l.make_norm_backward(x, torch.zeros(256), 1e-5, x, dh=torch.zeros(4, 256), dgain=torch.zeros(256).bfloat16())
    with pytest.raises(TypeError):
        l.scaled_matrix(x, x, 256)
    values, scales = torch.zeros(4, 256).to(torch.float8_e4m3fn), torch.zeros(2, 16, dtype=torch.uint8)
    q = l.scaled_matrix(values, scales, 200)
    assert (q.rows, q.cols) == (4, 200) and not q.dequantize().any()
    with pytest.raises(ValueError, match="128"):
        l.scaled_matrix(values, scales, 257)
    with pytest.raises(ValueError, match="multiple of 16"):
        l.scaled_matrix(values, torch.zeros(2, 4, dtype=torch.uint8), 200)
    with pytest.raises(ValueError, match="bfloat16"):
        l.make_product(q, q, out=torch.zeros(4, 4))
    with pytest.raises(ValueError, match="columns"):
        l.make_product(q, l.scaled_matrix(values, scales, 256), out=torch.zeros(4, 4).bfloat16())
    with pytest.raises(ValueError, match="norm_out"):
        l.make_clip([x], 1.0, norm_out=torch.zeros(1))
    with pytest.raises(ValueError, match="contiguous"):
        l.make_clip([x.t()], 1.0, norm_out=torch.zeros(2))


def test_scaled_matrix_on_two_devices():
    from paper_2505_23949_amd import layer as l

    values = torch.zeros(4, 256).to(torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="one device"):
        l.scaled_matrix(values, torch.zeros(2, 16, dtype=torch.uint8, device="meta"), 200)
