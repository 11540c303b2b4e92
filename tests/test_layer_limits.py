"""CPU-only checks of the layer operators at the edges of what they accept (no launches)."""
import ctypes
import re
from pathlib import Path

import pytest
import torch

ROOT = Path(__file__).resolve().parent.parent


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


def test_a_matrix_of_another_shape_is_not_one_that_is_not_wanted():
    from paper_2505_23949_amd import layer as l

    # (memory without elements has no address, which stands for "not wanted" in C)
    x = torch.zeros(4, 256)
    for one in (l.empty_scaled(0, 256, "cpu"), l.empty_scaled(4, 128, "cpu")):
        with pytest.raises(ValueError, match="out must be a scaled matrix of 4 x 256"):
            l.make_quantize(x, out=one)
        with pytest.raises(ValueError, match="out must be a scaled matrix of 4 x 256"):
            l.make_norm(x, torch.zeros(256), 1e-5, out=one, y_out=torch.zeros(4, 256))
    with pytest.raises(ValueError, match="out_t must be a scaled matrix of 256 x 4"):
        l.make_quantize(x, out=l.empty_scaled(4, 256, "cpu"), out_t=l.empty_scaled(0, 4, "cpu"))


def test_what_a_scale_byte_stands_for():
    from paper_2505_23949_amd import layer as l

    values = torch.full((4, 128), 1.5).to(torch.float8_e4m3fn)
    scales = torch.tensor([[0, 1, 254, 255] + [127] * 12], dtype=torch.uint8)
    wide = l.scaled_matrix(values, scales, 128).dequantize()
    assert (wide[0] == 1.5 * 2.0 ** -127).all() and (wide[1] == 1.5 * 2.0 ** -126).all() and (wide[2] == 1.5 * 2.0 ** 127).all()
    assert torch.isnan(wide[3]).all()


class FakeCuda:
    """Two GPUs as the binding sees them: the current one, its stream, and a library that notes what was current at each call."""

    def __init__(self, monkeypatch):
        from paper_2505_23949_amd import binding, layer

        self.current, self.calls = 0, []
        fake = self

        class Guard:
            def __init__(self, device):
                self.device = torch.device(device).index if isinstance(device, (str, torch.device)) else device

            def __enter__(self):
                self.before, fake.current = fake.current, self.device

            def __exit__(self, *_):
                fake.current = self.before

        class Library:
            def __getattr__(self, name):
                def call(problem, *rest):
                    fake.calls.append((name, fake.current, rest[-1]))
                    return 0
                return call

        monkeypatch.setattr(torch.cuda, "device", Guard)
        monkeypatch.setattr(torch.cuda, "init", lambda: None)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: fake.current, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
        for name in ("_current_device", "_raw_stream"):
            monkeypatch.setattr(binding, name, None)
        monkeypatch.setattr(layer, "load", lambda: Library())


class OnDevice:
    """A workspace on a GPU."""

    def __init__(self, index):
        self.index = index

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x100000

    def numel(self):
        return 4096

    def element_size(self):
        return 1


def test_calls_go_to_the_gpu_of_their_tensors(monkeypatch):
    from paper_2505_23949_amd import layer as l

    fake = FakeCuda(monkeypatch)
    monkeypatch.setattr(l, "_one_device", lambda **_: 1)
    x, bf16 = torch.zeros(4, 256), torch.zeros(4, 4).bfloat16()
    q, norm = l.empty_scaled(4, 256, "cpu"), torch.zeros(2)
    gain = torch.zeros(256)
    calls = [(l.tsenor_quantize, l.make_quantize(x, out=q)), (l.tsenor_norm, l.make_norm(x, gain, 1e-5, out=q)),
             (l.tsenor_norm_backward, l.make_norm_backward(x, gain, 1e-5, x, dh=x.clone(), dgain=gain.clone())),
             (l.tsenor_product, l.make_product(q, q, out=bf16)), (l.tsenor_clip, l.make_clip([x], 1.0, norm_out=norm))]
    for current in (0, 1):
        fake.current = current
        for call, p in calls:
            call(p, *(() if call in (l.tsenor_quantize, l.tsenor_norm) else (OnDevice(1),)))
            assert fake.calls[-1] == (call.__name__, 1, 101) and fake.current == current
    # a problem that was filled by hand goes to the current one
    fake.current = 0
    l.tsenor_quantize(l.tsenor_quantize_problem())
    assert fake.calls[-1] == ("tsenor_quantize", 0, 100)


def test_workspaces_elsewhere_are_refused(monkeypatch):
    from paper_2505_23949_amd import layer as l

    FakeCuda(monkeypatch)
    monkeypatch.setattr(l, "_one_device", lambda **_: 0)
    p = l.make_clip([torch.zeros(4)], 1.0, norm_out=torch.zeros(2))
    for workspace in (torch.zeros(4096, dtype=torch.uint8), OnDevice(1)):      # in host memory, and on another GPU
        with pytest.raises(ValueError, match="workspace"):
            l.tsenor_clip(p, workspace)


def test_assembly_names_the_registers_and_memory_it_changes():
    # a statement that writes m0 says so: the compiler may keep an address or a lane number there
    found = 0
    for source in sorted((ROOT / "paper_2505_23949_amd" / "csrc").glob("*.h*p*")):
        for statement in re.findall(r"asm volatile\((.*?)\);", source.read_text(), re.S):
            if re.search(r"s_mov_b32 m0", statement):
                found += 1
                assert '"m0"' in statement.split(":")[-1], (source.name, statement)
    assert found
