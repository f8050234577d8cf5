"""Operators for networks on decoded batches (include/rinr_nn.h), what needs no GPU: the binding against the header, and refusals."""
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2306_16699_amd import rinr, rinr_nn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "rinr_nn.h")


def test_binding_lists_what_the_header_declares():
    text = open(HEADER).read()
    declared = set(re.findall(r"^(?:int|size_t) (rinr_\w+)\(", text, re.M))
    assert declared == set(rinr_nn.EXPORTS)
    for name in declared:
        assert getattr(rinr_nn.lib(), name)
    for key, value in (("RINR_T_BF16", rinr_nn.TYPES[torch.bfloat16]), ("RINR_T_F16", rinr_nn.TYPES[torch.float16]),
                       ("RINR_T_F32", rinr_nn.TYPES[torch.float32]), ("RINR_T_PACKED8", rinr_nn.PACKED8), ("RINR_NN_MAX_COLS", rinr_nn.MAX_NORM_COLS),
                       *(("RINR_ACT_" + k.upper(), v) for k, v in rinr_nn.ACTS.items())):
        assert re.search(rf"\b{key} = {value}\b", text), key


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not found")
def test_argument_structures_have_the_headers_layout(tmp_path):
    """Every field of the C structures lies where the binding packs it."""
    text = open(HEADER).read()
    named = {"rinr_linear_args": rinr_nn._LINEAR, "rinr_linear_grad_args": rinr_nn._LINEAR_GRAD, "rinr_norm_args": rinr_nn._NORM,
             "rinr_norm_grad_args": rinr_nn._NORM_GRAD}
    lines = []
    for body, name in re.findall(r"typedef struct \{(.*?)\} (\w+);", text, re.S):
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = [f.strip().split()[-1].lstrip("*") for decl in body.split(";") for f in decl.split(",") if f.strip()]
        lines += [f'printf("{name} %zu %zu\\n", sizeof({name}), offsetof({name}, {f}));' for f in fields]
    c = tmp_path / "layout.c"
    c.write_text(f'#include <stdio.h>\n#include "{HEADER}"\nint main(void) {{ {" ".join(lines)} return 0; }}\n')
    subprocess.run(["gcc", str(c), "-o", str(tmp_path / "layout")], check=True)
    got = {}
    for ln in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.splitlines():
        name, size, at = ln.split()
        got.setdefault(name, (int(size), []))[1].append(int(at))
    assert set(got) == set(named)
    for name, s in named.items():
        at, here = 0, []
        for f in s.format.lstrip("="):
            here.append(at)
            at += {"q": 8, "Q": 8, "i": 4, "f": 4}[f]
        assert (at, here) == got[name], name


def linear_args(**k):
    d = dict(rows=4, n_in=8, n_out=8, x=4096, ld_x=8, x_scales=0, w=4096, ld_w=8, bias=0, residual=0, ld_residual=0, y=4096, ld_y=8, z=0, ld_z=0, z_scales=0,
             dtype=1, x_type=1, z_type=0, act=0, w0=30.0, reserved=0)
    d.update(k)
    return rinr_nn._LINEAR.pack(*d.values())


BAD_LINEAR = [(dict(rows=-1), rinr.E_ARG), (dict(n_in=0), rinr.E_ARG), (dict(n_out=0), rinr.E_ARG), (dict(n_in=(1 << 20) + 1), rinr.E_ARG),
              (dict(rows=1 << 31), rinr.E_ARG), (dict(dtype=0), rinr.E_ARG), (dict(dtype=4), rinr.E_ARG), (dict(x_type=2), rinr.E_ARG),
              (dict(z_type=3), rinr.E_ARG), (dict(act=5), rinr.E_ARG), (dict(act=-1), rinr.E_ARG), (dict(act=4, w0=float("nan")), rinr.E_ARG),
              (dict(act=4, w0=float("inf")), rinr.E_ARG), (dict(reserved=1), rinr.E_ARG), (dict(x=0), rinr.E_NULL), (dict(w=0), rinr.E_NULL),
              (dict(y=0), rinr.E_NULL), (dict(z_type=1), rinr.E_NULL), (dict(z_type=4, z=4096, ld_z=32), rinr.E_NULL), (dict(x_type=4, ld_x=32), rinr.E_NULL),
              (dict(x_type=4, ld_x=40, x_scales=64), rinr.E_ARG), (dict(x_type=4, ld_x=32, x_scales=64, x=4100), rinr.E_ALIGN), (dict(ld_x=7), rinr.E_ARG),
              (dict(ld_w=7), rinr.E_ARG), (dict(ld_y=7), rinr.E_ARG), (dict(residual=4096, ld_residual=7), rinr.E_ARG), (dict(x=4097), rinr.E_ALIGN),
              (dict(bias=4098), rinr.E_ALIGN), (dict(dtype=3, x_type=3, y=4098), rinr.E_ALIGN)]


@pytest.mark.parametrize("change,code", BAD_LINEAR, ids=[str(c) for c, _ in BAD_LINEAR])
def test_linear_refuses(change, code):
    assert rinr_nn.lib().rinr_linear(linear_args(**change), None, 0, None) == code


def test_linear_of_no_rows_and_null():
    assert rinr_nn.lib().rinr_linear(linear_args(rows=0, x=0, y=0), None, 0, None) == rinr.OK
    assert rinr_nn.lib().rinr_linear(None, None, 0, None) == rinr.E_NULL
    assert rinr_nn.lib().rinr_linear_workspace_bytes(None) == 0
    assert rinr_nn.lib().rinr_linear_workspace_bytes(linear_args(rows=-1)) == 0


def grad_args(**k):
    d = dict(rows=4, n_in=8, n_out=8, dy=4096, ld_dy=8, x=4096, ld_x=8, x_scales=0, w=4096, ld_w=8, z=0, ld_z=0, z_scales=0, dx=4096, ld_dx=8, dw=4096, ld_dw=8,
             dbias=4096, dtype=1, x_type=1, z_type=0, act=0, x_act=0, w0=30.0)
    d.update(k)
    return rinr_nn._LINEAR_GRAD.pack(*d.values())


BAD_GRAD = [(dict(rows=-1), rinr.E_ARG), (dict(n_in=0), rinr.E_ARG), (dict(dtype=7), rinr.E_ARG), (dict(x_type=3), rinr.E_ARG), (dict(act=1), rinr.E_ARG),
            (dict(z_type=1, z=4096, ld_z=8), rinr.E_ARG), (dict(x_act=9), rinr.E_ARG), (dict(act=1, z_type=1, ld_z=8), rinr.E_NULL), (dict(dy=0), rinr.E_NULL),
            (dict(w=0), rinr.E_NULL), (dict(x=0), rinr.E_NULL), (dict(dw=0, x=0, x_act=2), rinr.E_NULL), (dict(ld_dx=7), rinr.E_ARG), (dict(ld_dw=7), rinr.E_ARG),
            (dict(dx=4097), rinr.E_ALIGN), (dict(dbias=4098), rinr.E_ALIGN), (dict(act=4, z_type=1, z=4096, ld_z=8, w0=float("nan")), rinr.E_ARG)]


@pytest.mark.parametrize("change,code", BAD_GRAD, ids=[str(c) for c, _ in BAD_GRAD])
def test_linear_backward_refuses(change, code):
    L = rinr_nn.lib()
    assert L.rinr_linear_backward(grad_args(**change), 4096, 1 << 30, None) == code
    assert L.rinr_linear_backward_workspace_bytes(grad_args(**change)) == 0


def test_linear_backward_workspace_is_asked_for():
    L = rinr_nn.lib()
    need = L.rinr_linear_backward_workspace_bytes(grad_args())
    assert need >= 8 * 4
    assert L.rinr_linear_backward(grad_args(), None, 0, None) == rinr.E_NULL
    assert L.rinr_linear_backward(grad_args(), 4096, need - 1, None) == rinr.E_SIZE
    assert L.rinr_linear_backward(grad_args(), 4100, need, None) == rinr.E_ALIGN
    assert L.rinr_linear_backward(None, None, 0, None) == rinr.E_NULL


def norm_args(**k):
    d = dict(rows=4, cols=8, x=4096, ld_x=8, residual=0, ld_residual=0, gain=4096, y=4096, ld_y=8, y_scales=0, h=0, ld_h=0, dtype=1, y_type=1, eps=1e-6, reserved=0)
    d.update(k)
    return rinr_nn._NORM.pack(*d.values())


BAD_NORM = [(dict(rows=-1), rinr.E_ARG), (dict(cols=0), rinr.E_ARG), (dict(dtype=4), rinr.E_ARG), (dict(y_type=2), rinr.E_ARG), (dict(eps=0.0), rinr.E_ARG),
            (dict(eps=float("nan")), rinr.E_ARG), (dict(eps=float("inf")), rinr.E_ARG), (dict(reserved=1), rinr.E_ARG), (dict(cols=32769, ld_x=40000, ld_y=40000), rinr.E_UNSUPPORTED),
            (dict(x=0), rinr.E_NULL), (dict(gain=0), rinr.E_NULL), (dict(y=0), rinr.E_NULL), (dict(y_type=4, ld_y=32), rinr.E_NULL), (dict(ld_x=7), rinr.E_ARG),
            (dict(residual=4096, ld_residual=8, h=4096, ld_h=7), rinr.E_ARG), (dict(gain=4097), rinr.E_ALIGN), (dict(x=4097), rinr.E_ALIGN)]


@pytest.mark.parametrize("change,code", BAD_NORM, ids=[str(c) for c, _ in BAD_NORM])
def test_norm_refuses(change, code):
    assert rinr_nn.lib().rinr_rms_norm(norm_args(**change), None) == code


def norm_grad_args(**k):
    d = dict(rows=4, cols=8, dy=4096, ld_dy=8, h=4096, ld_h=8, gain=4096, dres=0, ld_dres=0, dh=4096, ld_dh=8, dgain=4096, dtype=1, eps=1e-6)
    d.update(k)
    return rinr_nn._NORM_GRAD.pack(*d.values())


def test_norm_backward_refuses():
    L = rinr_nn.lib()
    need = L.rinr_rms_norm_backward_workspace_bytes(4, 8)
    assert need >= 8 * 4
    for change, ws, size, code in ((dict(rows=-1), 4096, need, rinr.E_ARG), (dict(eps=-1.0), 4096, need, rinr.E_ARG), (dict(cols=40000), 4096, need, rinr.E_UNSUPPORTED),
                                   (dict(dy=0), 4096, need, rinr.E_NULL), (dict(h=0), 4096, need, rinr.E_NULL), (dict(dh=0), 4096, need, rinr.E_NULL),
                                   (dict(gain=0), 4096, need, rinr.E_NULL), (dict(ld_dh=7), 4096, need, rinr.E_ARG), (dict(dres=4096, ld_dres=7), 4096, need, rinr.E_ARG),
                                   (dict(dgain=4098), 4096, need, rinr.E_ALIGN), (dict(), None, 0, rinr.E_NULL), (dict(), 4096, need - 1, rinr.E_SIZE),
                                   (dict(), 4100, need, rinr.E_ALIGN), (dict(rows=0, dgain=0), None, 0, rinr.OK)):
        assert L.rinr_rms_norm_backward(norm_grad_args(**change), ws, size, None) == code, change
    assert L.rinr_rms_norm_backward_workspace_bytes(-1, 8) == 0 and L.rinr_rms_norm_backward_workspace_bytes(4, 0) == 0


def test_checkpoints_refuse():
    L = rinr_nn.lib()
    for args, code in (((-1, 8, 4096, 8, 1, 4096, 32, 4096, None), rinr.E_ARG), ((4, 0, 4096, 8, 1, 4096, 32, 4096, None), rinr.E_ARG),
                       ((4, 8, 4096, 8, 4, 4096, 32, 4096, None), rinr.E_ARG), ((4, 8, None, 8, 1, 4096, 32, 4096, None), rinr.E_NULL),
                       ((4, 8, 4096, 8, 1, 4096, 32, None, None), rinr.E_NULL), ((4, 8, 4096, 8, 1, 4096, 16, 4096, None), rinr.E_ARG),
                       ((4, 8, 4096, 8, 1, 4104, 32, 4096, None), rinr.E_ALIGN), ((4, 8, 4097, 8, 1, 4096, 32, 4096, None), rinr.E_ALIGN), ((0, 8, None, 8, 1, None, 32, None, None), rinr.OK)):
        assert L.rinr_pack8(*args) == code, args
    for args, code in (((4, 8, 4096, 32, 4096, 5, 30.0, 4096, 8, 1, None), rinr.E_ARG), ((4, 8, 4096, 32, 4096, 4, float("inf"), 4096, 8, 1, None), rinr.E_ARG),
                       ((4, 8, 4096, 32, 4096, 0, 30.0, 4096, 7, 1, None), rinr.E_ARG), ((4, 8, 4096, 32, None, 0, 30.0, 4096, 8, 1, None), rinr.E_NULL),
                       ((4, 8, 4096, 32, 4096, 0, 30.0, 4098, 8, 3, None), rinr.E_ALIGN), ((0, 8, None, 32, None, 0, 30.0, None, 8, 1, None), rinr.OK)):
        assert L.rinr_unpack8(*args) == code, args


def test_binding_refuses_what_no_kernel_takes():
    x, w = torch.zeros(4, 8), torch.zeros(8, 8)
    for call in (lambda: rinr_nn.linear(x, w), lambda: rinr_nn.linear_backward(x, x, w), lambda: rinr_nn.rms_norm(x, torch.ones(8)),
                 lambda: rinr_nn.rms_norm_backward(x, x, torch.ones(8)), lambda: rinr_nn.pack8(x), lambda: rinr_nn.pack8(x.double()), lambda: rinr_nn.linear(x, w.double()),
                 lambda: rinr_nn.linear(x, w, keep_z="z"), lambda: rinr_nn.unpack8(rinr_nn.Packed8(torch.zeros(4, 32, dtype=torch.int8), torch.ones(4, 1, dtype=torch.uint8), 8)),
                 lambda: rinr_nn.Packed8(torch.zeros(4, 8, dtype=torch.int8), torch.ones(4, 1, dtype=torch.uint8), 8),
                 lambda: rinr_nn.Packed8(torch.zeros(4, 32), torch.ones(4, 1, dtype=torch.uint8), 8)):
        with pytest.raises(rinr.RinrError) as e:
            call()
        assert e.value.code == rinr.E_ARG


def test_no_workspace_for_no_rows():
    L = rinr_nn.lib()
    assert L.rinr_linear_workspace_bytes(linear_args(rows=0)) == 0
    assert L.rinr_linear_backward_workspace_bytes(grad_args(rows=0)) == 0
    assert L.rinr_rms_norm_backward_workspace_bytes(0, 8) == 0


def test_a_packed_matrix_has_the_shape_of_its_rows():
    """Results are allocated by a Packed8's shape and written by its rows: one says the other."""
    codes, scales = torch.zeros(24, 64, dtype=torch.int8), torch.ones(24, 2, dtype=torch.uint8)
    for shape in ((2, 48), (24, 64), (24, 47), (23, 48), (25, 48), (), (48,), (2, 3, 5, 48), (-4, -6, 48), (24, 48, 1), (0, 48)):
        with pytest.raises(rinr.RinrError) as e:
            rinr_nn.Packed8(codes, scales, 48, shape=shape)
        assert e.value.code == rinr.E_ARG, shape
    for shape in (None, (24, 48), (2, 3, 4, 48), torch.Size((24, 1, 48))):
        p = rinr_nn.Packed8(codes, scales, 48, shape=shape)
        assert p.shape == ((24, 48) if shape is None else tuple(shape)) and (p.rows, p.cols, p.ld) == (24, 48, 64)
    assert rinr_nn.Packed8(codes[:1], scales[:1], 48, shape=(48,)).shape == (48,)
    assert rinr_nn.Packed8(codes[:0], scales[:0], 48, shape=(3, 0, 48)).shape == (3, 0, 48)
    for name in ("shape", "rows", "cols", "ld", "device", "codes", "scales"):
        with pytest.raises(AttributeError):
            setattr(p, name, getattr(p, name))


def test_what_is_no_stream_leaves_the_caller_on_its_gpu(monkeypatch):
    at = [0]

    class Guard:
        def __init__(self, dev):
            self.dev = dev

        def __enter__(self):
            self.before, at[0] = at[0], self.dev.index

        def __exit__(self, *_):
            at[0] = self.before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: at[0])
    monkeypatch.setattr(torch.cuda, "device", Guard)
    for stream in ("side", object(), 1.5):
        with pytest.raises(AttributeError):
            rinr_nn._on(torch.device("cuda:1"), stream)
        assert at[0] == 0


def _refusal(call):
    with pytest.raises(rinr.RinrError) as e:
        call()
    assert e.value.code == rinr.E_ARG
    return str(e.value)


def test_tensors_that_require_gradients_are_refused_while_these_are_recorded():
    """A result without a graph would leave its inputs without gradients, and say nothing."""
    x, v = torch.zeros(4, 8, requires_grad=True), torch.zeros(8, requires_grad=True)
    assert "no graph" in _refusal(lambda: rinr_nn._mat(x, "x")) and "no graph" in _refusal(lambda: rinr_nn._vector(v, 8, v.device, "bias"))
    assert "no graph" in _refusal(lambda: rinr_nn.pack8(x)) and "no graph" in _refusal(lambda: rinr_nn.rms_norm(x, v))
    with torch.no_grad():
        assert rinr_nn._vector(v, 8, v.device, "bias") == v.data_ptr()
        assert "on the GPU" in _refusal(lambda: rinr_nn.pack8(x))      # for where it is, not for its gradients

    class Packed(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return rinr_nn.pack8(x)

    assert "on the GPU" in _refusal(lambda: Packed.apply(x))


@pytest.mark.parametrize("change", [dict(), dict(y=4096 + 2), dict(y=4096 + 3 * 16 + 14), dict(y=1 << 20, z=4096, ld_z=8, z_type=1), dict(y=1 << 20, z=1 << 21, ld_z=8, z_type=1, w=1 << 21),
                                    dict(y=1 << 20, w=(1 << 20) + 14), dict(y=1 << 20, residual=(1 << 20) + 2, ld_residual=8), dict(y=1 << 20, residual=1 << 20, ld_residual=16),
                                    dict(y=4096 + 14, ld_y=16, ld_x=16), dict(y=4096 + 18, ld_y=16, ld_x=16), dict(x=4096 + 18, y=4096, ld_y=16, ld_x=16),
                                    dict(x=4096, x_type=4, ld_x=32, x_scales=1 << 22, y=4096 + 100), dict(y=4096 + 16, ld_y=9, ld_x=16)], ids=str)
def test_linear_refuses_results_on_top_of_what_it_reads(change):
    """Checked before anything else is done with the pointers: these never reach a kernel."""
    args = dict(w=1 << 30)
    args.update(change)
    assert rinr_nn.lib().rinr_linear(linear_args(**args), None, 0, None) == rinr.E_ARG
