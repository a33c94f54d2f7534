"""include/liec_train.h: the library exports what it declares, it is plain C, and checks that need no GPU refuse bad arguments."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "liec_train.h")


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("count", ctypes.c_int64), ("stride", ctypes.c_int64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("worker_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class Param(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_int64)]


@pytest.fixture(scope="module")
def lib():
    import paper_2402_11857_amd as pkg

    if not os.path.exists(pkg.library_path()):
        from paper_2402_11857_amd import _build

        _build.build_library()
    return pkg.lib()


@pytest.fixture(scope="module")
def pkg(lib):
    import paper_2402_11857_amd as package
    from paper_2402_11857_amd import _build

    if not os.path.exists(_build.BINDING_PATH):
        _build.build_binding()
    return package


def test_every_declared_symbol_is_exported_and_bound(lib):
    import paper_2402_11857_amd as pkg

    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(liec_[a-z0-9_]+)\s*\(", text)))
    assert len(names) == 7
    for name in names:
        assert hasattr(lib, name)
        assert hasattr(pkg, name) or name.endswith("_workspace")


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "use_header.c"
    src.write_text('#include "liec_train.h"\n'
                   "int main(void) {\n"
                   "    liec_grad_tensor t = {0, 0, 0, LIEC_BF16, 0};\n"
                   "    liec_rows r = {0, 0, 0};\n"
                   "    liec_param p = {0, 0};\n"
                   "    (void)t; (void)r; (void)p;\n"
                   "    return (int)sizeof(liec_grad_tensor) - 32;\n"
                   "}\n")
    run = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-fsyntax-only", "-I", os.path.dirname(HEADER), str(src)],
                         capture_output=True, text=True)
    assert run.returncode == 0, run.stderr


def test_workspace_sizes(lib):
    assert lib.liec_grads_workspace(0, 1) == -1
    assert lib.liec_grads_workspace(65_536, 1) == -1
    assert lib.liec_grads_workspace(1, -1) == -1
    assert lib.liec_grads_workspace(1, 65_537) == -1
    for N in (1, 3, 64, 65_535):
        for T in (0, 1, 128, 129, 65_536):
            assert lib.liec_grads_workspace(N, T) >= 8 * N
    assert lib.liec_layer_norm_workspace(0, 1, 1) == -1
    assert lib.liec_layer_norm_workspace(1, -1, 1) == -1
    assert lib.liec_layer_norm_workspace(1, 1, 0) == -1
    assert lib.liec_layer_norm_workspace(1, 1 << 31, 1) == -1
    assert lib.liec_layer_norm_workspace(1, 1, 1 << 31) == -1
    assert lib.liec_layer_norm_workspace(3, 0, 100) == 0
    assert lib.liec_layer_norm_workspace(3, 10, 100) >= 3 * 2 * 100 * 4


FAKE = 0x10000                                               # an address that the checks look at and nothing reads


def _norm(lib, t, T=1, N=2, norms=FAKE, ws=FAKE, bytes=None):
    need = max(0, lib.liec_grads_workspace(max(N, 1) if N <= 65_535 else 1, 1))
    return lib.liec_grad_norm(ctypes.byref(t) if t else None, T, N, norms, ws, need if bytes is None else bytes, None)


def test_grad_norm_refusals(lib):
    good = Tensor(FAKE, 10, 10, 0, 0)
    assert _norm(lib, None) == 1
    assert _norm(lib, good, T=-1) == 1
    assert _norm(lib, good, N=0) == 1
    assert _norm(lib, good, N=65_536) == 1
    assert _norm(lib, good, norms=None) == 1
    assert _norm(lib, good, norms=FAKE + 2) == 1
    assert _norm(lib, good, ws=None) == 1
    assert _norm(lib, good, ws=FAKE + 8) == 1
    assert _norm(lib, good, bytes=0) == 1
    assert _norm(lib, Tensor(None, 10, 10, 0, 0)) == 1
    assert _norm(lib, Tensor(FAKE, -1, 10, 0, 0)) == 1
    assert _norm(lib, Tensor(FAKE, 10, 10, 3, 0)) == 1
    assert _norm(lib, Tensor(FAKE + 2, 10, 10, 0, 0)) == 1
    assert _norm(lib, Tensor(FAKE + 1, 10, 10, 1, 0)) == 1
    assert _norm(lib, Tensor(FAKE, (1 << 44) + 1, 0, 0, 0)) == 1


def test_clip_and_gather_refusals(lib):
    need = lib.liec_grads_workspace(2, 2)

    def clip(ts, bound=1.0, N=2):
        arr = (Tensor * len(ts))(*ts)
        return lib.liec_clip_grads(arr, len(ts), N, bound, None, FAKE, need, None)

    def gather(ts, rows, stride, bound=1.0, N=2):
        arr = (Tensor * len(ts))(*ts)
        return lib.liec_gather_grads(arr, len(ts), N, rows, stride, bound, None, FAKE, need, None)

    t = Tensor(FAKE, 10, 10, 0, 0)
    assert clip([t], -0.5) == 1
    assert clip([t], float("nan")) == 1
    assert clip([Tensor(FAKE, 10, 9, 0, 0)]) == 1            # workers overlap
    assert clip([t, Tensor(FAKE + 36, 10, 10, 0, 0)]) == 1   # tensors overlap
    assert clip([t, Tensor(FAKE + 40, 10, 10, 0, 0)]) == 1   # the second worker of one is the first of the other
    assert clip([Tensor(FAKE, 10, 40, 0, 0), Tensor(FAKE + 40, 10, 40, 0, 0), Tensor(FAKE + 76, 10, 40, 0, 0)]) == 1     # columns of a matrix
    assert clip([Tensor(FAKE, 10, 40, 0, 0), Tensor(FAKE + 128, 10, 40, 0, 0)]) == 1     # one reaches into the next row
    assert clip([Tensor(FAKE, 10, 40, 0, 0), Tensor(FAKE + 40, 10, 41, 0, 0)]) == 1      # other distances: taken to meet
    assert clip([Tensor(FAKE, 3, 0, 0, 0)]) == 1
    far = 1 << 30
    assert gather([t], None, 10) == 1
    assert gather([t], far + 2, 10) == 1
    assert gather([t], far, 9) == 1
    assert gather([t], far, 10, -1.0) == 1
    assert gather([t], FAKE + 40, 10) == 1                   # the rows start inside the tensor
    assert gather([Tensor(FAKE + 39, 10, 40, 2, 0)], FAKE, 10) == 1      # misaligned
    assert gather([Tensor(FAKE + 38, 10, 40, 2, 0)], FAKE, 20) == 1      # a fp16 tensor that reaches into every row


def test_layer_norm_refusals(lib):
    r, w = Rows(FAKE, 640, 64), Param(FAKE, 64)
    far = Rows(1 << 30, 640, 64)
    ref = ctypes.byref

    def forward(x=r, y=far, weight=w, N=2, R=10, C=64, eps=1e-5, dtype=0, ptype=0, mean=FAKE):
        return lib.liec_layer_norm(ref(x) if x else None, ref(weight) if weight else None, None, ref(y) if y else None, mean, None, N, R, C, eps, dtype,
                                   ptype, None)

    assert forward(x=None) == 1
    assert forward(y=None) == 1
    assert forward(x=Rows(None, 640, 64)) == 1
    assert forward(x=Rows(FAKE + 2, 640, 64)) == 1
    assert forward(N=0) == 1
    assert forward(N=65_536) == 1
    assert forward(R=-1) == 1
    assert forward(C=0) == 1
    assert forward(eps=-1.0) == 1
    assert forward(eps=float("nan")) == 1
    assert forward(dtype=3) == 1
    assert forward(ptype=-1) == 1
    assert forward(weight=Param(FAKE + 2, 64)) == 1
    assert forward(mean=FAKE + 2) == 1
    assert forward(y=Rows(FAKE, 640, 65)) == 1               # the same start, other strides
    assert forward(y=Rows(FAKE + 64, 640, 64)) == 1          # dense, and they overlap
    assert forward(y=Rows(1 << 30, 640, 63)) == 1            # rows of y overlap
    assert forward(y=Rows(1 << 30, 0, 64)) == 1
    assert forward(y=Rows(1 << 30, 64, 64)) == 1
    assert forward(y=Rows(1 << 30, 32, 128)) == 1
    assert forward(x=Rows(FAKE, -(1 << 63), 64)) == 1
    assert forward(weight=Param(FAKE, -(1 << 63))) == 1
    assert forward(C=(1 << 28) + 1) == 1
    assert forward(R=0) == 0                                 # no rows: nothing is looked at

    need = lib.liec_layer_norm_workspace(2, 10, 64)

    def backward(dy=r, x=r, mean=FAKE, dx=far, dw=w, db=None, N=2, R=10, C=64, ws=FAKE, bytes=need):
        return lib.liec_layer_norm_backward(ref(dy) if dy else None, ref(x) if x else None, mean, FAKE, None, ref(dx) if dx else None,
                                            ref(dw) if dw else None, ref(db) if db else None, N, R, C, 0, 0, ws, bytes, None)

    assert backward(dy=None) == 1
    assert backward(x=None) == 1
    assert backward(mean=None) == 1
    assert backward(dx=Rows(FAKE + 64, 640, 64)) == 1
    assert backward(dx=Rows(1 << 30, 0, 64)) == 1
    assert backward(db=w) == 1                               # one place for both gradients
    assert backward(ws=None) == 1
    assert backward(bytes=need - 1) == 1
    assert backward(dw=Param(FAKE, 63)) == 1                 # workers' gradients overlap
    assert backward(db=Param(FAKE, 0)) == 1                  # one shared, one not
    assert backward(N=0) == 1


def test_binding_refuses_what_is_not_on_a_gpu_or_not_a_tensor(pkg):
    import torch

    x = torch.ones(2, 3, 8)
    for bad in (lambda: pkg.liec_layer_norm(x),
                lambda: pkg.liec_layer_norm(None),
                lambda: pkg.liec_layer_norm([1.0]),
                lambda: pkg.liec_layer_norm(x.double()),
                lambda: pkg.liec_layer_norm(x, eps="small"),
                lambda: pkg.liec_layer_norm_backward(x, x, x[..., 0], x[..., 0]),
                lambda: pkg.liec_layer_norm_backward(x, x, None, x[..., 0]),
                lambda: pkg.liec_grad_norm([x]),
                lambda: pkg.liec_grad_norm([1.0]),
                lambda: pkg.liec_grad_norm(3),
                lambda: pkg.liec_grad_norm(x),                # one tensor where a list is expected
                lambda: pkg.liec_clip_grads([x], "1"),
                lambda: pkg.liec_gather_grads([x], None)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(ValueError):
        pkg.liec_grad_norm([])
    with pytest.raises(ValueError):
        pkg.liec_grad_norm([x], workers=2)
    with pytest.raises(TypeError):
        pkg.train.native().grad_norm()
