"""include/liec_activations.h: the library exports what it declares, it is plain C, and checks that need no GPU refuse bad arguments
and operands that share memory."""
import ctypes
import os
import re
import subprocess
import sys

import pytest

sys.path.insert(0, os.path.dirname(__file__))
from test_train_abi import FAKE, Param, Rows, lib, pkg  # noqa: E402,F401

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "liec_activations.h")
MB = 1 << 20
EINVAL = 1
fakes = pytest.mark.skipif(torch.cuda.is_available(), reason="passes addresses that no memory stands behind")


class Saved(ctypes.Structure):
    _fields_ = [("values", ctypes.c_void_p), ("exponents", ctypes.c_void_p)]


class Images(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("worker_stride", ctypes.c_int64), ("image_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


class Matrices(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("worker_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64)]


def i64(v):
    return ctypes.c_int64(v)


@pytest.fixture(scope="module")
def calls(lib):  # noqa: F811
    for name in ("liec_group_norm_workspace", "liec_weight_grad_workspace"):
        getattr(lib, name).restype = ctypes.c_int64
    return lib


def test_every_declared_symbol_is_exported_and_bound(calls):
    import paper_2402_11857_amd as package

    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(liec_[a-z0-9_]+)\s*\(", text)))
    assert len(names) == 7
    for name in names:
        assert hasattr(calls, name)
        assert hasattr(package, name) or name.endswith("_workspace")


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "use_header.c"
    src.write_text('#include "liec_activations.h"\n'
                   "int main(void) {\n"
                   "    liec_checkpoint s = {0, 0};\n"
                   "    liec_images m = {0, 0, 0, 0};\n"
                   "    liec_matrices w = {0, 0, 0};\n"
                   "    (void)s; (void)m; (void)w;\n"
                   "    return LIEC_ACT_NONE + LIEC_CHECKPOINT_COLUMNS - 32;\n"
                   "}\n")
    run = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-fsyntax-only", "-I", os.path.dirname(HEADER), str(src)],
                         capture_output=True, text=True)
    assert run.returncode == 0, run.stderr


def test_workspace_sizes(calls):
    def norm(N, B, S, C, G):
        return calls.liec_group_norm_workspace(N, i64(B), i64(S), i64(C), i64(G))

    def weight(N, R, O, C):
        return calls.liec_weight_grad_workspace(N, i64(R), i64(O), i64(C))

    for bad in ((0, 1, 1, 8, 1), (65_536, 1, 1, 8, 1), (1, -1, 1, 8, 1), (1, 1, -1, 8, 1), (1, 1, 1, 0, 1), (1, 1, 1, 8, 0), (1, 1, 1, 8, 3), (1, 1, 1, 8, 16),
                (1, 1 << 31, 1, 8, 1), (1, 1, 1 << 31, 8, 1), (1, 1, 1, (1 << 20) + 1, 1), (65_535, 65_535, 65_535, 8, 1)):
        assert norm(*bad) == -1, bad
    assert norm(2, 0, 5, 8, 2) == norm(2, 5, 0, 8, 2) == 0
    for good in ((1, 1, 1, 1, 1), (3, 2, 7, 90, 9), (16, 8, 3136, 256, 32), (4, 4, 65_536, 7, 7), (1, 1, (1 << 31) - 1, 8, 1)):
        assert norm(*good) > 0, good
    for bad in ((0, 1, 1, 1), (65_536, 1, 1, 1), (1, -1, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (1, 1, (1 << 24) + 1, 1), (1, 1, 1, (1 << 24) + 1),
                (1, 1 << 31, 1, 1), (1 << 10, 1, 1 << 20, 1 << 20), (1, 1 << 30, 1 << 20, 1)):
        assert weight(*bad) == -1, bad
    assert weight(3, 0, 5, 7) == 0 and weight(1, 1, 1, 1) == 0
    # chains of at most 8192 rows: more of them need room for their sums
    assert weight(1, 100_000, 4096, 4096) >= 12 * 4096 * 4097 * 4


class Call:
    """A valid call whose arguments can be replaced: every operand has memory of its own."""

    def __init__(self, lib, N=3, B=2, S=5, C=24, G=3):  # noqa: F811
        self.lib, self.N, self.B, self.S, self.C, self.G = lib, N, B, S, C, G
        self.need = max(16, lib.liec_group_norm_workspace(N, i64(B), i64(S), i64(C), i64(G)))
        at = iter(range(MB, 100 * MB, MB))
        image = (B * S * C, S * C, C)
        self.x, self.y, self.dy, self.dx = (Images(next(at), *image) for _ in range(4))
        self.w, self.b, self.dw, self.db = (Param(next(at), C) for _ in range(4))
        self.mean, self.rstd, self.ws = (next(at) for _ in range(3))
        self.saved = Saved(next(at), next(at))
        self.stats = N * B * G * 4

    def forward(self, **kw):
        a = dict(x=self.x, w=self.w, b=self.b, y=self.y, mean=self.mean, rstd=self.rstd, saved=None, N=self.N, B=self.B, S=self.S, C=self.C, G=self.G, eps=1e-5,
                 act=0, dtype=0, pdtype=0, ws=self.ws, bytes=self.need)
        assert set(kw) <= set(a)
        a.update(kw)
        p = lambda v: ctypes.byref(v) if v is not None else None                        # noqa: E731
        return self.lib.liec_group_norm(p(a["x"]), p(a["w"]), p(a["b"]), p(a["y"]), ctypes.c_void_p(a["mean"]), ctypes.c_void_p(a["rstd"]), p(a["saved"]), a["N"],
                                        i64(a["B"]), i64(a["S"]), i64(a["C"]), i64(a["G"]), ctypes.c_float(a["eps"]), a["act"], a["dtype"], a["pdtype"],
                                        ctypes.c_void_p(a["ws"]), i64(a["bytes"]), None)

    def backward(self, **kw):
        a = dict(dy=self.dy, x=self.x, saved=None, mean=self.mean, rstd=self.rstd, w=self.w, b=self.b, dx=self.dx, dw=self.dw, db=self.db, N=self.N, B=self.B,
                 S=self.S, C=self.C, G=self.G, act=1, dtype=0, pdtype=0, ws=self.ws, bytes=self.need)
        assert set(kw) <= set(a)
        a.update(kw)
        p = lambda v: ctypes.byref(v) if v is not None else None                        # noqa: E731
        return self.lib.liec_group_norm_backward(p(a["dy"]), p(a["x"]), p(a["saved"]), ctypes.c_void_p(a["mean"]), ctypes.c_void_p(a["rstd"]), p(a["w"]), p(a["b"]),
                                                 p(a["dx"]), p(a["dw"]), p(a["db"]), a["N"], i64(a["B"]), i64(a["S"]), i64(a["C"]), i64(a["G"]), a["act"],
                                                 a["dtype"], a["pdtype"], ctypes.c_void_p(a["ws"]), i64(a["bytes"]), None)


def moved(m, by):
    return type(m)(m.data + by, *(getattr(m, f) for f, _ in m._fields_[1:]))


@fakes
def test_group_norm_refusals(calls):
    c = Call(calls)
    assert c.forward() != EINVAL and c.forward(saved=c.saved) != EINVAL and c.forward(w=None, b=None) != EINVAL
    for kw in (dict(N=0), dict(N=65_536), dict(B=-1), dict(S=-1), dict(C=0), dict(G=5), dict(G=0), dict(act=3), dict(act=-1), dict(dtype=3), dict(pdtype=-1),
               dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")), dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(mean=c.mean + 2),
               dict(ws=None), dict(ws=c.ws + 8), dict(bytes=c.need - 1), dict(x=Images(None, 1, 1, 1)), dict(x=moved(c.x, 2)), dict(w=Param(FAKE + 2, 24)),
               dict(saved=Saved(None, FAKE)), dict(saved=Saved(FAKE, None)), dict(x=Images(FAKE, 1 << 41, 1, 1)), dict(y=Images(FAKE, 240, 120, 23)),
               dict(y=Images(FAKE, 240, 100, 24)), dict(y=Images(FAKE, 230, 120, 24))):
        assert c.forward(**kw) == EINVAL, kw
    assert c.forward(S=0) == c.forward(B=0) == 0             # nothing to do
    assert c.forward(B=0, x=None, y=None, mean=None, ws=None) == 0


@fakes
def test_group_norm_overlaps(calls):
    c = Call(calls)
    size = 3 * 2 * 5 * 24
    assert c.forward(y=c.x) != EINVAL                        # in place
    assert c.forward(y=moved(c.x, 4)) == EINVAL and c.forward(y=moved(c.x, 4 * size - 4)) == EINVAL and c.forward(y=moved(c.x, 4 * size)) != EINVAL
    assert c.forward(y=Images(c.x.data, 240, 120, 48)) == EINVAL
    # channels of wider rows: between one another
    wide = (480, 240, 48)
    assert c.forward(x=Images(MB, *wide), y=Images(MB + 96, *wide)) != EINVAL and c.forward(x=Images(MB, *wide), y=Images(MB + 92, *wide)) == EINVAL
    # images of workers that lie apart, which no two distances describe
    far = (1000, 200, 30)
    assert c.forward(x=Images(MB, *far), y=Images(MB + 1600, *far)) != EINVAL and c.forward(x=Images(MB, *far), y=Images(MB + 800, *far)) == EINVAL
    for at in (c.x.data, c.y.data + 4 * size - 4, c.w.data + 4, c.b.data):
        assert c.forward(mean=at) == EINVAL and c.forward(rstd=at) == EINVAL
        ws = at & ~15
        assert c.forward(ws=ws) == EINVAL
        assert c.forward(saved=Saved(at, c.saved.exponents)) == EINVAL and c.forward(saved=Saved(c.saved.values, at)) == EINVAL
    assert c.forward(mean=c.rstd) == EINVAL and c.forward(mean=c.rstd + c.stats) != EINVAL
    assert c.forward(saved=Saved(MB * 50, MB * 50 + size - 1)) == EINVAL and c.forward(saved=Saved(MB * 50, MB * 50 + size)) != EINVAL
    assert c.forward(y=moved(c.y, c.w.data - c.y.data)) == EINVAL
    assert c.forward(ws=c.mean & ~15) == EINVAL


@fakes
def test_group_norm_backward_refusals(calls):
    c = Call(calls)
    assert c.backward() != EINVAL and c.backward(x=None, saved=c.saved) != EINVAL and c.backward(dx=None) != EINVAL and c.backward(dw=None, db=None) != EINVAL
    assert c.backward(x=Images(None, 0, 0, 0), saved=c.saved) != EINVAL and c.backward(saved=Saved(None, None)) != EINVAL
    for kw in (dict(N=0), dict(G=5), dict(act=3), dict(dtype=3), dict(pdtype=3), dict(dy=None), dict(x=None), dict(saved=c.saved), dict(mean=None), dict(rstd=None),
               dict(rstd=c.rstd + 2), dict(ws=None), dict(bytes=c.need - 1), dict(dy=moved(c.dy, 2)), dict(dx=Images(FAKE, 240, 120, 23)), dict(dw=Param(FAKE, 23)),
               dict(db=Param(FAKE, 0)), dict(dw=Param(FAKE + 2, 24)), dict(x=None, saved=Saved(FAKE, None))):
        assert c.backward(**kw) == EINVAL, kw
    assert c.backward(dw=Param(c.dw.data, 0), db=Param(c.db.data, 0)) != EINVAL
    # in place of dy or x, and nowhere else
    assert c.backward(dx=c.dy) != EINVAL and c.backward(dx=c.x) != EINVAL
    for m in (c.dy, c.x):
        assert c.backward(dx=moved(m, 4)) == EINVAL and c.backward(dx=moved(m, -4)) == EINVAL
    for at in (c.mean, c.rstd, c.w.data, c.b.data):
        assert c.backward(dx=moved(c.dx, at - c.dx.data)) == EINVAL
    for p in ("dw", "db"):
        for at in (c.dy.data, c.x.data, c.dx.data, c.mean, c.rstd, c.ws, c.w.data, c.b.data, c.dw.data if p == "db" else c.db.data):
            assert c.backward(**{p: Param(at, 24)}) == EINVAL, (p, at)
    for at in (c.dy.data, c.x.data, c.dx.data, c.mean, c.w.data, c.dw.data):
        assert c.backward(ws=at) == EINVAL
    for at in (c.dx.data, c.dw.data, c.ws):
        assert c.backward(x=None, saved=Saved(at, c.saved.exponents)) == EINVAL and c.backward(x=None, saved=Saved(c.saved.values, at)) == EINVAL


@fakes
def test_checkpoint_refusals(calls):
    rows, saved, size = Rows(MB, 240, 24), Saved(2 * MB, 3 * MB), 3 * 10 * 24

    def save(x=rows, s=saved, N=3, R=10, C=24, dtype=0):
        return calls.liec_checkpoint_save(ctypes.byref(x) if x else None, ctypes.byref(s) if s else None, N, i64(R), i64(C), dtype, None)

    def load(s=saved, y=rows, N=3, R=10, C=24, dtype=0):
        return calls.liec_checkpoint_load(ctypes.byref(s) if s else None, ctypes.byref(y) if y else None, N, i64(R), i64(C), dtype, None)

    for f, x in ((save, "x"), (load, "y")):
        assert f() != EINVAL and f(R=0) == 0
        for kw in (dict(N=0), dict(N=65_536), dict(R=-1), dict(R=1 << 31), dict(C=0), dict(C=(1 << 28) + 1), dict(dtype=3), dict(s=None), dict(s=Saved(None, FAKE)),
                   dict(s=Saved(FAKE, None)), {x: None}, {x: Rows(None, 240, 24)}, {x: Rows(MB + 2, 240, 24)}, {x: Rows(MB, 1 << 41, 24)},
                   dict(s=Saved(MB, 3 * MB)), dict(s=Saved(2 * MB, MB + 4 * size - 1))):
            assert f(**kw) == EINVAL, kw
        assert f(s=Saved(2 * MB, MB + 4 * size)) != EINVAL
    assert save(s=Saved(2 * MB, 2 * MB + size - 1)) == EINVAL and save(s=Saved(2 * MB, 2 * MB + size)) != EINVAL
    assert save(x=Rows(MB, 0, 24)) != EINVAL                 # one worker's rows for all
    assert load(y=Rows(MB, 0, 24)) == EINVAL and load(y=Rows(MB, 240, 23)) == EINVAL


@fakes
def test_weight_grad_refusals(calls):
    N, R, O, C = 3, 10, 20, 40
    need = calls.liec_weight_grad_workspace(N, i64(R), i64(O), i64(C))
    dy, saved, dw, db, ws = Rows(MB, R * O, O), Saved(2 * MB, 3 * MB), Matrices(4 * MB, O * C, C), Param(5 * MB, O), 6 * MB

    def grad(dy=dy, s=saved, dw=dw, db=db, N=N, R=R, O=O, C=C, dtype=0, pdtype=0, ws=ws, bytes=need):
        p = lambda v: ctypes.byref(v) if v is not None else None                        # noqa: E731
        return calls.liec_weight_grad(p(dy), p(s), p(dw), p(db), N, i64(R), i64(O), i64(C), dtype, pdtype, ctypes.c_void_p(ws), i64(bytes), None)

    assert grad() != EINVAL and grad(db=None) != EINVAL and grad(db=Param(None, 0)) != EINVAL
    for kw in (dict(N=0), dict(R=-1), dict(O=0), dict(C=0), dict(dtype=3), dict(pdtype=3), dict(dy=None), dict(s=None), dict(dw=None), dict(dy=Rows(MB + 2, 200, 20)),
               dict(dw=Matrices(None, 800, 40)), dict(dw=Matrices(4 * MB + 2, 800, 40)), dict(dw=Matrices(4 * MB, 0, 40)), dict(dw=Matrices(4 * MB, 800, 39)),
               dict(dw=Matrices(4 * MB, 790, 40)), dict(db=Param(5 * MB, 0)), dict(db=Param(5 * MB + 2, 20)), dict(dw=Matrices(MB, 800, 40)),
               dict(dw=Matrices(2 * MB, 800, 40)), dict(dw=Matrices(3 * MB, 800, 40)), dict(db=Param(MB, 20)), dict(db=Param(2 * MB, 20)), dict(db=Param(3 * MB, 20)),
               dict(db=Param(4 * MB + 400, 20))):
        assert grad(**kw) == EINVAL, kw
    many = calls.liec_weight_grad_workspace(1, i64(100_000), i64(O), i64(C))
    big = dict(N=1, R=100_000, dy=Rows(100 * MB, 0, O), s=Saved(200 * MB, 300 * MB))
    assert grad(**big, bytes=many) != EINVAL
    for kw in (dict(bytes=many - 1), dict(bytes=many, ws=None), dict(bytes=many, ws=ws + 8), dict(bytes=many, ws=4 * MB), dict(bytes=many, ws=5 * MB),
               dict(bytes=many, ws=100 * MB), dict(bytes=many, ws=200 * MB)):
        assert grad(**{**big, **kw}) == EINVAL, kw


def test_python_refuses_what_is_not_on_the_gpu(pkg):  # noqa: F811
    x, w = torch.zeros(2, 3, 4, 16), torch.ones(2, 16)
    saved = pkg.Checkpoint(torch.zeros(2, 3, 4, 16, dtype=torch.int8), torch.zeros(2, 3, 4, 1, dtype=torch.uint8))
    for call in (lambda: pkg.liec_checkpoint_save(x), lambda: pkg.liec_checkpoint_load(saved), lambda: pkg.liec_group_norm(x, 4, w, w),
                 lambda: pkg.liec_group_norm_backward(x, x, x, x, w, w), lambda: pkg.liec_weight_grad(x, saved), lambda: pkg.liec_checkpoint_save([1.0]),
                 lambda: pkg.liec_checkpoint_load(x), lambda: pkg.liec_group_norm(None, 4)):
        with pytest.raises(TypeError):
            call()
    for name in ("gelu", None, 1, ["relu"]):
        with pytest.raises(ValueError, match="activation"):
            pkg.liec_group_norm(x, 4, activation=name)
