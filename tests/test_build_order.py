"""What build() needs for which part: a binding that cannot be compiled leaves the step's library and the oracle built, and g++ is
not the only compiler that will do."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)


def test_a_binding_that_fails_leaves_the_rest_built(monkeypatch):
    import oracle
    import __graft_entry__ as entry
    from paper_2402_11857_amd import _build

    done = []

    def fails(**_):
        raise RuntimeError("the binding did not compile")

    monkeypatch.setattr(_build, "build_library", lambda **_: done.append("library") or __file__)
    monkeypatch.setattr(_build, "build_binding", fails)
    monkeypatch.setattr(oracle, "build", lambda **_: done.append("oracle"))
    monkeypatch.setattr(oracle, "build_all_cores", lambda **_: done.append("oracle of all cores"))
    with pytest.raises(RuntimeError, match="binding"):
        entry.build()
    assert done == ["library", "oracle", "oracle of all cores"]


@pytest.mark.parametrize("absent", [("g++",), ("g++", "c++")])
def test_other_compilers_are_taken(monkeypatch, absent):
    from paper_2402_11857_amd import _build

    which, ran = shutil.which, []
    monkeypatch.setattr(shutil, "which", lambda name, *a, **kw: None if os.path.basename(name) in absent else which(name, *a, **kw))
    monkeypatch.setattr(subprocess, "run", lambda cmd, **_: ran.append(cmd) or subprocess.CompletedProcess(cmd, 0, "", ""))
    assert _build.build_binding() == _build.BINDING_PATH
    assert len(ran) == 1 and os.path.exists(ran[0][0]) and os.path.basename(ran[0][0]) not in absent


def test_missing_headers_of_python_are_named(monkeypatch, tmp_path):
    import sysconfig

    from paper_2402_11857_amd import _build

    monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **kw: {"include": str(tmp_path)})
    with pytest.raises(RuntimeError, match="Python.h"):
        _build.build_binding()
