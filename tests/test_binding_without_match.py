"""The package without its _match: a build that has no C compiler or headers for this interpreter, an interpreter that it was not built
for.  Each call is then made anew."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
import sys
sys.path[:0] = [%r, %r]
sys.modules["paper_2107_06960_gb300._match"] = None  # as if it were not there
import torch
import paper_2107_06960_gb300 as mf
from test_operator_tensors import OnGpu
assert mf.version() and mf.Net([("conv", 3, 1, 1, 8)], 16, 16, 3).shape(0)
from test_draft_operators import _calls
mf._current_device = lambda: 0
for which, (entry, call, tensors) in _calls(mf).items():
    if which in ("rotary", "tree"):
        plan = [c.cell_contents for c in call.__closure__][0]
        plan.device = 0
    here, seen = {n: OnGpu(t) for n, t in tensors.items()}, []
    setattr(mf.lib, entry, lambda *a: seen.append(a) or mf.OK)
    for _ in range(3):
        call(**here)
    assert len(seen) == 3, which
    call(**{**here, **{n: OnGpu(t.clone()) for n, t in tensors.items()}})
    assert len(seen) == 4
    try:
        call(**{**here, list(tensors)[0]: list(tensors.values())[0]})
    except mf.MafatError:
        continue
    raise AssertionError("taken from the host")
print("ok")
"""


def test_calls():
    pytest.importorskip("torch")
    import __graft_entry__ as g
    g.build()
    r = subprocess.run([sys.executable, "-c", CALLS % (ROOT, os.path.join(ROOT, "tests"))], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr


@pytest.mark.parametrize("how", ["no compiler", "no headers"])
def test_builds(monkeypatch, tmp_path, how):
    """The library is built all the same, what an earlier build left is taken away, and the build says so."""
    import __graft_entry__ as g
    b = g._load_module("_build_alone", os.path.join(ROOT, "paper_2107_06960_gb300", "build.py"))
    there = tmp_path / "_match.so"
    there.write_bytes(b"of an earlier build")
    os.utime(there, (1, 1))
    monkeypatch.setattr(b, "MATCH", str(there))
    run = subprocess.run

    def fake(cmd, **kw):
        if not any(str(c).endswith("match.c") for c in cmd):
            return run(cmd, **kw)
        if how == "no compiler":
            raise FileNotFoundError(2, "gcc")
        return subprocess.CompletedProcess(cmd, 1, "", "fatal error: Python.h: No such file or directory")
    monkeypatch.setattr(b.subprocess, "run", fake)
    with pytest.warns(RuntimeWarning, match="_match"):
        lib = b.build()
    assert os.path.exists(lib) and not there.exists()
