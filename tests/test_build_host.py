"""What the build makes of the compiled part of the binding."""

import os
import subprocess
import sys
import sysconfig

from paper_2605_28803_gb300 import build, qvla

SUFFIX = sysconfig.get_config_var("EXT_SUFFIX")


def test_the_compiled_calls_are_this_interpreters():
    """Named with the interpreter's tag, so that another one neither imports them nor takes them for its own."""
    assert os.path.basename(qvla._calls.__file__) == "_calls" + SUFFIX
    assert build.CALLS == qvla._calls.__file__
    assert not os.path.exists(os.path.join(build.PKG, "_calls.so"))  # (a file without a tag serves every interpreter)


def test_calls_of_another_interpreter_do_not_count_as_built():
    other = build.CALLS.replace(SUFFIX, ".cpython-399-" + SUFFIX.split("-", 2)[2])
    assert other != build.CALLS and build._stale(other)


WITHOUT = """
import importlib.abc, sys
class Missing(importlib.abc.MetaPathFinder):
    def find_spec(self, name, path=None, target=None):
        if name == "paper_2605_28803_gb300._calls":
            raise ImportError("as if it were not there")
sys.meta_path.insert(0, Missing())
import numpy as np
from paper_2605_28803_gb300 import qvla as Q
n, k = 16, 128
w = np.ones((n, k), np.float32)
wq, ws = np.zeros((n, k // 2), np.uint8), np.zeros(n, np.float32)
Q.qvla_pack_weights_host(w, Q.F32, n, k, wq=wq, wscale=ws)
assert (ws > 0).all()
codes, scales = np.zeros((n, k // 2), np.uint8), np.zeros(Q.qvla_fp4_scale_bytes(Q.MXFP4, n, k), np.uint8)
Q.qvla_fp4_pack_weights_host(w, Q.F32, n, k, fmt=Q.MXFP4, wq=codes, ws=scales)
for name in ("qvla_fp4_quantize_rows", "qvla_fp4_dequantize_rows", "qvla_gemm_fp4", "qvla_fp4_linear", "qvla_block_norm", "qvla_block_norm_fp4"):
    try:
        getattr(Q, name)(1, stream=None)
    except ImportError as e:
        print(e)
"""


def test_without_the_compiled_calls_the_others_work():
    """What needs CPython's headers to build is missed by the calls that it is, and by no other."""
    run = subprocess.run([sys.executable, "-c", WITHOUT], capture_output=True, text=True, cwd=os.path.dirname(build.PKG))
    assert run.returncode == 0, run.stderr
    assert run.stdout.count("as if it were not there") == 6 and "qvla_block_norm_fp4()" in run.stdout


def test_a_build_without_cpythons_headers(monkeypatch, tmp_path, capsys):
    def never(*a, **kw):
        raise AssertionError("nothing is compiled")

    monkeypatch.setattr(build.sysconfig, "get_paths", lambda: {"include": str(tmp_path)})
    monkeypatch.setattr(build.subprocess, "run", never)
    build._build_calls()
    assert "Python.h" in capsys.readouterr().err
