"""The extension module of the operators: trees do without it, and it is rebuilt for another torch or Python."""
import os
import shutil
import subprocess
import sys

from paper_2207_09682_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_library_loads_without_the_tensors_module(tmp_path):
    build.build()
    package = tmp_path / "paper_2207_09682_b200"
    package.mkdir()
    for name in ("__init__.py", "binding.py", "libqgbdt.so"):
        shutil.copy(os.path.join(ROOT, "paper_2207_09682_b200", name), package / name)
    code = ("from paper_2207_09682_b200 import binding\n"
            "lib = binding.load_library()\n"
            "assert lib.qgbdt_destroy(None) == binding.ERR_ARG\n"
            "ctx = binding.Context.__new__(binding.Context)\n"
            "ctx.h, ctx.device = binding.C.c_void_p(), 0\n"
            "try:\n"
            "    ctx.embed(None, None)\n"
            "except ImportError as e:\n"
            "    assert '_tensors.so is not built' in str(e)\n"
            "else:\n"
            "    raise SystemExit('an operator ran without its module')\n")
    subprocess.run([sys.executable, "-c", code], cwd=tmp_path, env={**os.environ, "PYTHONPATH": str(tmp_path)}, check=True)


def test_the_tensors_module_is_rebuilt_for_another_torch_or_python(monkeypatch):
    import platform

    import torch
    build.build()
    assert not build.tensors_stale()
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "0.0.0")
        assert build.tensors_stale()
    with monkeypatch.context() as m:
        m.setattr(platform, "python_version", lambda: "0.0.0")
        assert build.tensors_stale()
    with monkeypatch.context() as m:
        m.setattr(build, "TENSORS_MADE_FOR", build.TENSORS_MADE_FOR + ".absent")
        assert build.tensors_stale()
    assert not build.tensors_stale()
