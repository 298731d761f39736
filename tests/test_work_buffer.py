"""The operators' work buffer over a stand-in for the CUDA runtime: order between streams, growth, captured graphs, failures."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("work_buffer") / "work_buffer")
    csrc = os.path.join(ROOT, "paper_2207_09682_b200", "csrc")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-O1", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "none",
                           "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "api_ops.cu"),
                           os.path.join(ROOT, "tests", "host", "work_buffer.cu"), os.path.join(ROOT, "tests", "host", "fake_cuda.cpp"), "-o", out])
    return out


@pytest.mark.parametrize("scenario", ["streams", "grow", "grow after a capture", "grow twice after a capture", "one capture", "two captures"])
def test_work_buffer(program, scenario):
    run = subprocess.run([program, scenario], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout


@pytest.mark.parametrize("scenario", ["failure", "no host memory"])
def test_work_buffer_failures(program, scenario):
    run = subprocess.run([program, scenario], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout + run.stderr
