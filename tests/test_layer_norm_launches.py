"""What the layer norm's launches ask for, over a stand-in for the CUDA runtime, without a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("layer_norm") / "launches")
    csrc = os.path.join(ROOT, "paper_2207_09682_b200", "csrc")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-O1", "-Xcicc", "-O0", "-Xptxas", "-O0", "-std=c++17",
                           "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "none", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                           os.path.join(csrc, "api_ops.cu"), os.path.join(csrc, "layer_norm.cu"), os.path.join(ROOT, "tests", "host", "layer_norm_launches.cu"),
                           os.path.join(ROOT, "tests", "host", "fake_cuda.cpp"), "-o", out])
    return out


@pytest.mark.parametrize("calls", ["first", "one after the other"])
def test_shared_memory_of_the_launches(program, calls):
    """first: a launch gets the shared memory that it asks for without an earlier call of other sizes.  One after the other: no
    call takes from a kernel what another call, of another thread perhaps, has asked for."""
    run = subprocess.run([program, calls], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout[-4000:]
