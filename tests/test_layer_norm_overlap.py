"""Outputs of the layer norm that overlap its inputs, without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_outputs_that_overlap_inputs_are_refused(tmp_path):
    out = str(tmp_path / "overlap")
    csrc = os.path.join(ROOT, "paper_2207_09682_b200", "csrc")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-O1", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "none",
                           "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "api_ops.cu"), os.path.join(csrc, "api_train_ops.cu"),
                           os.path.join(ROOT, "tests", "host", "layer_norm_overlap.cu"), os.path.join(ROOT, "tests", "host", "fake_cuda.cpp"), "-o", out])
    run = subprocess.run([out], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout[-4000:]
