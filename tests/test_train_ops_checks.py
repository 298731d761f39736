"""Argument checks of the layer norm and of the AdamW step, without a GPU."""
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_c_calls_refuse_what_they_cannot_take(tmp_path):
    out = str(tmp_path / "train_ops")
    csrc = os.path.join(ROOT, "paper_2207_09682_b200", "csrc")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-O1", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "none",
                           "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "api_ops.cu"), os.path.join(csrc, "api_train_ops.cu"),
                           os.path.join(ROOT, "tests", "host", "train_ops.cu"), os.path.join(ROOT, "tests", "host", "fake_cuda.cpp"), "-o", out])
    run = subprocess.run([out], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout + run.stderr


def test_states_before_the_first_step():
    from paper_2207_09682_b200 import binding
    params = [torch.ones(n) for n in (1, 256, 257)] + [torch.ones((3, 100))]
    m, v, none = binding.adamw_states(params)
    assert none is None and all(t.dtype == torch.float32 and not t.any() for t in m + v)
    m, v, e = binding.adamw_states(iter(params), bits=8)
    assert all(t.dtype == torch.uint8 and not t.any() for t in m + v + e)
    assert [tuple(t.shape) for t in m] == [tuple(p.shape) for p in params] and [tuple(t.shape) for t in e] == [(1, 2), (1, 2), (2, 2), (2, 2)]
    with pytest.raises(binding.QgbdtError):
        binding.adamw_states(params, bits=16)


def test_tensors_that_are_not_on_the_device_are_refused():
    """By the module that takes them apart, before the library is called."""
    from paper_2207_09682_b200 import binding
    binding.load_library()
    ctx = binding.Context.__new__(binding.Context)
    ctx.h, ctx.device = binding.C.c_void_p(), 0
    x = torch.ones((3, 4))
    calls = [
        lambda: ctx.layer_norm(x), lambda: ctx.layer_norm([1.0]), lambda: ctx.layer_norm_backward(x, x, x[:, 0], x[:, 0]),
        lambda: ctx.adamw([x], [x], [x], [x], 1, 0.1), lambda: ctx.adamw([x], [], [x], [x], 1, 0.1), lambda: ctx.adamw_values([x], [x], [x]),
        lambda: ctx.adamw_values([], [], [], dtype=torch.float16),
    ]
    for call in calls:
        with pytest.raises((binding.QgbdtError, RuntimeError)) as e:
            call()
        if isinstance(e.value, binding.QgbdtError):
            assert e.value.code == binding.ERR_ARG
