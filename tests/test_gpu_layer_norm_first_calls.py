"""The layer norm's calls whose blocks need just more shared memory than a launch gets unasked, as the first ones of a process: each
goes to a kernel that no earlier call of other sizes has been through."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import sys
import torch
from paper_2207_09682_b200 import binding
ctx, rows = binding.Context(binding.make_params()), int(sys.argv[1])
for dtype, dim, backward in ((torch.float32, 3068, False), (torch.bfloat16, 6136, False), (torch.bfloat16, 6144, False), (torch.float16, 5128, False),
                             (torch.bfloat16, 3064, True), (torch.float16, 2568, True)):
    x, g = torch.randn((rows, dim), device="cuda").to(dtype), torch.randn((rows, dim), device="cuda").to(dtype)
    mean = x.double().mean(1)
    rstd = (x.double().var(1, unbiased=False) + 1e-5).rsqrt()
    xh = (x.double() - mean[:, None]) * rstd[:, None]
    # twice a rounding to the type, and 2^-12 of a unit for the sums of single precision
    def near(got, want):
        return bool(((got.double() - want).abs() <= torch.finfo(dtype).eps * want.abs() + 2.0 ** -12).all())
    if not backward:
        assert near(ctx.layer_norm(x).out, xh), (dtype, dim)
        continue
    want = (g.double() - g.double().mean(1, keepdim=True) - xh * (g.double() * xh).mean(1, keepdim=True)) * rstd[:, None]
    assert near(ctx.layer_norm_backward(g, x, mean.float(), rstd.float())[0], want), (dtype, dim)
print("fine")
"""


@pytest.mark.parametrize("rows", [100, 3000])
def test_first_calls_of_a_process(rows):
    """Fewer rows than the GPU holds at once, and more."""
    run = subprocess.run([sys.executable, "-c", PROGRAM, str(rows)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "fine", run.stdout + run.stderr
