"""The norm where its numbers or its shapes come to an end."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent


GAIN_GRADIENT = """
import sys, torch
sys.path[:0] = [{root!r}, {tests!r}]
import fp4_reference as R
from paper_2409_12517_b200 import binding as B
gen = torch.Generator().manual_seed(0)
for dtype in (torch.bfloat16, torch.float32):
    for pad in (0, 16 // torch.empty(0, dtype=dtype).element_size()):
        for d in (12032, 12096, 12112, 12176, 12272, 12288, 12304):
            for T in (3, 40):
                dy, h = (torch.randn(T, d + pad, generator=gen).to(dtype).cuda()[:, :d] for _ in range(2))
                rstd = torch.rand(T, generator=gen).cuda() + 0.5
                dx, d_gain = torch.empty(T, d, dtype=dtype, device="cuda"), torch.empty(d, device="cuda")
                B.fp8mlp_rmsnorm_backward(dy, h, None, rstd, None, dx, d_gain, B.new_rmsnorm_workspace(d))
                want = R.norm_backward(dy.cpu(), h.cpu(), None, rstd.cpu(), None)[1].cuda()
                sizes = (dy.double() * h.double() * rstd.double()[:, None]).abs().sum(0)
                # one rounding of h rstd, and one for each row and each block's sum
                assert ((d_gain.double() - want).abs() <= (2 * T + 20) * 2.0 ** -24 * sizes).all(), (dtype, pad, d, T)
print("fine")
"""


def test_gain_gradient_at_every_width():
    """Widths whose sums take nearly the 48 KB of shared memory that a launch has without asking, from the first call of a process on."""
    script = GAIN_GRADIENT.format(root=str(ROOT), tests=str(ROOT / "tests"))
    done = subprocess.run([sys.executable, "-c", script], capture_output=True, text=True, timeout=600)
    assert done.returncode == 0 and done.stdout.strip().endswith("fine"), done.stdout + done.stderr
