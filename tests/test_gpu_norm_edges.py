"""The norm where its numbers or its shapes come to an end."""
import subprocess
import sys
from pathlib import Path

import pytest
import torch

import fp4_reference as R
from paper_2409_12517_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
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


@pytest.mark.parametrize("out", [B.RMS_SAME, B.RMS_E4M3, B.RMS_E4M3_ROWS])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 4096])
def test_rows_of_tiny_numbers_without_eps(d, dtype, out):
    """eps = 0 and rows down to 2^-68: 1 / rms has no square in fp32, but is a number, and so are maximum and scale.
    Squares are fp32 numbers, for fp32 rows to codes 64-bit ones: each of the d squares and of the sums is off by half of the
    smallest number (2^-150) at most, beside the roundings counted in test_gpu_norm.py (32 for 1 / rms, 4 more for the scale)."""
    gen = torch.Generator().manual_seed(d)
    tops = torch.tensor([1.0, 2.0 ** -40, 2.0 ** -60, 2.0 ** -64, 2.0 ** -66, 2.0 ** -68])
    x = (torch.randn(6, d, generator=gen) * tops[:, None]).to(dtype).cuda()
    want, want_rstd = R.norm(x.cpu(), None, 0.0)
    want, want_rstd = want.cuda(), want_rstd.cuda()
    y = torch.empty_like(x) if out == B.RMS_SAME else torch.empty(6, d, dtype=torch.uint8, device="cuda")
    scale = None if out == B.RMS_SAME else torch.full((6 if out == B.RMS_E4M3_ROWS else 1,), 50.0, device="cuda")
    amax = None if out == B.RMS_E4M3_ROWS else torch.zeros(1, device="cuda")
    rstd = torch.empty(6, device="cuda")
    B.fp8mlp_rmsnorm(x, None, None, 0.0, y, out=out, scale=scale, amax=amax, rstd=rstd)
    wide = out != B.RMS_SAME and dtype == torch.float32
    low = torch.zeros_like(want_rstd) if wide else 2 * d * 2.0 ** -150 / x.double().square().sum(-1)
    off = 32 * U + low + (2.0 ** -150 * want_rstd ** 2 if out == B.RMS_SAME else 0.0)          # (there the mean is an fp32 number too)
    assert ((rstd.double() - want_rstd).abs() <= off * want_rstd).all()
    if out == B.RMS_E4M3_ROWS:
        want_scale = 448.0 / want.abs().amax(-1)
        assert ((scale.double() - want_scale).abs() <= (off + 4 * U) * want_scale).all()
        assert (y.view(torch.float8_e4m3fn).float().abs().amax(-1) == 448).all()
    else:
        top = want.abs().amax(-1)
        assert float(amax) >= float((top * (1 - off - 4 * U)).max()) and float(amax) <= float((top * (1 + off + 4 * U)).max())


def between(y, exact, slack):
    """E4M3 codes that a value within `slack` of the exact one has next to it."""
    low, high = (R.nearest(R.E4M3_CODES[:127], exact.abs() * (1 + s * slack)) for s in (-1, 1))
    got = (y & 0x7f).cpu().long()
    return ((got >= low) & (got <= high)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_codes_of_products_below_the_normal_numbers(dtype):
    """h gain below 2^-126, where an fp32 product has few bits left, and a factor that brings it back among the codes."""
    gen = torch.Generator().manual_seed(1)
    T, d = 256, 1024
    x = (torch.randn(T, d, generator=gen).sign() * torch.exp2(-116 - 12 * torch.rand(T, d, generator=gen))).to(dtype)
    gain = 2.0 ** -8 * (1 + torch.rand(d, generator=gen))
    x[:, 0] = 2.0 ** -110                                     # a row's largest: 448 / (h gain) stays in fp32
    y, own = torch.empty(T, d, dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda")
    want, _ = R.norm(x, gain, 1.0)
    given = torch.full((1,), 2.0 ** 126, device="cuda")
    B.fp8mlp_rmsnorm(x.cuda(), None, gain.cuda(), 1.0, y, out=B.RMS_E4M3, scale=given)
    assert between(y, want * 2.0 ** 126, 6 * U)
    B.fp8mlp_rmsnorm(x.cuda(), None, gain.cuda(), 1.0, y, out=B.RMS_E4M3_ROWS, scale=own)
    # the largest h gain, about 2^-118, is known to the smallest number, half of 2^-149
    assert between(y, want * (448.0 / want.abs().amax(-1, keepdim=True)), 2.0 ** -30)


def test_codes_stay_inside_a_context_s_buffer():
    """More rows than the context has room for, rows from an offset on, and addresses whose size nobody knows are refused by the call."""
    T, d = 24, 64
    ctx = B.fp8mlp_create(T, d, 64, 0)
    try:
        ptr, nbytes = B.fp8mlp_workspace(ctx, B.WS_XQ)
        assert ptr.nbytes == nbytes == T * d and (ptr + 3 * d).nbytes == (T - 3) * d
        x, scale = torch.randn(T + 1, d, device="cuda"), torch.full((1,), 50.0, device="cuda")
        whole = torch.empty(T, d, dtype=torch.uint8, device="cuda")
        B.fp8mlp_rmsnorm(x[:T], None, None, 1e-5, whole, out=B.RMS_E4M3, scale=scale)
        B.fp8mlp_rmsnorm(x[:5], None, None, 1e-5, ptr, out=B.RMS_E4M3, scale=scale)
        B.fp8mlp_rmsnorm(x[5:T], None, None, 1e-5, ptr + 5 * d, out=B.RMS_E4M3, scale=scale)
        assert torch.equal(B.workspace_tensor(ctx, B.WS_XQ, (T, d), torch.uint8), whole)
        for rows, y, out in ((T + 1, ptr, B.RMS_E4M3), (T, ptr + d, B.RMS_E4M3), (T, int(ptr), B.RMS_E4M3), (T, ptr + (T * d + 16), B.RMS_E4M3),
                             (1, ptr - d, B.RMS_E4M3), (1, ptr, B.RMS_SAME)):
            with pytest.raises(ValueError, match="codes go to"):
                B.fp8mlp_rmsnorm(x[:rows], None, None, 1e-5, y, out=out, scale=scale)
        assert torch.equal(B.workspace_tensor(ctx, B.WS_XQ, (T, d), torch.uint8), whole)
    finally:
        B.fp8mlp_destroy(ctx)
