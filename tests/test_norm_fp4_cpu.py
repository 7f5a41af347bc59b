"""Without a GPU: what the norm's and the 4-bit operands' entry points refuse, before anything is launched, and the plain
implementations that the GPU tests compare with."""
import math

import pytest
import torch

import fp4_reference as R
from paper_2409_12517_b200 import binding as B
from paper_2409_12517_b200 import build as libbuild

P = 4096            # a pointer that is aligned to everything; refused calls never follow it


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return B.lib()


@pytest.fixture(autouse=True)
def nothing_launched(lib):
    before = lib.fp8mlp_launch_count()
    yield
    assert lib.fp8mlp_launch_count() == before


def test_norm_refusals(lib):
    def norm(T=4, d=64, dt=B.BF16, x=P, ldx=64, res=None, ldr=64, h=None, ldh=64, gain=P, eps=1e-5, out=B.RMS_SAME, y=8 * P, ldy=64,
             scale=None, amax=None, rstd=None):
        return lib.fp8mlp_rmsnorm(T, d, dt, x, ldx, res, ldr, h, ldh, gain, eps, out, y, ldy, scale, amax, rstd, None)
    for bad in (dict(dt=2), dict(dt=-1), dict(out=3), dict(out=-1), dict(h=P), dict(x=None), dict(y=None), dict(eps=-1.0),
                dict(eps=math.nan), dict(out=B.RMS_E4M3), dict(out=B.RMS_E4M3_ROWS), dict(out=B.RMS_E4M3_ROWS, scale=P, amax=P)):
        assert norm(**bad) == B.ERR_ARG, bad
    for bad in (dict(T=-1), dict(d=0), dict(d=24), dict(d=B.MAX_NORM_WIDTH + 16), dict(ldx=48), dict(ldx=68), dict(ldy=0),
                dict(res=P, ldr=60), dict(res=P, h=P, ldh=-64), dict(out=B.RMS_E4M3, scale=P, ldy=72)):
        assert norm(**bad) == B.ERR_SHAPE, bad
    for bad in (dict(x=P + 8), dict(y=8 * P + 2), dict(gain=P + 4), dict(res=P + 8), dict(res=P, h=P + 8), dict(rstd=P + 2),
                dict(amax=P + 1), dict(out=B.RMS_E4M3, scale=P + 2)):
        assert norm(**bad) == B.ERR_ALIGN, bad
    assert norm(T=0, x=None, y=None) == B.OK
    # outputs that overlap an input or each other
    for bad in (dict(y=P, x=P), dict(y=P, x=2 * P, res=P), dict(y=P, x=2 * P, res=3 * P, h=P)):
        assert norm(**bad) == B.ERR_ARG, bad


def test_norm_in_place_refuses_other_row_strides(lib):
    """A row of the output would lie over another row of the input than its own.  (Refused before anything is launched.)"""
    def norm(T=4, x=P, ldx=64, res=2 * P, ldr=64, h=3 * P, ldh=64):
        return lib.fp8mlp_rmsnorm(T, 64, B.BF16, x, ldx, res, ldr, h, ldh, None, 1e-5, B.RMS_SAME, 8 * P, 64, None, None, None, None)

    def back(T=4, dy=P, lddy=64, dh=2 * P, lddh=64, dx=3 * P, lddx=64):
        return lib.fp8mlp_rmsnorm_backward(T, 64, B.BF16, dy, lddy, 4 * P, 64, None, P, dh, lddh, dx, lddx, None, None, None)
    for bad in (dict(h=P, ldx=128), dict(h=P, ldh=128), dict(h=2 * P, ldr=72), dict(h=2 * P, ldh=80), dict(x=2 * P, h=2 * P, ldr=128)):
        assert norm(**bad) == B.ERR_ARG, bad
    for bad in (dict(dx=P, lddx=128), dict(dx=P, lddy=72), dict(dx=2 * P, lddx=80), dict(dx=2 * P, lddh=128), dict(dy=2 * P, dx=2 * P, lddy=128)):
        assert back(**bad) == B.ERR_ARG, bad


def test_norm_backward_refusals(lib):
    def back(T=4, d=64, dt=B.BF16, dy=P, lddy=64, h=2 * P, ldh=64, gain=P, rstd=P, dh=None, lddh=64, dx=P, lddx=64, dg=None, ws=None):
        return lib.fp8mlp_rmsnorm_backward(T, d, dt, dy, lddy, h, ldh, gain, rstd, dh, lddh, dx, lddx, dg, ws, None)
    for bad in (dict(dt=7), dict(dg=P), dict(dy=None), dict(h=None), dict(rstd=None), dict(dx=None), dict(dx=2 * P)):
        assert back(**bad) == B.ERR_ARG, bad
    for bad in (dict(T=-1), dict(d=8), dict(d=B.MAX_NORM_WIDTH + 16), dict(lddy=32), dict(ldh=60), dict(lddx=63), dict(dh=P, lddh=1)):
        assert back(**bad) == B.ERR_SHAPE, bad
    for bad in (dict(dy=P + 8), dict(h=P + 2), dict(dx=P + 4), dict(dh=P + 8), dict(gain=P + 4), dict(rstd=P + 2), dict(dg=P + 2, ws=P),
                dict(dg=P, ws=P + 8)):
        assert back(**bad) == B.ERR_ALIGN, bad
    assert back(T=0, dy=None, h=None, rstd=None, dx=None) == B.OK


def test_fp4_refusals(lib):
    def quant(src=P, dt=B.BF16, rows=4, cols=40, ld=40, t=0, fmt=B.NVFP4, mode=B.SCALE_GIVEN, scale=P, amax=None, codes=P, ldc=32, bs=P):
        return lib.fp8mlp_quantize_fp4(src, dt, rows, cols, ld, t, fmt, mode, scale, amax, codes, ldc, bs, None)
    current = B.SCALE_FROM_CURRENT_AMAX
    for bad in (dict(dt=3), dict(fmt=2), dict(mode=2), dict(scale=None), dict(mode=current), dict(fmt=B.MXFP4), dict(src=None),
                dict(fmt=B.MXFP4, scale=None, mode=current, amax=P), dict(codes=None), dict(bs=None)):
        assert quant(**bad) == B.ERR_ARG, bad
    for bad in (dict(rows=-1), dict(cols=-1), dict(ld=39), dict(ldc=16), dict(ldc=40), dict(rows=40, t=1, ldc=16), dict(rows=1 << 25)):
        assert quant(**bad) == B.ERR_SHAPE, bad
    for bad in (dict(src=P + 1), dict(src=P + 2, dt=B.F32), dict(codes=P + 8), dict(bs=P + 4), dict(scale=P + 2), dict(amax=P + 2)):
        assert quant(**bad) == B.ERR_ALIGN, bad

    def back(codes=P, ldc=32, bs=P, scale=None, rows=4, cols=40, fmt=B.NVFP4, out=P, dt=B.BF16, ld=40):
        return lib.fp8mlp_dequantize_fp4(codes, ldc, bs, scale, rows, cols, fmt, out, dt, ld, None)
    for bad in (dict(fmt=5), dict(dt=5), dict(fmt=B.MXFP4, scale=P), dict(codes=None), dict(bs=None), dict(out=None)):
        assert back(**bad) == B.ERR_ARG, bad
    for bad in (dict(rows=-1), dict(cols=-4), dict(ld=39), dict(ldc=16), dict(ldc=33)):
        assert back(**bad) == B.ERR_SHAPE, bad
    for bad in (dict(codes=P + 8), dict(bs=P + 8), dict(out=P + 1), dict(out=P + 2, dt=B.F32), dict(scale=P + 1)):
        assert back(**bad) == B.ERR_ALIGN, bad
    assert back(rows=0) == B.OK and back(cols=0, ldc=0) == B.OK

    def gemm(M=4, N=8, K=40, fmt=B.NVFP4, a=P, lda=32, sa=P, ga=None, b=P, ldb=32, sb=P, gb=None, out=P, dt=B.BF16, ld=8):
        return lib.fp8mlp_gemm_fp4(M, N, K, fmt, a, lda, sa, ga, b, ldb, sb, gb, out, dt, ld, None)
    for bad in (dict(fmt=2), dict(dt=2), dict(fmt=B.MXFP4, ga=P), dict(fmt=B.MXFP4, gb=P), dict(a=None), dict(b=None), dict(sa=None),
                dict(sb=None), dict(out=None)):
        assert gemm(**bad) == B.ERR_ARG, bad
    for bad in (dict(M=-1), dict(N=-1), dict(K=0), dict(lda=16), dict(ldb=40), dict(ld=7), dict(M=1 << 25), dict(K=(1 << 24) + 1, lda=1 << 24, ldb=1 << 24)):
        assert gemm(**bad) == B.ERR_SHAPE, bad
    for bad in (dict(a=P + 8), dict(b=P + 8), dict(sa=P + 8), dict(sb=P + 4), dict(out=P + 1), dict(out=P + 2, dt=B.F32), dict(ga=P + 2), dict(gb=P + 1)):
        assert gemm(**bad) == B.ERR_ALIGN, bad
    assert gemm(M=0) == B.OK and gemm(N=0, ld=0) == B.OK
    size = lib.fp8mlp_fp4_scale_bytes
    assert size(B.MXFP4, 1, 1) == 512 and size(B.MXFP4, 129, 129) == 2048 and size(B.NVFP4, 128, 65) == 1024
    assert size(2, 1, 1) == 0 and size(B.NVFP4, -1, 1) == 0 and size(B.NVFP4, 0, 16) == 0


def test_forward_refuses_cast_x_where_nothing_is_kept(lib):
    for mode in (B.SCALE_GIVEN_X_CAST, B.SCALE_GIVEN_BOTH_CAST):
        assert lib.fp8mlp_forward_static(1, 16, 16, 0, P, P, P, P, mode, None, None, P, None) == B.ERR_ARG
        assert lib.fp8mlp_forward(None, 1, None, P, P, P, mode, None, None, P, None) == B.ERR_ARG


def test_binding_refuses(lib):
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current GPU"):
        B.fp8mlp_rmsnorm(x, None, None, 1e-5, x)
    with pytest.raises(ValueError, match="current GPU"):
        B.fp8mlp_rmsnorm_backward(x, x, None, None, None, x, None, None)
    for other in (x.half(), x[0], x.int()):
        with pytest.raises(ValueError, match="2-D bfloat16 or float32"):
            B.fp8mlp_rmsnorm(other, None, None, 1e-5, other)
        with pytest.raises(ValueError, match="2-D bfloat16 or float32"):
            B.fp8mlp_rmsnorm_backward(other, other, None, None, None, other, None, None)
    op = B.new_fp4(B.MXFP4, 4, 64, device="cpu")
    assert op.scales.numel() == 512 and op.codes.shape == (4, 32) and op.scale is None
    with pytest.raises(ValueError, match="current GPU"):
        B.fp8mlp_quantize_fp4(x, op)
    with pytest.raises(ValueError, match="contractions"):
        B.fp8mlp_gemm_fp4(op, B.new_fp4(B.MXFP4, 4, 32, device="cpu"), x)
    with pytest.raises(ValueError, match="formats"):
        B.fp8mlp_gemm_fp4(op, B.new_fp4(B.NVFP4, 4, 64, device="cpu"), x)


# ---------------------------------------------------------------- the plain implementations themselves

def test_nearest_is_nearest_with_ties_to_even():
    table = torch.tensor(R.E2M1, dtype=torch.float64)
    x = torch.cat([torch.linspace(0, 7, 1401, dtype=torch.float64), (table[:-1] + table[1:]) / 2])
    for v, got in zip(x.tolist(), R.nearest(table, x).tolist()):
        far = [abs(v - t) for t in R.E2M1]
        best = [i for i, f in enumerate(far) if f == min(far)]
        assert got == (best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1]), v
    # E4M3 against the library's cast
    x = torch.rand(20000) * 448
    assert torch.equal(R.nearest(R.E4M3_CODES[:127], x.double()).to(torch.uint8), x.to(torch.float8_e4m3fn).view(torch.uint8))


@pytest.mark.parametrize("fmt", [R.MX, R.NV])
def test_quantised_values_are_within_half_a_step(fmt):
    gen = torch.Generator().manual_seed(fmt)
    src = torch.randn(33, 71, generator=gen) * torch.exp(4 * torch.randn(33, 1, generator=gen))
    g = R.tensor_scale(float(src.abs().max())) if fmt == R.NV else 1.0
    assert fmt == R.MX or 1344 < g * float(src.abs().max()) <= 2688
    code, byte = R.quantise(src, fmt, g)
    out = R.values(code, byte, fmt, g)
    top = src.double().abs()
    top = torch.nn.functional.pad(top, (0, -71 % R.BLOCK[fmt])).view(33, -1, R.BLOCK[fmt]).amax(-1).repeat_interleave(R.BLOCK[fmt], 1)[:, :71]
    # between 4 and 6 scales' units a step is 2; the scale is within 2^-4 of top / 6, or, as a power of two, may cut 8 to 6
    # (NVFP4 scales below 2^-6 are multiples of 2^-9: up to 2^-10 off, which six units of the scale magnify)
    worst, small = ((1 / 6) * (1 + 2 ** -4), 6 * 2 ** -10 / g) if fmt == R.NV else (1 / 4, 0.0)
    assert ((out - src.double()).abs() <= worst * top + small + 1e-12).all()
    packed, tiled = R.pack_codes(code), R.tile_scales(byte)
    assert torch.equal(R.untile_scales(tiled, 33, byte.shape[1]).long(), byte)
    assert torch.equal(torch.stack([packed & 15, packed >> 4], -1).flatten(1)[:, :71].long(), code)


def test_norm_gradient_against_differences():
    gen = torch.Generator().manual_seed(0)
    h, dy, dh, gain = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((3, 32), (3, 32), (3, 32), (32,)))
    eps, step = 1e-3, 1e-6
    loss = lambda h, gain: float((R.norm(h, gain, eps)[0] * dy).sum() + (h * dh).sum())
    dx, d_gain = R.norm_backward(dy, h, gain, R.norm(h, gain, eps)[1], dh)
    for t, i in ((0, 0), (1, 7), (2, 31)):
        at = torch.zeros_like(h)
        at[t, i] = step
        assert abs((loss(h + at, gain) - loss(h - at, gain)) / (2 * step) - float(dx[t, i])) < 1e-7
    for i in (0, 15, 31):
        at = torch.zeros_like(gain)
        at[i] = step
        assert abs((loss(h, gain + at) - loss(h, gain - at)) / (2 * step) - float(d_gain[i])) < 1e-7
