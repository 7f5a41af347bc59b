"""4-bit operands on the GPU: codes and scales bit for bit, products within their roundings of 64-bit sums."""
import math

import pytest
import torch

import fp4_reference as R
from paper_2409_12517_b200 import binding as B

pytestmark = pytest.mark.gpu
FORMATS = [B.MXFP4, B.NVFP4]


def matrix(rows, cols, dtype, pad=0, offset=0, seed=0):
    """[rows, cols] over several binades with ties, zeros and all-zero stretches, in rows of cols + pad elements."""
    gen = torch.Generator().manual_seed(seed)
    v = torch.randn(rows, cols, generator=gen) * torch.exp2(torch.randint(-6, 7, (rows, 1), generator=gen).float())
    v = torch.where(torch.rand(rows, cols, generator=gen) < 0.3, torch.randint(-24, 25, (rows, cols), generator=gen) / 4.0, v)
    v = torch.where(torch.rand(rows, 1, generator=gen) < 0.1, torch.zeros(()), v)
    base = torch.zeros(offset + rows * (cols + pad) + 8, dtype=dtype, device="cuda")
    view = base[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(v.to(dtype))
    return view


def check_operand(op, src, g, transpose):
    code, byte = R.quantise(src.cpu().t() if transpose else src.cpu(), op.fmt, g)
    got = op.codes.cpu()
    assert torch.equal(op.scales.cpu(), R.tile_scales(byte))
    # the sign of an element that rounds to zero is not part of its value
    got_codes = torch.stack([got & 15, got >> 4], -1).flatten(1)[:, :op.cols].long()
    sure = torch.isfinite(R.values(code, byte, op.fmt))
    zero = ((got_codes & 7) == 0) & ((code & 7) == 0)
    assert ((got_codes == code) | zero | ~sure).all()
    assert (torch.stack([got & 15, got >> 4], -1).flatten(1)[:, op.cols:-(-op.cols // 32) * 32] == 0).all()
    return code, byte


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FORMATS)
def test_quantise(fmt, dtype, transpose):
    for rows, cols, pad, offset in ((1, 1, 0, 0), (1, 15, 0, 0), (3, 16, 0, 0), (2, 17, 1, 1), (5, 33, 3, 0), (130, 64, 0, 0), (127, 129, 7, 1),
                                    (128, 256, 8, 8), (129, 257, 0, 0), (300, 520, 8, 2), (64, 1000, 0, 0), (513, 31, 1, 0)):
        src = matrix(rows, cols, dtype, pad, offset, rows)
        R_, C_ = (cols, rows) if transpose else (rows, cols)
        g = 0.3 if fmt == B.NVFP4 else 1.0
        op = B.new_fp4(fmt, R_, C_, scale=torch.full((1,), g, device="cuda") if fmt == B.NVFP4 else None)
        op.codes.fill_(0xAB)
        op.scales.fill_(0xCD)
        amax = torch.full((1,), 7e7, device="cuda")
        B.fp8mlp_quantize_fp4(src, op, transpose=transpose, amax=amax)
        check_operand(op, src, g, transpose)
        assert float(amax) == float(src.float().abs().max())
        if fmt == B.NVFP4:                                       # the scale from the data
            op.codes.fill_(0xAB)
            B.fp8mlp_quantize_fp4(src, op, transpose=transpose, scale_mode=B.SCALE_FROM_CURRENT_AMAX)
            assert float(op.scale) == R.tensor_scale(float(src.float().abs().max())) and float(op.amax) == float(src.float().abs().max())
            check_operand(op, src, float(op.scale), transpose)


def test_negative_scale_of_the_tensor():
    """g < 0: the block scales stay positive (the tensor cores know no sign of theirs), the elements change theirs."""
    src = matrix(40, 96, torch.float32, seed=3)
    op, out = B.new_fp4(B.NVFP4, 40, 96, scale=torch.full((1,), -4.0, device="cuda")), torch.empty(40, 96, device="cuda")
    ref, same = B.new_fp4(B.NVFP4, 40, 96, scale=torch.full((1,), 4.0, device="cuda")), torch.empty(40, 96, device="cuda")
    B.fp8mlp_quantize_fp4(src, op)
    B.fp8mlp_quantize_fp4(src, ref)
    assert torch.equal(op.scales, ref.scales)
    B.fp8mlp_dequantize_fp4(op, out)
    B.fp8mlp_dequantize_fp4(ref, same)
    assert torch.equal(out, same)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (1, 7, 0, 3), (300, 517, 0, 0), (300, 517, 0, 1), (97, 515, 5, 3), (4, 100000, 0, 0),
                                                  (2000, 9, 1, 0), (700, 1024, 8, 8)])
def test_maximum_wherever_it_lies(rows, cols, pad, offset, dtype):
    """The data's maximum in the corners and at the edges of rows on any boundary, with larger values and NaN between the rows."""
    base = torch.full((offset + rows * (cols + pad) + 16,), 1e6, dtype=dtype, device="cuda")
    base[::2] = math.nan
    src = base[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    op = B.new_fp4(B.NVFP4, rows, cols)
    for at in {(0, 0), (0, cols - 1), (rows - 1, 0), (rows - 1, cols - 1), (rows // 2, cols // 2), (rows // 3, cols - 1)}:
        src.fill_(0.5)
        src[at] = -3.0
        B.fp8mlp_quantize_fp4(src, op, scale_mode=B.SCALE_FROM_CURRENT_AMAX)
        assert float(op.amax) == 3.0 and float(op.scale) == R.tensor_scale(3.0)
        check_operand(op, src, float(op.scale), False)


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("rows,cols", [(128, 2048), (128, 2056), (513, 512), (1, 65536), (65536, 1), (2048, 128), (400, 700), (300, 4096)])
def test_scale_of_the_data_on_either_side_of_one_launch(rows, cols, transpose):
    """Matrices around the size up to which one cluster does all; their largest element in the last row, column or both."""
    for seed, at in enumerate(((rows - 1, cols - 1), (rows - 1, 0), (0, cols - 1))):
        src = matrix(rows, cols, torch.bfloat16, seed=seed)
        src[at] = -1000.0
        op = B.new_fp4(B.NVFP4, cols if transpose else rows, rows if transpose else cols)
        op.codes.fill_(0xAB)
        op.scales.fill_(0xCD)
        B.fp8mlp_quantize_fp4(src, op, transpose=transpose, scale_mode=B.SCALE_FROM_CURRENT_AMAX)
        assert float(op.amax) == 1000.0 and float(op.scale) == R.tensor_scale(1000.0)
        check_operand(op, src, float(op.scale), transpose)


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
def test_quantise_special_blocks(fmt, transpose):
    n = R.BLOCK[fmt]
    src = torch.randn(6, 4 * n, device="cuda")
    src[0] = 0
    src[1, :n] = math.nan
    src[2, n] = math.inf
    src[2, 2 * n + 1] = -math.inf
    src[3] = 1e-42                                               # subnormal in fp32
    src[3, :n] = 0
    src[4, :n] = 3e38
    src[5] *= 1e-6                                               # below NVFP4's smallest scale
    src = src.t().contiguous() if transpose else src
    op = B.new_fp4(fmt, 6, 4 * n)
    B.fp8mlp_quantize_fp4(src, op, transpose=transpose)
    code, byte = check_operand(op, src, 1.0, transpose)
    nan = 0xff if fmt == B.MXFP4 else 0x7f
    assert (byte[1, 0], byte[2, 1], byte[2, 2], byte[2, 3]) == (nan, nan, nan, byte[2, 3]) and byte[2, 3] != nan
    out = torch.empty(6, 4 * n, device="cuda")
    B.fp8mlp_dequantize_fp4(op, out)
    want = R.values(code, byte, fmt).float().cuda()
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))
    # a maximum that is not finite gives the scale 1, a matrix without elements too
    if fmt == B.NVFP4:
        B.fp8mlp_quantize_fp4(src, op, transpose=transpose, scale_mode=B.SCALE_FROM_CURRENT_AMAX)
        assert float(op.scale) == 1.0
        empty = B.new_fp4(fmt, 0, 16, scale=torch.full((1,), 5.0, device="cuda"))
        B.fp8mlp_quantize_fp4(torch.empty(0, 16, device="cuda"), empty, scale_mode=B.SCALE_FROM_CURRENT_AMAX)
        assert float(empty.scale) == 1.0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FORMATS)
def test_every_border_rounds_as_it_should(fmt, dtype):
    """Blocks of every significand of a maximum, and in them the borders between codes and their neighbours."""
    n = R.BLOCK[fmt]
    tops = torch.arange(128, 256) / 16.0
    rows = []
    for top in tops.tolist():
        s = float(R.values(torch.tensor([[1]]), R.quantise(torch.full((1, 1), top), fmt)[1], fmt)) * 2
        around = []
        for border in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
            v = torch.tensor(border * s, dtype=dtype)
            bits = v.view(torch.int16 if dtype == torch.bfloat16 else torch.int32)
            around += [float((bits + k).view(dtype)) for k in (-1, 0, 1)]
        around = [v for v in around if abs(v) <= top]
        for i in range(0, len(around), n - 1):
            rows.append(([top] + around[i:i + n - 1] + [0.0] * n)[:n])
    src = torch.tensor(rows).to(dtype).cuda()
    op = B.new_fp4(fmt, *src.shape)
    B.fp8mlp_quantize_fp4(src, op)
    check_operand(op, src, 1.0, False)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_dequantise(fmt, dtype):
    for rows, cols, pad in ((1, 1, 0), (3, 17, 0), (130, 64, 8), (129, 300, 3), (1000, 48, 0)):
        gen = torch.Generator().manual_seed(cols)
        code = torch.randint(0, 16, (rows, cols), generator=gen)
        byte = torch.randint(100, 150, (rows, -(-cols // R.BLOCK[fmt])), generator=gen) if fmt == B.MXFP4 else \
            torch.randint(0, 127, (rows, -(-cols // R.BLOCK[fmt])), generator=gen)
        g = torch.full((1,), 3.0, device="cuda") if fmt == B.NVFP4 else None
        op = B.Fp4Operand(fmt, rows, cols, R.pack_codes(code).cuda(), R.tile_scales(byte).cuda(), g)
        base = torch.full((rows, cols + pad), 55.0, dtype=dtype, device="cuda")
        B.fp8mlp_dequantize_fp4(op, base[:, :cols])
        inv = 1.0 if g is None else float(torch.tensor(1.0) / torch.tensor(3.0))
        want = (R.values(code, byte, fmt) * inv).float().to(dtype)          # one rounding to fp32, one to the type
        assert torch.equal(base[:, :cols].cpu(), want)
        assert (base[:, cols:] == 55.0).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,pad,offset", [(33, 129, 0, 0), (160, 300, 0, 1), (31, 127, 2, 1), (4100, 1153, 0, 0), (4097, 1153, 1, 3), (5000, 1032, 8, 8)])
def test_dequantise_rows_on_any_boundary(fmt, dtype, rows, cols, pad, offset):
    """Rows that begin on even and odd elements, few tiles and many, and what lies around them."""
    gen = torch.Generator().manual_seed(cols)
    code = torch.randint(0, 16, (rows, cols), generator=gen)
    byte = torch.randint(100, 150, (rows, -(-cols // R.BLOCK[fmt])), generator=gen) if fmt == B.MXFP4 else \
        torch.randint(0, 127, (rows, -(-cols // R.BLOCK[fmt])), generator=gen)
    op = B.Fp4Operand(fmt, rows, cols, R.pack_codes(code).cuda(), R.tile_scales(byte).cuda())
    base = torch.full((offset + rows * (cols + pad) + 64,), 55.0, dtype=dtype, device="cuda")
    out = base[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    B.fp8mlp_dequantize_fp4(op, out)
    assert torch.equal(out.cpu(), R.values(code, byte, fmt).float().to(dtype))
    out.fill_(55.0)
    assert (base == 55.0).all()


# ---------------------------------------------------------------- products

def operand(rows, cols, fmt, seed, g=None):
    """An operand of random codes and of scales over a few binades, and the matrix (64 bits, on the GPU) it stands for."""
    gen = torch.Generator().manual_seed(seed)
    code = torch.randint(0, 16, (rows, cols), generator=gen)
    nb = -(-cols // R.BLOCK[fmt])
    byte = torch.randint(122, 131, (rows, nb), generator=gen) if fmt == B.MXFP4 else torch.randint(40, 80, (rows, nb), generator=gen)
    scale = None if g is None else torch.full((1,), g, device="cuda")
    op = B.Fp4Operand(fmt, rows, cols, R.pack_codes(code).cuda(), R.tile_scales(byte).cuda(), scale)
    return op, R.values(code, byte, fmt, 1.0 if g is None else g).cuda()


def product_close(out, a, b):
    """An MMA adds 64 products to the accumulator, a split 8 sums: each such sum is taken to be off by two last places of fp32
    (2^-22) of the sizes' sum, whether the tensor core rounds or cuts; the factor of the tensor scales adds 4 roundings."""
    want, sizes = a @ b.T, a.abs() @ b.abs().T
    off = (a.shape[1] / 64 + 12) * 2.0 ** -22 * sizes
    half = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24
    assert ((out.double() - want).abs() <= off + half * (want.abs() + off)).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 128, 64), (16, 128, 256), (3, 130, 17), (1, 4096, 4096), (17, 500, 1000), (33, 257, 65),
                                   (64, 640, 4112), (100, 300, 130), (128, 129, 511), (700, 1, 96), (300, 20, 2048), (129, 129, 33),
                                   (200, 333, 1536), (513, 1411, 200)])
def test_product_small(fmt, M, N, K):
    g = (0.25, 3.0) if fmt == B.NVFP4 and M % 2 else (None, None)
    a, av = operand(M, K, fmt, 1, g[0])
    b, bv = operand(N, K, fmt, 2, g[1])
    for dtype, pad, offset in ((torch.float32, 0, 0), (torch.bfloat16, 0, 0), (torch.float32, 3, 1), (torch.bfloat16, 16, 8)):
        base = torch.full((offset + M * (N + pad) + 64,), 33.0, dtype=dtype, device="cuda")
        out = base[offset:offset + M * (N + pad)].view(M, N + pad)[:, :N]
        B.fp8mlp_gemm_fp4(a, b, out)
        product_close(out, av, bv)
        out.fill_(33.0)
        assert (base == 33.0).all()                              # nothing beside the rows


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", [(2048, 4096, 1024), (1500, 8000, 600), (4096, 1411, 2050), (5000, 3000, 64), (300, 20000, 777)])
def test_product_on_cta_pairs(fmt, M, N, K):
    a, av = operand(M, K, fmt, 1)
    b, bv = operand(N, K, fmt, 2)
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((M, N), 33.0, dtype=dtype, device="cuda")
        B.fp8mlp_gemm_fp4(a, b, out)
        product_close(out, av, bv)


@pytest.mark.parametrize("M,N,K", [(2100, 2070, 320), (300, 1000, 64), (140, 129, 2048), (2049, 1985, 33)])
def test_product_rows_on_any_boundary(M, N, K):
    """Rows that begin on even and odd elements, ends inside a block of 32 x 32, and what lies around them."""
    a, av = operand(M, K, B.MXFP4, 1)
    b, bv = operand(N, K, B.MXFP4, 2)
    for dtype in (torch.float32, torch.bfloat16):
        for pad, offset in ((0, 0), (1, 0), (2, 1), (2 + N % 2, 1), (8 - N % 8, 8), (8 - N % 8, 4)):
            base = torch.full((offset + M * (N + pad) + 64,), 33.0, dtype=dtype, device="cuda")
            out = base[offset:offset + M * (N + pad)].view(M, N + pad)[:, :N]
            B.fp8mlp_gemm_fp4(a, b, out)
            product_close(out, av, bv)
            out.fill_(33.0)
            assert (base == 33.0).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M", [1, 40, 2048])
def test_product_nan_stays_in_its_row(fmt, M):
    a, _ = operand(M, 512, fmt, 1)
    b, _ = operand(2048, 512, fmt, 2)
    nan = 0xff if fmt == B.MXFP4 else 0x7f
    b.scales[((300 // 128) * (512 // R.BLOCK[fmt] // 4) + 1) * 512 + (300 % 32) * 16 + (300 % 128) // 32 * 4 + 2] = nan
    out = torch.empty(M, 2048, device="cuda")
    B.fp8mlp_gemm_fp4(a, b, out)
    assert torch.isnan(out[:, 300]).all()
    out[:, 300] = 0
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_linear_layer_and_its_gradients(fmt):
    """y = x W^T and both gradients, every operand quantised along its contraction, against 64-bit products of what the plain
    implementation makes of the same matrices; twice over, on another stream and from a captured graph."""
    T, d, f = 333, 256, 700
    gen = torch.Generator().manual_seed(5)
    x, W, dy = (torch.randn(s, generator=gen).bfloat16().cuda() for s in ((T, d), (f, d), (T, f)))
    mode = B.SCALE_FROM_CURRENT_AMAX if fmt == B.NVFP4 else B.SCALE_GIVEN

    def buffers():
        ops = {k: B.new_fp4(fmt, *s) for k, s in dict(x=(T, d), W=(f, d), dy=(T, f), Wt=(d, f), dyt=(f, T), xt=(d, T)).items()}
        outs = [torch.empty(T, f, dtype=torch.bfloat16, device="cuda"), torch.empty(T, d, dtype=torch.bfloat16, device="cuda"),
                torch.empty(f, d, device="cuda")]
        return ops, outs

    def step(o, outs):
        for k, src, t in (("x", x, False), ("W", W, False), ("dy", dy, False), ("Wt", W, True), ("dyt", dy, True), ("xt", x, True)):
            B.fp8mlp_quantize_fp4(src, o[k], transpose=t, scale_mode=mode)
        B.fp8mlp_gemm_fp4(o["x"], o["W"], outs[0])
        B.fp8mlp_gemm_fp4(o["dy"], o["Wt"], outs[1])
        B.fp8mlp_gemm_fp4(o["dyt"], o["xt"], outs[2])
    first = buffers()
    step(*first)

    def plain(v):
        g = R.tensor_scale(float(v.float().abs().max())) if fmt == B.NVFP4 else 1.0
        return R.values(*R.quantise(v.cpu(), fmt, g), fmt, g).cuda()
    product_close(first[1][0], plain(x), plain(W))
    product_close(first[1][1], plain(dy), plain(W.t()))
    product_close(first[1][2], plain(dy.t()), plain(x.t()))
    # the layer's own gradient (straight-through), from the quantised operands: 4 bits keep it within a fifth
    exact = dy.double().T @ x.double()
    assert float((first[1][2].double() - exact).norm() / exact.norm()) < 0.2
    other, captured, graph = buffers(), buffers(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        step(*other)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(*captured)
    for _ in range(3):
        graph.replay()
        step(*first)
    torch.cuda.synchronize()
    for i in range(3):
        assert torch.equal(first[1][i], other[1][i]) and torch.equal(first[1][i], captured[1][i])


def test_norm_into_a_four_bit_layer():
    """What a served model runs in front of its block: residual added and normed, quantised, multiplied; a token at a time
    gives the rows that the whole prompt gives, up to the order of the sums."""
    T, d, f = 40, 512, 384
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.randn(T, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    gain, W = 1 + 0.1 * torch.randn(d, generator=gen, device="cuda"), 0.05 * torch.randn(f, d, generator=gen, device="cuda")
    w4 = B.new_fp4(B.MXFP4, f, d)
    B.fp8mlp_quantize_fp4(W, w4)

    def run(x, r):
        h, y, x4 = torch.empty_like(x), torch.empty_like(x), B.new_fp4(B.MXFP4, x.shape[0], d)
        out = torch.empty(x.shape[0], f, device="cuda")
        B.fp8mlp_rmsnorm(x, r, gain, 1e-5, y, h=h)
        B.fp8mlp_quantize_fp4(y, x4)
        B.fp8mlp_gemm_fp4(x4, w4, out)
        return h, y, out
    h, y, out = run(x, r)
    code, byte = R.quantise(y.cpu(), R.MX)
    wcode, wbyte = R.quantise(W.cpu(), R.MX)
    product_close(out, R.values(code, byte, R.MX).cuda(), R.values(wcode, wbyte, R.MX).cuda())
    for t in (0, 17, 39):
        one = run(x[t:t + 1], r[t:t + 1])
        assert torch.equal(one[0][0], h[t]) and torch.equal(one[1][0], y[t])
        assert float((one[2][0] - out[t]).abs().max()) <= 1e-5 * float(out[t].abs().max())


def test_wrong_shapes_are_refused():
    a, b = operand(4, 64, B.MXFP4, 1)[0], operand(8, 64, B.MXFP4, 2)[0]
    src = torch.zeros(4, 64, device="cuda")
    for bad in (lambda: B.fp8mlp_gemm_fp4(a, b, torch.empty(4, 9, device="cuda")), lambda: B.fp8mlp_gemm_fp4(a, b, torch.empty(5, 8, device="cuda")),
                lambda: B.fp8mlp_gemm_fp4(a, b, torch.empty(4, 8)), lambda: B.fp8mlp_gemm_fp4(a, b, torch.empty(4, 8, device="cuda", dtype=torch.float16)),
                lambda: B.fp8mlp_quantize_fp4(src, b), lambda: B.fp8mlp_quantize_fp4(src, a, transpose=True),
                lambda: B.fp8mlp_dequantize_fp4(a, torch.empty(4, 63, device="cuda")),
                lambda: B.fp8mlp_gemm_fp4(a, B.Fp4Operand(B.MXFP4, 8, 64, b.codes[:, :16], b.scales), torch.empty(4, 8, device="cuda")),
                lambda: B.fp8mlp_gemm_fp4(a, B.Fp4Operand(B.MXFP4, 8, 64, b.codes, b.scales[:511]), torch.empty(4, 8, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.Fp8MlpError):
        B.fp8mlp_quantize_fp4(src, a, scale_mode=B.SCALE_FROM_CURRENT_AMAX)
