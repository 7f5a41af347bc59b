"""The residual norm and its gradient on the GPU against plain 64-bit evaluations (fp4_reference.py).

Tolerances count roundings.  u = 2^-24 (fp32).  The sum of squares has only positive terms: at most 32 sequential additions
in a thread, 5 in a warp and 16 over warps, each off by u of the running sum: 53 u, and 3 u for the mean, eps and one division;
the root halves what it takes in; root and division add 2 u: rstd is within 32 u.  y takes two more."""
import math

import pytest
import torch

import fp4_reference as R
from paper_2409_12517_b200 import binding as B

pytestmark = pytest.mark.gpu
U, RSTD, Y = 2.0 ** -24, 32 * 2.0 ** -24, 34 * 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
EPS = 1e-5


def rows_of(T, d, dtype, pad=0, offset=0, scale=1.0, seed=0):
    """[T, d] with rows of d + pad elements, starting `offset` elements past a 256-byte boundary, and its surroundings."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    base = torch.full((offset + T * (d + pad) + 64,), 77.0, dtype=dtype, device="cuda")
    view = base[offset:offset + T * (d + pad)].view(T, d + pad)[:, :d]
    view.copy_((scale * torch.randn(T, d, generator=gen, device="cuda")).to(dtype))
    return view, base


def codes_close(codes, exact, rel):
    """E4M3 codes of values that are `rel` off: within half a step (2^-4 of a normal value, 2^-10 below 2^-6) of them."""
    got = codes.view(torch.float8_e4m3fn).float().double()
    want = exact.clamp(-448, 448)
    assert ((got - want).abs() <= torch.maximum(want.abs() * 2 ** -4, torch.full_like(want, 2 ** -10)) * (1 + 4 * rel) + want.abs() * rel).all()


SHAPES = [(1, 16), (3, 32), (5, 48), (257, 64), (2, 256), (31, 496), (700, 512), (130, 1040), (9, 2064), (300, 4096), (7, 4112),
          (5, 8192), (4, 8208), (3, 12304), (2, 16384), (4100, 128)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", SHAPES)
def test_forward(T, d, dtype):
    per16 = 16 // torch.empty(0, dtype=dtype).element_size()
    for residual, pad, offset, out in ((False, 0, 0, B.RMS_SAME), (True, 2 * per16, 0, B.RMS_SAME), (True, per16, per16, B.RMS_E4M3),
                                       (True, 0, 0, B.RMS_E4M3), (False, 0, per16, B.RMS_E4M3_ROWS), (True, 0, 0, B.RMS_E4M3_ROWS)):
        x, _ = rows_of(T, d, dtype, pad, offset, 2.0, 1)
        r = rows_of(T, d, dtype, pad, offset, 1.0, 2)[0] if residual else None
        h, h_all = rows_of(T, d, dtype, pad, offset, 0.0, 3) if residual else (None, None)
        gain = 1 + 0.2 * torch.randn(d, device="cuda") if not (residual and pad) else None
        rstd, amax = torch.empty(T, device="cuda"), torch.full((1,), 5e9, device="cuda")
        if out == B.RMS_SAME:
            y, y_all = rows_of(T, d, dtype, pad, offset, 0.0, 4)
        else:
            y_all = torch.full((T, d + 16), 0x77, dtype=torch.uint8, device="cuda")
            y = y_all[:, :d]
        scale = torch.full((1,), 96.5, device="cuda") if out == B.RMS_E4M3 else torch.empty(T, device="cuda") if out == B.RMS_E4M3_ROWS else None
        B.fp8mlp_rmsnorm(x, r, gain, EPS, y, h=h, out=out, scale=scale, amax=None if out == B.RMS_E4M3_ROWS else amax, rstd=rstd)
        stored = x if r is None else (x.float() + r.float()).to(dtype)
        if residual:
            assert torch.equal(h, stored)
            assert int((h_all == 77.0).sum()) >= h_all.numel() - T * d          # what lies between and behind the rows
        want, want_rstd = R.norm(stored.cpu(), None if gain is None else gain.cpu(), EPS)
        want, want_rstd = want.cuda(), want_rstd.cuda()
        assert ((rstd.double() - want_rstd).abs() <= RSTD * want_rstd).all()
        if out == B.RMS_SAME:
            assert ((y.double() - want).abs() <= want.abs() * (HALF[dtype] + Y + HALF[dtype] * Y)).all()
            assert int((y_all == 77.0).sum()) >= y_all.numel() - T * d
        else:
            assert (y_all[:, d:] == 0x77).all()
            if out == B.RMS_E4M3_ROWS:
                want_scale = 448.0 / want.abs().amax(-1)
                assert ((scale.double() - want_scale).abs() <= want_scale * (Y + 2 * U)).all()
                codes_close(y, want * want_scale[:, None], 2 * Y + 4 * U)
                assert (y.view(torch.float8_e4m3fn).float().abs().amax(-1) == 448).all()
            else:
                codes_close(y, want * 96.5, Y + U)
        if out != B.RMS_E4M3_ROWS:
            top = float(want.abs().max())
            assert abs(float(amax) - top) <= Y * top


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_forward_in_place_and_repeated(dtype):
    x, r = rows_of(300, 512, dtype, seed=1)[0], rows_of(300, 512, dtype, seed=2)[0]
    gain = torch.randn(512, device="cuda")
    y0, h0 = torch.empty(300, 512, dtype=dtype, device="cuda"), torch.empty(300, 512, dtype=dtype, device="cuda")
    B.fp8mlp_rmsnorm(x, r, gain, EPS, y0, h=h0)
    for where in ("x", "residual", "not wanted"):
        a, b, y = x.clone(), r.clone(), torch.empty_like(y0)
        B.fp8mlp_rmsnorm(a, b, gain, EPS, y, h={"x": a, "residual": b}.get(where))
        assert torch.equal(y, y0)
        assert torch.equal({"x": a, "residual": b}.get(where, h0), h0)
        assert torch.equal(a, h0 if where == "x" else x) and torch.equal(b, h0 if where == "residual" else r)


def test_forward_rows_without_a_norm():
    """Rows of zeros, with NaN and with infinities: the formulas' values, and nothing of them in their neighbours."""
    x = torch.randn(6, 128, device="cuda")
    x[1] = 0
    x[2, 5] = math.nan
    x[3, 127] = math.inf
    x[4] = 1e-30
    for out in (B.RMS_SAME, B.RMS_E4M3, B.RMS_E4M3_ROWS):
        y = torch.empty(6, 128, device="cuda") if out == B.RMS_SAME else torch.empty(6, 128, dtype=torch.uint8, device="cuda")
        scale = torch.ones(6 if out == B.RMS_E4M3_ROWS else 1, device="cuda")
        amax = torch.zeros(1, device="cuda")
        B.fp8mlp_rmsnorm(x, None, None, EPS, y, out=out, scale=scale, amax=None if out == B.RMS_E4M3_ROWS else amax)
        v = y if out == B.RMS_SAME else y.view(torch.float8_e4m3fn).float()
        assert (v[1] == 0).all() and torch.isnan(v[2]).all() and torch.isfinite(v[0]).all() and torch.isfinite(v[5]).all()
        assert torch.isnan(v[3, 127]) and (v[3, :127] == 0).all()
        if out == B.RMS_E4M3_ROWS:
            assert scale[1] == 1 and scale[2] == 1 and scale[3] == 1 and float(v[4].max()) == 448
        else:
            assert math.isfinite(float(amax)) and float(amax) > 1
    y = torch.empty(6, 128, device="cuda")
    B.fp8mlp_rmsnorm(x[1:2], None, None, 0.0, y[:1])
    assert torch.isnan(y[0]).all()                                       # 0 / 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,gained", [(2000, 512, True), (700, 4096, True), (700, 4096, False), (64, 16384, True), (3000, 48, True)])
def test_codes_are_those_next_to_the_exact_values(T, d, gained, dtype):
    """Not one code off, but for values within 6 roundings (2^-24) of a border: a row's squares are added in fp32 within a warp at most,
    3 roundings for four of them, 2 for a thread's sixteen and 5 for the warp, which the root halves; one more for 1 / rms (the second
    fp32 number of the factor has the rest).  Values on a border are among them (bf16 rows without a gain: products with 448 / maximum
    that end in a five)."""
    x = rows_of(T, d, dtype, scale=2.0, seed=d)[0]
    gain = 1 + 0.2 * torch.randn(d, device="cuda") if gained else None
    y = torch.empty(T, d, dtype=torch.uint8, device="cuda")
    given, own = torch.full((1,), 96.5, device="cuda"), torch.empty(T, device="cuda")
    want, _ = R.norm(x.cpu(), None if gain is None else gain.cpu(), EPS)
    for out, scale in ((B.RMS_E4M3, given), (B.RMS_E4M3_ROWS, own)):
        B.fp8mlp_rmsnorm(x, None, gain, EPS, y, out=out, scale=scale)
        exact = (want * 96.5 if out == B.RMS_E4M3 else want * (448.0 / want.abs().amax(-1, keepdim=True))).abs()
        slack = 6 * U if out == B.RMS_E4M3 else 2.0 ** -40          # (1 / rms is not in the codes of a row of its own scale)
        low, high = (R.nearest(R.E4M3_CODES[:127], exact * (1 + s * slack)) for s in (-1, 1))
        got = (y & 0x7f).cpu().long()
        assert ((got >= low) & (got <= high)).all()
        assert torch.equal((y >= 0x80).cpu() | (got == 0), (want < 0) | (got == 0))


def test_rows_too_small_for_a_scale_of_their_own():
    """448 / maximum beyond fp32, with the maximum of y, or of h gain alone: scale 1, codes of y as it is, no NaN."""
    x = torch.randn(5, 64, device="cuda")
    for row, top in ((1, 1e-37), (2, 1.2e-36), (3, 1e-44)):
        x[row] = 0
        x[row, 3], x[row, 4] = top, -top / 2
    for gain in (None, torch.full((64,), 1.0, device="cuda")):
        y, scale = torch.full((5, 64), 0x55, dtype=torch.uint8, device="cuda"), torch.zeros(5, device="cuda")
        B.fp8mlp_rmsnorm(x, None, gain, EPS, y, out=B.RMS_E4M3_ROWS, scale=scale)
        v = y.view(torch.float8_e4m3fn).float()
        assert (scale[1:4] == 1).all() and (v[1:4] == 0).all()
        assert (v[[0, 4]].abs().amax(-1) == 448).all() and (scale[[0, 4]] > 1).all()


@pytest.mark.parametrize("T", [0, 1, 2000])
def test_amax_is_of_this_call(T):
    amax = torch.full((1,), 1e30, device="cuda")
    x = torch.ones(T, 64, dtype=torch.bfloat16, device="cuda")
    B.fp8mlp_rmsnorm(x, None, None, 0.0, torch.empty_like(x), amax=amax)
    assert float(amax) == (1.0 if T else 0.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", SHAPES)
def test_backward(T, d, dtype):
    per16 = 16 // torch.empty(0, dtype=dtype).element_size()
    for with_dh, with_gain, pad, offset in ((True, True, 0, 0), (False, True, per16, per16), (True, False, 2 * per16, 0)):
        dy, _ = rows_of(T, d, dtype, pad, offset, 1e-3, 1)
        h, _ = rows_of(T, d, dtype, pad, offset, 2.0, 2)
        dh = rows_of(T, d, dtype, pad, offset, 1e-3, 3)[0] if with_dh else None
        dx, dx_all = rows_of(T, d, dtype, pad, offset, 0.0, 4)
        gain = 1 + 0.2 * torch.randn(d, device="cuda") if with_gain else None
        rstd = (1 / torch.sqrt(h.float().square().mean(-1) + EPS)).contiguous()
        d_gain = torch.full((d,), 9e9, device="cuda")
        B.fp8mlp_rmsnorm_backward(dy, h, gain, rstd, dh, dx, d_gain, B.new_rmsnorm_workspace(d))
        cpu = lambda t: None if t is None else t.cpu()
        want, want_gain = (t.cuda() for t in R.norm_backward(dy.cpu(), h.cpu(), cpu(gain), rstd.cpu(), cpu(dh)))
        # the mean's terms have both signs: its error is 53 + 4 roundings of the sum of their sizes
        g = dy.double() * (1.0 if gain is None else gain.double())
        unit = h.double() * rstd.double()[:, None]
        sizes = (g * unit).abs().mean(-1, keepdim=True)
        off = rstd.double()[:, None] * (4 * U * (g.abs() + (unit * sizes).abs()) + unit.abs() * 57 * U * sizes) + U * want.abs()
        assert ((dx.double() - want).abs() <= off + HALF[dtype] * (want.abs() + off)).all()
        assert int((dx_all == 77.0).sum()) >= dx_all.numel() - T * d
        # a block adds its rows one after the other, then the blocks' sums are added: at most T + 70 roundings of the sizes' sum
        gain_sizes = (dy.double() * unit).abs().sum(0)
        assert ((d_gain.double() - want_gain).abs() <= (min(T, 600) + 70) * U * gain_sizes).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(16, 8192), (17, 4096), (32, 4096), (33, 4096), (16, 12304), (17, 12304), (40, 8208), (17, 16384), (513, 256)])
def test_batches_on_either_side_of_one_cluster(T, d, dtype):
    test_forward(T, d, dtype)
    test_backward(T, d, dtype)


def test_backward_in_place_without_gain_gradient_and_empty():
    dy, h, dh = (rows_of(64, 256, torch.bfloat16, seed=s)[0] for s in (1, 2, 3))
    rstd = torch.rand(64, device="cuda") + 0.5
    out = torch.empty_like(dy)
    B.fp8mlp_rmsnorm_backward(dy, h, None, rstd, dh, out, None, None)
    for which in (0, 1):
        pair = [dy.clone(), dh.clone()]
        B.fp8mlp_rmsnorm_backward(pair[0], h, None, rstd, pair[1], pair[which], None, None)
        assert torch.equal(pair[which], out)
    d_gain = torch.ones(256, device="cuda")
    B.fp8mlp_rmsnorm_backward(dy[:0], h[:0], None, rstd[:0], None, out[:0], d_gain, B.new_rmsnorm_workspace(256))
    assert (d_gain == 0).all()


def test_backward_gradient_against_differences():
    """Directional difference of the forward kernel's own output (fp32): error of order step^2 plus roundings / step."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    T, d, step = 4, 96, 1e-2
    h, way, dy = (torch.randn(T, d, generator=gen, device="cuda") for _ in range(3))
    gain = torch.randn(d, generator=gen, device="cuda")
    rstd, y, dx, d_gain = torch.empty(T, device="cuda"), torch.empty_like(h), torch.empty_like(h), torch.empty(d, device="cuda")
    B.fp8mlp_rmsnorm(h, None, gain, EPS, y, rstd=rstd)
    B.fp8mlp_rmsnorm_backward(dy, h, gain, rstd, None, dx, d_gain, B.new_rmsnorm_workspace(d))
    ends = []
    for s in (step, -step):
        B.fp8mlp_rmsnorm(h + s * way, None, gain, EPS, y)
        ends.append(float((y.double() * dy.double()).sum()))
    slope = (ends[0] - ends[1]) / (2 * step)
    size = float(dy.norm() * way.norm() * gain.abs().max())
    assert abs(slope - float((dx.double() * way.double()).sum())) <= size * (10 * step ** 2 + 40 * U / step)


def test_repeats_streams_and_graphs():
    x, r, dy = (rows_of(3000, 1024, torch.bfloat16, seed=s)[0] for s in (1, 2, 3))
    gain, scale = 1 + 0.1 * torch.randn(1024, device="cuda"), torch.full((1,), 50.0, device="cuda")
    new = lambda: dict(h=torch.empty_like(x), y=torch.empty(3000, 1024, dtype=torch.uint8, device="cuda"), amax=torch.zeros(1, device="cuda"),
                       rstd=torch.empty(3000, device="cuda"), dx=torch.empty_like(x), d_gain=torch.empty(1024, device="cuda"),
                       ws=B.new_rmsnorm_workspace(1024))

    def both(o):
        B.fp8mlp_rmsnorm(x, r, gain, EPS, o["y"], h=o["h"], out=B.RMS_E4M3, scale=scale, amax=o["amax"], rstd=o["rstd"])
        B.fp8mlp_rmsnorm_backward(dy, o["h"], gain, o["rstd"], None, o["dx"], o["d_gain"], o["ws"])
    first = new()
    both(first)
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), new()
    with torch.cuda.stream(side):
        both(other)
    captured, graph = new(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(captured)
    for _ in range(3):
        graph.replay()
        both(first)
    torch.cuda.synchronize()
    for k in ("h", "y", "amax", "rstd", "dx", "d_gain"):
        assert torch.equal(first[k], other[k]) and torch.equal(first[k], captured[k]), k


@pytest.mark.parametrize("merged", [False, True])
def test_codes_go_straight_into_the_block(merged):
    """The norm writes the block's operand and its maximum; the forward takes both as they are, as if it had cast x itself."""
    T, d, f = 200, 256, 704
    gen = torch.Generator(device="cuda").manual_seed(3)
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")
    x, r, gain = randn(T, d).bfloat16(), randn(T, d).bfloat16(), 1 + 0.1 * randn(d)
    W1, W2, W3 = 0.05 * randn(d, f), 0.05 * randn(d, f), 0.05 * randn(f, d)
    ctx = B.fp8mlp_create(T, d, f, B.SMOOTH if merged else B.SMOOTH | B.SAVE_FOR_BWD)
    try:
        sc, am = B.new_scales(f), B.new_amax(f)
        y = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
        norm16 = torch.empty_like(x)
        B.fp8mlp_rmsnorm(x, r, gain, EPS, norm16)
        if merged:
            B.fp8mlp_merge_weights(ctx, W1, W2, W3, torch.ones(f, device="cuda"), B.SCALE_FROM_CURRENT_AMAX, sc, am)
            B.fp8mlp_forward_merged(ctx, T, norm16, B.SCALE_FROM_CURRENT_AMAX, sc, am, y)
        else:
            B.fp8mlp_forward(ctx, T, norm16, W1, W2, W3, B.SCALE_FROM_CURRENT_AMAX, sc, am, y)
        sc["x"].fill_(64.0)                       # a power of two: the codes' values are bf16 numbers
        h, ptr = torch.empty_like(x), B.fp8mlp_workspace(ctx, B.WS_XQ)[0]
        am["x"].fill_(0)
        B.fp8mlp_rmsnorm(x, r, gain, EPS, ptr, h=h, out=B.RMS_E4M3, scale=sc["x"], amax=am["x"])
        codes, top = B.workspace_tensor(ctx, B.WS_XQ, (T, d), torch.uint8), float(am["x"])
        if merged:
            B.fp8mlp_forward_merged(ctx, T, None, B.SCALE_GIVEN_X_CAST, sc, am, y)
        else:
            B.fp8mlp_forward(ctx, T, None, W1, W2, W3, B.SCALE_GIVEN_X_CAST, sc, am, y)
        assert float(am["x"]) == top and top > 1
        assert torch.equal(B.workspace_tensor(ctx, B.WS_XQ, (T, d), torch.uint8), codes)
        same = (codes.view(torch.float8_e4m3fn).float() / 64).bfloat16()
        y2 = torch.empty_like(y)
        if merged:
            B.fp8mlp_forward_merged(ctx, T, same, B.SCALE_GIVEN, sc, am, y2)
        else:
            B.fp8mlp_forward(ctx, T, same, W1, W2, W3, B.SCALE_GIVEN, sc, am, y2)
            B.fp8mlp_rmsnorm(x, r, gain, EPS, ptr, out=B.RMS_E4M3, scale=sc["x"], amax=am["x"])
            y3 = torch.empty_like(y)
            B.fp8mlp_forward(ctx, T, None, None, None, None, B.SCALE_GIVEN_BOTH_CAST, sc, am, y3)
            assert torch.equal(y3, y)
            dx, grads = torch.empty_like(x), [torch.empty_like(w) for w in (W1, W2, W3)]
            B.fp8mlp_backward(ctx, T, norm16, B.SCALE_FROM_CURRENT_AMAX, sc, am, dx, *grads)
            assert torch.isfinite(dx.float()).all()
        assert torch.equal(y, y2)
        assert B.fp8mlp_status(ctx) == B.OK
    finally:
        B.fp8mlp_destroy(ctx)


@pytest.mark.parametrize("flags", [B.SAVE_FOR_BWD, B.SMOOTH | B.SAVE_FOR_BWD | B.GU_FP8, B.SAVE_FOR_BWD | B.H_BF16, B.SMOOTH])
def test_codes_in_every_kind_of_context(flags):
    """x as codes gives what the same x gives in bf16 (its codes are numbers of that type), forward and backward."""
    T, d, f = 72, 256, 320
    gen = torch.Generator(device="cuda").manual_seed(9)
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")
    x, dy, W1, W2, W3 = randn(T, d).bfloat16(), (1e-3 * randn(T, d)).bfloat16(), 0.05 * randn(d, f), 0.05 * randn(d, f), 0.05 * randn(f, d)
    ctx = B.fp8mlp_create(T, d, f, flags)
    try:
        sc, am = B.new_scales(f), B.new_amax(f)
        y = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
        B.fp8mlp_forward(ctx, T, x, W1, W2, W3, B.SCALE_FROM_CURRENT_AMAX, sc, am, y)
        sc["x"].fill_(64.0)
        codes = torch.empty(T, d, dtype=torch.uint8, device="cuda")
        ptr = B.fp8mlp_workspace(ctx, B.WS_XQ)[0]
        for at in (codes, ptr):
            B.fp8mlp_rmsnorm(x, None, None, EPS, at, out=B.RMS_E4M3, scale=sc["x"], amax=am["x"])
        results = []
        for mode, x_in in ((B.SCALE_GIVEN_X_CAST, None), (B.SCALE_GIVEN, (codes.view(torch.float8_e4m3fn).float() / 64).bfloat16())):
            B.fp8mlp_forward(ctx, T, x_in, W1, W2, W3, mode, sc, am, y)
            out = [y.clone()]
            if flags & B.SAVE_FOR_BWD:
                grads = [torch.empty_like(x)] + [torch.empty_like(w) for w in (W1, W2, W3)]
                B.fp8mlp_backward(ctx, T, dy, B.SCALE_FROM_CURRENT_AMAX, sc, am, *grads)
                out += grads
            results.append(out)
        assert all(torch.equal(a, b) for a, b in zip(*results)) and torch.isfinite(results[0][0].float()).all()
        assert B.fp8mlp_status(ctx) == B.OK
    finally:
        B.fp8mlp_destroy(ctx)


def test_another_device_or_shape_is_refused():
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros_like(x)
    for bad in (lambda: B.fp8mlp_rmsnorm(x, x[:3], None, EPS, y), lambda: B.fp8mlp_rmsnorm(x, x.float(), None, EPS, y),
                lambda: B.fp8mlp_rmsnorm(x, None, torch.ones(64), EPS, y), lambda: B.fp8mlp_rmsnorm(x, None, None, EPS, y.cpu()),
                lambda: B.fp8mlp_rmsnorm(x, None, None, EPS, y, out=B.RMS_E4M3),
                lambda: B.fp8mlp_rmsnorm(x, None, None, EPS, y, rstd=torch.ones(3, device="cuda")),
                lambda: B.fp8mlp_rmsnorm_backward(x, x.clone(), None, torch.ones(4, device="cuda"), None, y, torch.ones(64, device="cuda"),
                                                  B.new_rmsnorm_workspace(32)),
                lambda: B.fp8mlp_rmsnorm(x.t(), None, None, EPS, y)):
        with pytest.raises(ValueError):
            bad()
