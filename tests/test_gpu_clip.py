"""fp8mlp_grad_norm, fp8mlp_clip_grads and fp8mlp_adam_step_scaled against plain 64-bit implementations.

The squares are summed in fp64 and the root is rounded once: the norm is held to 2^-23 of itself, the coefficient (an fp32
sum and quotient of it) to 4 2^-24; the maximum norm is exact.  The clipped tensors are one fp32 product with the reported
coefficient, rounded once: bit for bit."""
import numpy as np
import pytest
import torch

import experts_reference as R
from paper_2409_12517_b200 import binding as B

pytestmark = pytest.mark.gpu

KINDS = pytest.mark.parametrize("kind", ["l2", "inf"])
F32, BF16 = torch.float32, torch.bfloat16


def _grad(rng, n, dtype, shift=0, scale=1e-2):
    """n elements that start `shift` elements into their buffer, with their buffer."""
    flat = torch.full((n + shift + 40,), 3.0, dtype=dtype, device="cuda")
    g = flat[shift:shift + n]
    g.copy_(torch.from_numpy((rng.normal(0, scale, n)).astype(np.float32)))
    return flat, g


def _run(grads, outs, max_norm, kind, norm_only=False):
    norm_coef = torch.full((2,), -1.0, device="cuda")
    lst = B.new_grad_list(grads, outs)
    call = B.fp8mlp_grad_norm if norm_only else B.fp8mlp_clip_grads
    call(lst, B.NORM_L2 if kind == "l2" else B.NORM_INF, max_norm, norm_coef, B.new_norm_workspace())
    torch.cuda.synchronize()
    return norm_coef.cpu().numpy()


def _check_norm(got, grads, max_norm, kind):
    norm, coef = R.clip([g.float().cpu().numpy() for g in grads], max_norm, kind)
    if kind == "l2":
        np.testing.assert_allclose(got[0], norm, rtol=2.0 ** -23, atol=1e-45)
    else:
        assert got[0] == np.float32(norm)
    np.testing.assert_allclose(got[1], coef, rtol=5 * 2.0 ** -24)


LISTS = {
    "one": [(1, F32, 0)],
    "odd_f32": [(n, F32, s) for n, s in ((1, 0), (7, 1), (8, 0), (9, 3), (31, 5), (33, 7), (1000, 2), (8191, 0), (32769, 1))],
    "odd_bf16": [(n, BF16, s) for n, s in ((1, 0), (3, 1), (15, 0), (17, 15), (33, 7), (4097, 3), (16384, 0), (70001, 9))],
    "mixed": [(256 * 704, BF16, 0), (5, F32, 1), (0, F32, 0), (704 * 256, F32, 0), (0, BF16, 3), (4096, BF16, 1), (300001, F32, 0)],
    "tiny_config": [(256 * 704, F32, 0)] * 3,
    "large": [(5_000_003, F32, 0), (3_000_001, BF16, 1)],
    "17_tensors": [(100 + 13 * i, F32 if i % 3 else BF16, i % 5) for i in range(17)],
    "200_tensors": [(1 + 37 * i, F32 if i % 3 else BF16, i % 5) for i in range(200)],
    "2100_tensors": [(1 + (7 * i) % 300, BF16 if i % 3 else F32, i % 4) for i in range(2100)],
}


@KINDS
@pytest.mark.parametrize("name", list(LISTS))
def test_clip(name, kind):
    rng = np.random.default_rng(len(name))
    made = [_grad(rng, n, dt, s) for n, dt, s in LISTS[name]]
    grads = [g for _, g in made]
    before = [g.clone() for g in grads]
    norm, _ = R.clip([g.float().cpu().numpy() for g in grads], 1.0, kind)
    for max_norm in (0.37 * norm, 2.0 * norm + 1.0):
        got = _run(grads, None, max_norm, kind, norm_only=True)
        _check_norm(got, grads, max_norm, kind)
        # into other buffers, of the same and of another alignment
        for shift in (0, 3):
            made_out = [_grad(rng, n, dt, shift) for n, dt, _ in LISTS[name]]
            outs = [o for _, o in made_out]
            again = _run(grads, outs, max_norm, kind)
            assert np.array_equal(got, again)
            for g, o, (flat, _) in zip(grads, outs, made_out):
                assert torch.equal(o, (g.float() * torch.tensor(got[1], device="cuda")).to(g.dtype))
                assert bool((flat[:shift] == 3.0).all()) and bool((flat[shift + g.numel():] == 3.0).all())
    for g, b in zip(grads, before):
        assert torch.equal(g, b)
    got = _run(grads, None, 0.37 * norm, kind)         # in place
    for (flat, g), b, (n, _, s) in zip(made, before, LISTS[name]):
        assert torch.equal(g, (b.float() * torch.tensor(got[1], device="cuda")).to(g.dtype))
        assert bool((flat[:s] == 3.0).all()) and bool((flat[s + n:] == 3.0).all())


@KINDS
def test_range_of_the_values(kind):
    """Squares far outside the fp32 range, zeros, and lists without an element."""
    for scale in (1e30, 1e-30, 3e-42):
        g = torch.full((1000,), scale, device="cuda")
        got = _run([g], None, 1.0, kind, norm_only=True)
        _check_norm(got, [g], 1.0, kind)
    zero = torch.zeros(100, device="cuda")
    assert np.array_equal(_run([zero], None, 1.0, kind), [0.0, 1.0])
    assert np.array_equal(_run([], None, 1.0, kind), [0.0, 1.0])
    assert np.array_equal(_run([zero[:0], zero[:0].bfloat16()], None, 1.0, kind), [0.0, 1.0])
    g = torch.ones(50, device="cuda")
    assert _run([g], None, 0.0, kind)[1] == 0.0 and not g.any()                      # max_norm 0: everything goes to 0
    g = torch.full((16,), 3e38, device="cuda")
    got = _run([g], None, 1.0, "l2", norm_only=True)
    assert np.isinf(got[0]) and got[1] == 0.0                                        # the norm itself leaves fp32


@KINDS
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_nan_and_infinity(kind, dtype):
    rng = np.random.default_rng(1)
    for at in (0, 12345, 49999):
        _, g = _grad(rng, 50000, dtype)
        g[at] = float("nan")
        got = _run([g], None, 1.0, kind, norm_only=True)
        assert np.isnan(got).all()
        g[at] = float("-inf")
        out = torch.empty_like(g)
        got = _run([g], [out], 1.0, kind)
        assert np.isposinf(got[0]) and got[1] == 0.0
        assert bool(torch.isnan(out[at])) and int(torch.isnan(out).sum()) == 1 and not out[torch.arange(50000, device="cuda") != at].any()


def test_more_than_2_to_the_31_elements():
    n = 2 ** 31 + 1003
    g = torch.zeros(n, dtype=BF16, device="cuda")
    g[0], g[2 ** 31 - 1], g[n - 1] = 2.0, 4.0, 4.0
    got = _run([g], None, 3.0, "l2")
    assert got[0] == 6.0
    # the coefficient rounds to 0.49999991...; in bf16 the products round back to the exact halves
    assert float(g[0]) == 1.0 and float(g[2 ** 31 - 1]) == 2.0 and float(g[n - 1]) == 2.0 and float(g[1]) == 0.0


def test_repeats_bit_for_bit_and_other_stream():
    rng = np.random.default_rng(6)
    grads = [_grad(rng, n, dt)[1] for n, dt in ((3_000_000, F32), (1_000_001, BF16), (17, F32))]
    first = _run(grads, None, 0.1, "l2", norm_only=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        assert np.array_equal(first, _run(grads, None, 0.1, "l2", norm_only=True))
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        late = [torch.empty_like(g) for g in grads]
        for a, b in zip(late, grads):
            a.copy_(b)
        assert np.array_equal(first, _run(late, None, 0.1, "l2", norm_only=True))


def test_workspace_holds_no_state():
    ws = B.new_norm_workspace()
    out = torch.empty(2, device="cuda")
    g = torch.full((200_000,), 0.5, device="cuda")
    want = None
    for fill in (0, 255, 127):
        ws.fill_(fill)
        B.fp8mlp_grad_norm(B.new_grad_list([g]), B.NORM_L2, 1.0, out, ws)
        want = out.clone() if want is None else want
        assert torch.equal(out, want)


@pytest.mark.parametrize("cast", [False, True])
def test_adam_with_the_clip_coefficient(cast):
    """The fused form against clipping in place and then the plain step: the same fp32 product, so the same bits."""
    rng = np.random.default_rng(9)
    n, cols = 256 * 704, 704
    w0 = torch.from_numpy(rng.normal(0, 0.02, n).astype(np.float32)).cuda()
    _, g = _grad(rng, n, F32)
    one = lambda: torch.ones(1, device="cuda")
    states = []
    for _ in range(2):
        states.append(dict(w=w0.clone(), g=g.clone(), m=torch.zeros(n, dtype=torch.uint8, device="cuda"),
                           v=torch.zeros(n, dtype=torch.uint8, device="cuda"), scale_m_in=one(), scale_v_in=one(),
                           scale_m_out=torch.full((1,), 2.0 ** 14, device="cuda"), scale_v_out=torch.full((1,), 2.0 ** 24, device="cuda"),
                           amax_m=torch.zeros(1, device="cuda"), amax_v=torch.zeros(1, device="cuda")))
    codes = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    hp = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=1)
    casts = [[dict(dst=c, cols=cols, ld_dst=cols, scale=torch.full((1,), 64.0, device="cuda"))] for c in codes]
    norm_coef, ws = torch.empty(2, device="cuda"), B.new_norm_workspace()
    B.fp8mlp_grad_norm(B.new_grad_list([states[0]["g"]]), B.NORM_L2, 1.0, norm_coef, ws)
    assert float(norm_coef[1]) < 1.0
    B.fp8mlp_adam_step_scaled([states[0]], casts[0] if cast else None, norm_coef[1:], **hp)
    B.fp8mlp_clip_grads(B.new_grad_list([states[1]["g"]]), B.NORM_L2, 1.0, norm_coef, ws)
    if cast:
        B.fp8mlp_adam_step_cast([states[1]], casts[1], **hp)
    else:
        B.fp8mlp_adam_step([states[1]], **hp)
    for key in ("w", "m", "v", "amax_m", "amax_v"):
        assert torch.equal(states[0][key], states[1][key]), key
    assert torch.equal(codes[0], codes[1]) and bool(codes[0].any()) == cast
    assert torch.equal(states[0]["g"], g)              # the fused form leaves the gradient as it was


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 16, 33, 1000, 8191, 70001, 3_000_003])
def test_norm_of_the_same_values_at_other_addresses(n, dtype):
    """The grouping of the sum follows the addresses modulo 32: at equal ones the norm has the same bits, at others it stays within
    its bound.  The 8 or 16 squares of a 32-byte unit are summed in fp32, at most four roundings of 2^-24 one after the other (the
    squares of bf16 are exact there), the units in fp64; the root halves a relative error and is rounded once: 2 + 1 times 2^-24."""
    rng = np.random.default_rng(n)
    values = torch.from_numpy((rng.normal(0, 1, n) * np.exp(rng.normal(0, 2, n))).astype(np.float32)).to(dtype)
    exact, _ = R.clip([values.float().numpy()], 1.0, "l2")
    size = values.element_size()
    by_shift = {}
    for shift in range(32 // size):
        for _ in range(2):
            flat = torch.zeros(n + 2 * shift + 64, dtype=dtype, device="cuda")
            g = flat[shift:shift + n]
            g.copy_(values)
            assert g.data_ptr() % 32 == shift * size
            got = _run([g], None, 1.0, "l2", norm_only=True)
            assert abs(float(got[0]) - exact) <= 3.001 * 2.0 ** -24 * exact
            assert np.array_equal(by_shift.setdefault(shift, got), got)
