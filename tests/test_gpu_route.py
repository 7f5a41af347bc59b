"""fp8mlp_route, fp8mlp_route_backward and fp8mlp_route_update_bias against plain 64-bit implementations.

Tolerances, derived: an fp32 logit difference x - max carries a relative rounding of 2^-24, which e^. turns into |x - max| 2^-24;
e^., the division and the products add a few roundings each and the sums of at most E terms (over lanes, then a tree) at most
E / 8 + 8 more.  So a weight is held to (range + E / 8 + 32) 2^-23 of itself, and a gradient to the same of the largest
|scale dw| that enters its row; bf16 gradients have half a bf16 step (2^-8) of their value more.  Experts have to be equal
wherever the 64-bit values that were compared differ by 1e-5 of themselves or not at all."""
import numpy as np
import pytest
import torch

import experts_reference as R
from paper_2409_12517_b200 import binding as B

pytestmark = pytest.mark.gpu

KIND = {"softmax": B.SCORE_SOFTMAX, "sigmoid": B.SCORE_SIGMOID}


def _logits(rng, T, E, dtype, pad=0, shift=0):
    """[T, E] with row stride E + pad, starting `shift` elements into its buffer."""
    ld = E + pad
    flat = torch.zeros(shift + T * ld + 64, dtype=dtype, device="cuda")
    view = flat[shift:shift + T * ld].view(T, ld)[:, :E]
    view.copy_(torch.from_numpy(rng.normal(0, 1.5, (T, E)).astype(np.float32)))
    return view


def _route(logits, bias, k, kind, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0):
    T, E = logits.shape
    router = B.new_router(E, k, KIND[kind], groups, top_groups, group_top, renorm, scale)
    experts = torch.full((T, k), -77, dtype=torch.int32, device="cuda")
    weights = torch.full((T, k), float("nan"), device="cuda")
    B.fp8mlp_route(router, logits, bias, experts, weights)
    torch.cuda.synchronize()
    return router, experts, weights


def _tol(x, E):
    finite = x[np.isfinite(x)]
    spread = float(finite.max() - finite.min()) if finite.size else 0.0
    return (min(spread, 110.0) + E / 8 + 32) * 2.0 ** -23


def _compare(logits, bias, experts, weights, k, kind, **kw):
    x = logits.float().cpu().numpy()
    b = None if bias is None else bias.cpu().numpy()
    got_e, got_w = experts.cpu().numpy(), weights.cpu().numpy()
    compared = 0
    for t in range(x.shape[0]):
        ref_e, ref_w, margin = R.route_row(x[t], b, k, kind, **kw)
        if margin < 1e-5:
            continue
        compared += 1
        assert np.array_equal(got_e[t], ref_e), f"token {t}: {got_e[t]} instead of {ref_e}"
        np.testing.assert_allclose(got_w[t], ref_w, rtol=_tol(x[t], x.shape[1]), atol=1e-38, err_msg=f"token {t}")
    assert compared >= 0.5 * x.shape[0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("E,k,T", [(1, 1, 3), (2, 2, 1), (5, 3, 130), (8, 2, 257), (9, 9, 33), (16, 1, 65), (31, 4, 20), (33, 8, 7),
                                   (60, 4, 67), (64, 6, 100), (100, 32, 9), (128, 8, 17), (160, 6, 33), (256, 8, 50), (257, 8, 9),
                                   (512, 10, 6), (1000, 32, 5), (1024, 8, 5)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_route_and_backward(kind, E, k, T, dtype):
    rng = np.random.default_rng(E * 1000 + k)
    for pad, shift, renorm, scale, with_bias in ((0, 0, True, 1.0, False), (3, 1, False, 2.5, True), (8, 8, True, 0.5, True),
                                                 (16, 0, False, 1.0, False)):
        logits = _logits(rng, T, E, dtype, pad, shift)
        bias = torch.from_numpy(rng.normal(0, 0.1, E).astype(np.float32)).cuda() if with_bias else None
        router, experts, weights = _route(logits, bias, k, kind, renorm=renorm, scale=scale)
        _compare(logits, bias, experts, weights, k, kind, renorm=renorm, scale=scale)
        _check_backward(rng, router, logits, experts, kind, renorm, scale, pad, shift)


def _check_backward(rng, router, logits, experts, kind, renorm, scale, pad=0, shift=0):
    T, E = logits.shape
    dw = rng.normal(0, 1, tuple(experts.shape)).astype(np.float32)
    flat = torch.full((shift + T * (E + pad) + 64,), 7.0, dtype=logits.dtype, device="cuda")
    d_logits = flat[shift:shift + T * (E + pad)].view(T, E + pad)[:, :E]
    d_logits.fill_(float("nan"))
    B.fp8mlp_route_backward(router, logits, experts, torch.from_numpy(dw).cuda(), d_logits)
    got, x, chosen = d_logits.float().cpu().numpy(), logits.float().cpu().numpy(), experts.cpu().numpy()
    half_step = 2.0 ** -8 if logits.dtype == torch.bfloat16 else 2.0 ** -24
    for t in range(T):
        ref = R.route_backward_row(x[t], chosen[t], dw[t], kind, renorm, scale)
        used = (chosen[t] >= 0) & (chosen[t] < E)
        size = scale * np.abs(dw[t][used]).max() if used.any() else 0.0
        allowed = 4 * _tol(x[t], E) * size + half_step * np.abs(ref)
        assert (np.abs(got[t] - ref) <= allowed).all(), f"token {t}: off by {np.abs(got[t] - ref).max()}"
    # nothing outside the rows was written
    keep = torch.ones_like(flat, dtype=torch.bool)
    keep[shift:shift + T * (E + pad)].view(T, E + pad)[:, :E] = False
    assert bool((flat[keep] == 7.0).all())


@pytest.mark.parametrize("E,groups,top_groups,k", [(64, 8, 3, 6), (256, 8, 4, 8), (32, 4, 1, 8), (128, 2, 1, 8), (512, 8, 4, 8),
                                                   (60, 4, 2, 6), (96, 4, 3, 8), (12, 6, 2, 3), (21, 7, 7, 5), (8, 8, 3, 3),
                                                   (1024, 32, 5, 16), (1000, 8, 4, 8), (24, 3, 1, 8), (160, 8, 3, 6), (128, 64, 10, 8),
                                                   (255, 3, 2, 8), (300, 5, 2, 8), (16, 8, 4, 4), (1024, 512, 40, 32), (204, 17, 4, 9),
                                                   (800, 100, 7, 12)])
@pytest.mark.parametrize("group_top", [1, 2])
def test_route_groups(E, groups, top_groups, k, group_top):
    rng = np.random.default_rng(E + groups)
    for kind, with_bias, dtype in (("sigmoid", True, torch.float32), ("softmax", False, torch.bfloat16)):
        logits = _logits(rng, 37, E, dtype)
        bias = torch.from_numpy(rng.normal(0, 0.1, E).astype(np.float32)).cuda() if with_bias else None
        kw = dict(groups=groups, top_groups=top_groups, group_top=group_top, renorm=True, scale=2.5)
        router, experts, weights = _route(logits, bias, k, kind, **kw)
        _compare(logits, bias, experts, weights, k, kind, **kw)
        _check_backward(rng, router, logits, experts, kind, True, 2.5)


@pytest.mark.parametrize("E,groups,top_groups,k,group_top", [(256, 8, 4, 8, 2), (192, 6, 2, 5, 1), (144, 9, 4, 8, 2), (136, 17, 3, 20, 2),
                                                             (256, 2, 1, 32, 2), (160, 8, 3, 6, 1), (216, 8, 4, 8, 2)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_many_tokens_as_few(E, groups, top_groups, k, group_top, dtype):
    """Large calls take two tokens per warp at a time: the same bits as small calls on parts of the rows, masks among them,
    and the plain form on the last rows (an odd number of them)."""
    rng = np.random.default_rng(E + k)
    T = 1501
    logits = _logits(rng, T, E, dtype)
    logits[5] = -float("inf")
    logits[6, ::3] = -float("inf")
    logits[1499, 4:] = -float("inf")
    logits[1500, 7] = float("nan")
    bias = torch.from_numpy(rng.normal(0, 0.1, E).astype(np.float32)).cuda()
    for kind, b in (("sigmoid", bias), ("softmax", None)):
        kw = dict(groups=groups, top_groups=top_groups, group_top=group_top, renorm=True, scale=2.5)
        _, experts, weights = _route(logits, b, k, kind, **kw)
        for begin, end in ((0, 700), (700, 1500), (1500, 1501)):
            _, e, w = _route(logits[begin:end], b, k, kind, **kw)
            assert torch.equal(e, experts[begin:end]) and torch.equal(w, weights[begin:end])
        tail = slice(1470, 1501)
        _compare(logits[tail], b, experts[tail], weights[tail], k, kind, **kw)


@pytest.mark.parametrize("E", [7, 64, 256, 600])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_equal_values_go_to_the_lowest_index(kind, E):
    rng = np.random.default_rng(E)
    k = min(6, E)
    x = rng.integers(-2, 3, (40, E)).astype(np.float32)
    x[0] = 1.0
    logits = torch.from_numpy(x).cuda()
    _, experts, weights = _route(logits, None, k, kind)
    assert np.array_equal(experts[0].cpu().numpy(), np.arange(k))
    _compare(logits, None, experts, weights, k, kind)
    if E % 4 == 0:
        kw = dict(groups=4, top_groups=2, group_top=2)
        _, experts, weights = _route(logits, None, k, kind, **kw)
        _compare(logits, None, experts, weights, k, kind, **kw)


@pytest.mark.parametrize("E,groups", [(6, 1), (64, 1), (64, 8), (60, 5), (256, 8), (300, 1), (700, 7)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_masked_experts_and_odd_values(kind, E, groups):
    rng = np.random.default_rng(E + groups)
    k = 4
    x = rng.normal(0, 1, (12, E)).astype(np.float32)
    lowest = np.finfo(np.float32).min
    x[0] = -np.inf                                     # nothing to choose
    x[1] = -np.inf
    x[1, [1, E - 1]] = [0.5, -3.0]                     # fewer than top_k
    x[2, ::2] = -np.inf
    x[3, 1:] = lowest                                  # a finite mask: chosen last, weight 0 (softmax) or 0 (sigmoid)
    x[4] = lowest                                      # a finite mask everywhere: equal scores (softmax), none above 0 (sigmoid)
    x[5] = -200.0                                      # sigmoid underflows: D = 0
    x[6, 0] = np.nan
    x[7, 2] = np.inf
    x[8] = 60.0 * rng.normal(0, 1, E)
    x[9] = np.inf
    x[10, E // 2] = 3e38
    bias = rng.normal(0, 0.05, E).astype(np.float32)
    bias[1] = -np.inf                                  # out of service
    for b in (None, bias):
        for renorm in (True, False):
            kw = dict(renorm=renorm, scale=1.5)
            if groups > 1:
                kw.update(groups=groups, top_groups=max(1, groups // 2), group_top=2)
            logits = torch.from_numpy(x).cuda()
            dev_bias = None if b is None else torch.from_numpy(b).cuda()
            router, experts, weights = _route(logits, dev_bias, k, kind, **kw)
            got_e, got_w = experts.cpu().numpy(), weights.cpu().numpy()
            for t in range(12):
                ref_e, ref_w, margin = R.route_row(x[t], b, k, kind, **kw)
                if margin >= 1e-5 or t in (0, 1, 4):
                    assert np.array_equal(got_e[t], ref_e), f"token {t}: {got_e[t]} instead of {ref_e}"
                    np.testing.assert_allclose(got_w[t], ref_w, rtol=_tol(x[t], E), atol=1e-37, err_msg=f"token {t}")
                assert ((got_e[t] >= -1) & (got_e[t] < E)).all()
                assert len(set(got_e[t][got_e[t] >= 0])) == (got_e[t] >= 0).sum()
                assert not np.isin(got_e[t][got_e[t] >= 0], np.nonzero(np.isneginf(x[t]))[0]).any()
            d_logits = torch.full_like(logits, 7.0)
            B.fp8mlp_route_backward(router, logits, experts, torch.ones_like(weights), d_logits)
            got = d_logits.cpu().numpy()
            assert not got[0].any()                    # a row without an expert has no gradient
            for t in (1, 2):
                ref = R.route_backward_row(x[t], got_e[t], np.ones(k), kind, renorm, 1.5)
                assert np.abs(got[t] - ref).max() <= 6 * _tol(x[t], E)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_backward_against_differences(kind, renorm):
    """The kernel's gradient against central differences of the 64-bit forward for the same choice: with step h their
    error is h^2 times the third derivative (below 1 here) and 1e-16 / h of rounding: 1e-9, well under the fp32 bar."""
    rng = np.random.default_rng(5)
    T, E, k, h = 6, 24, 3, 1e-5
    logits = _logits(rng, T, E, torch.float32)
    router, experts, _ = _route(logits, None, k, kind, renorm=renorm, scale=2.0)
    dw = rng.normal(0, 1, (T, k)).astype(np.float32)
    d_logits = torch.empty_like(logits)
    B.fp8mlp_route_backward(router, logits, experts, torch.from_numpy(dw).cuda(), d_logits)
    x, chosen, got = logits.cpu().numpy().astype(np.float64), experts.cpu().numpy(), d_logits.cpu().numpy()
    for t in range(T):
        for e in range(E):
            up, down = x[t].copy(), x[t].copy()
            up[e] += h
            down[e] -= h
            diff = (R.weights_of(up, chosen[t], kind, renorm, 2.0) - R.weights_of(down, chosen[t], kind, renorm, 2.0)) @ dw[t] / (2 * h)
            assert abs(got[t, e] - diff) <= 4 * _tol(x[t], E) * 2.0 * np.abs(dw[t]).max() + 1e-9


def test_backward_skips_unused_and_invalid_slots():
    rng = np.random.default_rng(8)
    T, E, k = 9, 40, 5
    logits = _logits(rng, T, E, torch.float32)
    chosen = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    chosen[0] = -1
    chosen[1, 2] = E
    chosen[2, 0] = -2 ** 31
    chosen[3, 4] = 2 ** 31 - 1
    for kind in ("softmax", "sigmoid"):
        for renorm in (True, False):
            router = B.new_router(E, k, KIND[kind], renormalise=renorm)
            _check_backward(rng, router, logits, torch.from_numpy(chosen).cuda(), kind, renorm, 1.0)


def test_zero_tokens_and_other_stream():
    router = B.new_router(8, 2)
    empty = torch.empty((0, 8), device="cuda")
    B.fp8mlp_route(router, empty, None, torch.empty((0, 2), dtype=torch.int32, device="cuda"), torch.empty((0, 2), device="cuda"))
    B.fp8mlp_route_backward(router, empty, torch.empty((0, 2), dtype=torch.int32, device="cuda"), torch.empty((0, 2), device="cuda"),
                            torch.empty((0, 8), device="cuda"))
    rng = np.random.default_rng(2)
    side = torch.cuda.Stream()
    logits = torch.from_numpy(rng.normal(0, 1, (4000, 64)).astype(np.float32)).cuda()
    _, e0, w0 = _route(logits, None, 4, "softmax")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late = torch.zeros_like(logits)
        torch.cuda._sleep(2_000_000)
        late.copy_(logits)                            # the kernel has to wait for this copy: same stream, not the default one
        _, e1, w1 = _route(late, None, 4, "softmax")
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(e0, e1) and torch.equal(w0, w1)


def test_route_repeats_bit_for_bit():
    rng = np.random.default_rng(3)
    logits = _logits(rng, 5000, 256, torch.float32)
    bias = torch.from_numpy(rng.normal(0, 0.1, 256).astype(np.float32)).cuda()
    kw = dict(groups=8, top_groups=4, group_top=2)
    first = _route(logits, bias, 8, "sigmoid", **kw)[1:]
    for _ in range(3):
        again = _route(logits, bias, 8, "sigmoid", **kw)[1:]
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("E,T", [(6, 40), (64, 33), (100, 9), (256, 1300), (512, 7)])
def test_arrays_on_4_byte_boundaries(E, T):
    """Bias, experts, weights and their gradients 4 bytes past a 32-byte boundary: the same bits as aligned ones."""
    rng = np.random.default_rng(E)
    k = min(E, 5)
    logits = _logits(rng, T, E, torch.float32)
    bias = torch.from_numpy(rng.normal(0, 0.1, E).astype(np.float32)).cuda()
    off = lambda n, dtype: torch.full((n + 9,), 7, dtype=dtype, device="cuda")
    bias_, experts_, weights_, dw_ = off(E, torch.float32), off(T * k, torch.int32), off(T * k, torch.float32), off(T * k, torch.float32)
    bias_[1:E + 1] = bias
    router, experts, weights = _route(logits, bias, k, "sigmoid")
    B.fp8mlp_route(router, logits, bias_[1:E + 1], experts_[1:T * k + 1].view(T, k), weights_[1:T * k + 1].view(T, k))
    assert torch.equal(experts_[1:T * k + 1].view(T, k), experts) and torch.equal(weights_[1:T * k + 1].view(T, k), weights)
    for a in (experts_, weights_):
        assert bool((a[0] == 7) & (a[T * k + 1:] == 7).all())
    dw = torch.from_numpy(rng.normal(0, 1, (T, k)).astype(np.float32)).cuda()
    dw_[1:T * k + 1] = dw.flatten()
    for kind in ("sigmoid", "softmax"):
        router = B.new_router(E, k, KIND[kind], renormalise=False)
        a, b = torch.empty_like(logits), torch.empty_like(logits)
        B.fp8mlp_route_backward(router, logits, experts, dw, a)
        B.fp8mlp_route_backward(router, logits, experts_[1:T * k + 1].view(T, k), dw_[1:T * k + 1].view(T, k), b)
        assert torch.equal(a, b)


@pytest.mark.parametrize("E", [1, 8, 60, 1024])
def test_update_bias(E):
    rng = np.random.default_rng(E)
    counts = rng.integers(0, 50, E).astype(np.int32)
    if E > 4:
        counts[0] = counts.sum()                       # uneven
    bias = rng.normal(0, 0.1, E).astype(np.float32)
    dev = torch.from_numpy(bias.copy()).cuda()
    B.fp8mlp_route_update_bias(torch.from_numpy(counts).cuda(), 1e-3, dev)
    sign = np.sign(int(counts.sum()) - counts.astype(np.int64) * E).astype(np.float32)
    assert np.array_equal(dev.cpu().numpy(), bias + np.float32(1e-3) * sign)


def _softmax_of_chosen(x, experts):
    """e^x_j / sum_i e^x_i over the chosen experts, in 64 bits: what renormalised softmax weights are, whatever the rest of the row."""
    v = np.exp(x[experts].astype(np.float64) - x[experts].max())
    return v / v.sum()


@pytest.mark.parametrize("E,groups,top_groups", [(3, 1, 1), (12, 1, 1), (16, 4, 2), (40, 1, 1), (256, 1, 1), (256, 8, 4), (66, 33, 20),
                                                 (600, 1, 1)])
def test_renormalised_softmax_far_below_the_rows_maximum(E, groups, top_groups):
    """An expert out of service (bias -inf), or held back by a finite bias, may stand so far above the others that their scores
    leave fp32.  Their renormalised weights are still the softmax over the chosen logits, and the gradient is that formula's.
    Rows of every distance share warps; rows that lose nothing keep the bits that they have alone.  A weight has in addition the
    subnormal spacing 2^-149 of its score over D >= 2^-64."""
    rng = np.random.default_rng(E + groups)
    k, per = min(2 if E < 12 else 5, E - 1), E // groups
    gaps = np.array([0.0, 120.0, 3.0, 40.0, 45.0, 60.0, 80.0, 86.0, 88.0, 95.0, 100.0, 103.0, 104.0, 106.0, 110.0, 150.0, 1e4, 3e38, 0.5],
                    np.float32)
    x = rng.normal(0, 1, (gaps.size, E)).astype(np.float32)
    x[:, 0] = gaps
    if E == 3:
        x[1] = [0.0, -120.0, -121.0]
    for out_of_service in (-np.inf, -4.0):
        bias = rng.normal(0, 1e-3, E).astype(np.float32)
        bias[0] = out_of_service
        if groups > 1:
            bias[:per] = out_of_service
        logits, dev_bias = torch.from_numpy(x).cuda(), torch.from_numpy(bias).cuda()
        kw = dict(groups=groups, top_groups=top_groups, group_top=min(2, per), renorm=True, scale=2.5)
        router, experts, weights = _route(logits, dev_bias, k, "softmax", **kw)
        dw = rng.normal(0, 1, (gaps.size, k)).astype(np.float32)
        if E == 3:
            dw[1] = [1.0, -1.0]
        d_logits = torch.full_like(logits, 7.0)
        B.fp8mlp_route_backward(router, logits, experts, torch.from_numpy(dw).cuda(), d_logits)
        got_e, got_w, got_dx = experts.cpu().numpy(), weights.cpu().numpy(), d_logits.cpu().numpy().astype(np.float64)
        for t in range(gaps.size):
            assert (got_e[t] > 0).all() and len(set(got_e[t])) == k
            r = _softmax_of_chosen(x[t], got_e[t])
            np.testing.assert_allclose(got_w[t], 2.5 * r, rtol=_tol(x[t], E), atol=2.5 * 2.0 ** -85, err_msg=f"gap {gaps[t]}")
            want = np.zeros(E)
            want[got_e[t]] = 2.5 * r * (dw[t] - (dw[t] * r).sum())
            allowed = 4 * _tol(x[t], E) * 2.5 * np.abs(dw[t]).max() + 2.0 ** -24 * np.abs(want)
            assert (np.abs(got_dx[t] - want) <= allowed).all(), f"gap {gaps[t]}"
        for t in (0, 2, 18):
            _, e, w = _route(logits[t:t + 1], dev_bias, k, "softmax", **kw)
            assert torch.equal(e[0], experts[t]) and torch.equal(w[0], weights[t])


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_backward_of_finite_masks_and_lost_scores(kind, renorm):
    """Rows under a finite mask (all but one expert, and all of them), rows of equal logits whose sigmoid is 0 in fp32, and a row
    that spreads over hundreds: the gradient follows from the forward's weights."""
    rng = np.random.default_rng(17)
    E, k = 24, 4
    x = rng.normal(0, 1, (4, E)).astype(np.float32)
    lowest = np.finfo(np.float32).min
    x[0, 1:] = lowest
    x[1] = lowest
    x[2] = -200.0
    x[3] *= 100.0
    logits = torch.from_numpy(x).cuda()
    router, experts, weights = _route(logits, None, k, kind, renorm=renorm, scale=1.5)
    dw = rng.normal(0, 1, (4, k)).astype(np.float32)
    d_logits = torch.full_like(logits, 7.0)
    B.fp8mlp_route_backward(router, logits, experts, torch.from_numpy(dw).cuda(), d_logits)
    got_e, got = experts.cpu().numpy(), d_logits.cpu().numpy()
    if kind == "sigmoid":
        assert not got[1:3].any() and not weights[1:3].any()         # weights that are 0 whatever the logits do
    for t in range(4):
        ref = R.route_backward_row(x[t], got_e[t], dw[t], kind, renorm, 1.5)
        assert (np.abs(got[t] - ref) <= 4 * _tol(x[t], E) * 1.5 * np.abs(dw[t]).max() + 2.0 ** -24 * np.abs(ref)).all(), f"row {t}"


@pytest.mark.parametrize("E,groups", [(16, 4), (24, 6), (66, 33), (256, 16), (300, 20), (700, 50), (960, 32)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_groups_under_the_lowest_bias(kind, E, groups):
    """A bias of the type's lowest value puts experts last, not out of service: two of them add up beyond fp32, and their group
    still stands before one that has nothing to choose."""
    rng = np.random.default_rng(E)
    per = E // groups
    k = per + 1                                        # the last group's experts and one more
    x = rng.normal(0, 1, (9, E)).astype(np.float32)
    x[:, :per] = -np.inf                               # the first group is masked
    bias = np.full(E, np.finfo(np.float32).min, np.float32)
    bias[-per:] = rng.normal(0, 0.1, per)              # and only the last one is in use without a bias of that size
    kw = dict(groups=groups, top_groups=2, group_top=2, renorm=False, scale=1.0)
    _, experts, weights = _route(torch.from_numpy(x).cuda(), torch.from_numpy(bias).cuda(), k, kind, **kw)
    got = experts.cpu().numpy()
    for t in range(9):
        ref_e, ref_w, _ = R.route_row(x[t], bias, k, kind, **kw)
        assert ref_e[-1] == per                        # the first of the second group
        # near scores of the last group may be ordered either way
        assert set(got[t]) == set(ref_e) and got[t][-1] == per
        order = np.argsort(got[t])
        np.testing.assert_allclose(weights[t].cpu().numpy()[order], ref_w[np.argsort(ref_e)], rtol=_tol(x[t], E), atol=1e-38)


@pytest.mark.parametrize("E,groups,top_groups,k", [(256, 8, 4, 8), (160, 8, 3, 6), (144, 9, 4, 4)])
@pytest.mark.parametrize("T", [2301, 5003, 7001, 9001, 10901])
def test_any_number_of_tokens_as_few(E, groups, top_groups, k, T):
    """One or two tokens per warp, by the number of tokens: the same bits as small calls on parts of the rows."""
    rng = np.random.default_rng(T + E)
    logits = _logits(rng, T, E, torch.float32)
    logits[11] = -float("inf")
    logits[T - 2, 5:] = -float("inf")
    bias = torch.from_numpy(rng.normal(0, 0.1, E).astype(np.float32)).cuda()
    for kind, b in (("sigmoid", bias), ("softmax", bias), ("softmax", None)):
        kw = dict(groups=groups, top_groups=top_groups, group_top=2, renorm=True, scale=2.5)
        _, experts, weights = _route(logits, b, k, kind, **kw)
        for begin in range(0, T, 1000):
            _, e, w = _route(logits[begin:begin + 1000], b, k, kind, **kw)
            assert torch.equal(e, experts[begin:begin + 1000]) and torch.equal(w, weights[begin:begin + 1000])
        _compare(logits[T - 20:], b, experts[T - 20:], weights[T - 20:], k, kind, **kw)


@pytest.mark.parametrize("E,groups,top_groups,k", [(2, 2, 1, 1), (2, 2, 2, 2), (6, 2, 1, 3), (10, 2, 1, 4), (14, 2, 2, 9), (16, 2, 1, 8), (16, 2, 2, 16),
                                                   (9, 3, 2, 4), (15, 3, 1, 5), (20, 4, 3, 15), (28, 7, 2, 8), (8, 4, 3, 5)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_top", [1, 2])
def test_few_experts_in_groups(kind, E, groups, top_groups, k, group_top):
    """Tokens on two, four and eight lanes whose groups are lanes of their own; nearly every row is decided by more than a rounding
    and has to be equal."""
    rng = np.random.default_rng(100 * E + groups)
    for T, dtype, with_bias in ((1, torch.float32, False), (131, torch.float32, True), (257, torch.bfloat16, False)):
        logits = _logits(rng, T, E, dtype)
        if T > 100:
            logits[3] = -float("inf")
            logits[4, 1:] = -float("inf")
            logits[5, : E // groups] = -float("inf")
        bias = torch.from_numpy(rng.normal(0, 0.1, E).astype(np.float32)).cuda() if with_bias else None
        kw = dict(groups=groups, top_groups=top_groups, group_top=group_top, renorm=True, scale=2.5)
        router, experts, weights = _route(logits, bias, k, kind, **kw)
        _compare(logits, bias, experts, weights, k, kind, **kw)
        x, b = logits.float().cpu().numpy(), None if bias is None else bias.cpu().numpy()
        decided = [t for t in range(T) if R.route_row(x[t], b, k, kind, **kw)[2] >= 1e-5]
        assert len(decided) >= 0.9 * T
        _check_backward(rng, router, logits, experts, kind, True, 2.5)
