"""fp8mlp_dispatch_plan, fp8mlp_dispatch, fp8mlp_combine and fp8mlp_combine_backward against plain implementations.

Plans, copied rows and the rows of dye (one fp32 product, rounded once) are compared bit for bit.  A sum of k products is
held to k 2^-24 of the sum of their absolute values and one rounding to the output's type; a dot product over d elements,
summed over threads and then in a tree, to (d / 32 + 32) 2^-24 of the sum of the absolute products."""
import numpy as np
import pytest
import torch

import experts_reference as R
from paper_2409_12517_b200 import binding as B

pytestmark = pytest.mark.gpu

DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])


def _plan(experts, E):
    T, k = experts.shape
    dev = torch.from_numpy(experts).cuda()
    counts = torch.full((E,), -5, dtype=torch.int32, device="cuda")
    offsets = torch.full((E + 1,), -5, dtype=torch.int32, device="cuda")
    rows = torch.full((T, k), -5, dtype=torch.int32, device="cuda")
    B.fp8mlp_dispatch_plan(dev, E, counts, offsets, rows)
    return counts, offsets, rows


def _experts(rng, T, k, E, unused=0.0):
    """k different experts per token where E allows it."""
    if T == 0:
        return np.zeros((0, k), np.int32)
    e = np.stack([rng.permutation(E)[:k] for _ in range(T)]) if k <= E and T <= 4000 else rng.integers(0, E, (T, k))
    e = e.astype(np.int32).reshape(T, k)
    e[rng.random(T) < unused] = -1
    return e


@pytest.mark.parametrize("T,k,E", [(0, 2, 8), (1, 1, 1), (1, 8, 256), (4, 8, 256), (3, 1, 1024), (16, 2, 8), (33, 3, 5), (127, 7, 60),
                                   (257, 8, 64), (1000, 6, 1000), (4096, 4, 1), (5000, 8, 1024), (20001, 3, 33), (70000, 8, 256),
                                   (300000, 2, 8)])
def test_plan(T, k, E):
    rng = np.random.default_rng(T + E)
    for unused in (0.0, 0.3):
        experts = _experts(rng, T, k, E, unused)
        if unused and T > 2:                           # outside the range: unused slots
            experts[0, 0], experts[1, 0], experts[2, 0] = E, -2 ** 31, 2 ** 31 - 1
        counts, offsets, rows = _plan(experts, E)
        rc, ro, rr = R.plan(np.where((experts < 0) | (experts >= E), -1, experts), E)
        assert np.array_equal(counts.cpu().numpy(), rc)
        assert np.array_equal(offsets.cpu().numpy(), ro)
        assert np.array_equal(rows.cpu().numpy(), rr)


def test_plan_all_unused_and_one_expert_for_all():
    counts, offsets, rows = _plan(np.full((50, 4), -1, np.int32), 16)
    assert not counts.any() and not offsets.any() and bool((rows == -1).all())
    counts, offsets, rows = _plan(np.full((3000, 1), 7, np.int32), 16)
    assert int(counts[7]) == 3000 and torch.equal(rows.flatten().cpu(), torch.arange(3000, dtype=torch.int32))


def _tokens(rng, T, d, dtype, pad=0, scale=1.0):
    flat = torch.full((T * (d + pad) + 32,), 9.0, dtype=dtype, device="cuda")
    view = flat[:T * (d + pad)].view(T, d + pad)[:, :d]
    view.copy_(torch.from_numpy(rng.normal(0, scale, (T, d)).astype(np.float32)))
    return flat, view


SHAPES = pytest.mark.parametrize("T,k,E,d,pad", [(1, 1, 1, 16, 0), (1, 8, 256, 4096, 0), (5, 2, 8, 48, 16), (67, 4, 60, 512, 0),
                                                 (33, 6, 64, 272, 8), (200, 3, 4, 1040, 32), (9, 32, 40, 160, 0), (300, 9, 12, 64, 0),
                                                 (3, 2, 8, 8192, 0), (2, 5, 8, 12304, 0)])


@DTYPES
@SHAPES
def test_dispatch(T, k, E, d, pad, dtype):
    rng = np.random.default_rng(T * d)
    experts = _experts(rng, T, k, E, 0.2)
    _, offsets, rows = _plan(experts, E)
    _, x = _tokens(rng, T, d, dtype, pad)
    n = T * k
    xe = torch.full((n + 3, d), 5.0, dtype=dtype, device="cuda")
    B.fp8mlp_dispatch(x, rows, xe)
    want = torch.full((n + 3, d), 5.0, dtype=dtype)
    r = rows.cpu().numpy()
    for t in range(T):
        for j in range(k):
            if r[t, j] >= 0:
                want[r[t, j]] = x[t].cpu()
    assert torch.equal(xe.cpu(), want)
    # fewer rows than the plan names, and rows outside: nothing is written beyond
    short = torch.full((n + 3, d), 5.0, dtype=dtype, device="cuda")
    limit = max(1, n // 2)
    bad = rows.clone()
    bad[0, 0] = 2 ** 31 - 1
    B.fp8mlp_dispatch(x, bad, short[:limit])
    assert bool((short[limit:] == 5.0).all())


@DTYPES
@SHAPES
def test_combine(T, k, E, d, pad, dtype):
    rng = np.random.default_rng(T * d + 1)
    experts = _experts(rng, T, k, E, 0.2)
    _, _, rows = _plan(experts, E)
    n = T * k
    ye = torch.from_numpy(rng.normal(0, 1, (n, d)).astype(np.float32)).cuda().to(dtype)
    weights = torch.from_numpy(rng.random((T, k)).astype(np.float32)).cuda()
    if T > 1:
        rows[-1] = -1                                  # a token without any expert
        rows[0, 0] = n                                 # outside: adds nothing
    for w in (weights, None):
        flat, y = _tokens(rng, T, d, dtype, pad)
        B.fp8mlp_combine(ye, rows, w, y)
        want, size = R.combine(ye.float().cpu().numpy(), rows.cpu().numpy(), None if w is None else w.cpu().numpy())
        step = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -23
        err = np.abs(y.float().cpu().numpy() - want)
        assert (err <= k * 2.0 ** -24 * size + 0.51 * step * np.abs(want)).all()
        if T > 1:
            assert not y[-1].any()
        if pad:
            assert bool((flat[:T * (d + pad)].view(T, d + pad)[:, d:] == 9.0).all())
        assert bool((flat[T * (d + pad):] == 9.0).all())


@DTYPES
@SHAPES
def test_combine_backward(T, k, E, d, pad, dtype):
    rng = np.random.default_rng(T * d + 2)
    experts = _experts(rng, T, k, E, 0.2)
    _, _, rows = _plan(experts, E)
    n = T * k
    ye = torch.from_numpy(rng.normal(0, 1, (n, d)).astype(np.float32)).cuda().to(dtype)
    weights = torch.from_numpy(rng.random((T, k)).astype(np.float32)).cuda()
    _, dy = _tokens(rng, T, d, dtype, pad)
    if T > 1:
        rows[-1] = -1
        rows[0, 0] = n
    dye = torch.full((n + 2, d), 5.0, dtype=dtype, device="cuda")
    d_weights = torch.full((T, k), float("nan"), device="cuda")
    B.fp8mlp_combine_backward(dy, ye, rows, weights, dye[:n], d_weights)
    want = torch.full((n + 2, d), 5.0, dtype=dtype)
    dw, size = np.zeros((T, k)), np.zeros((T, k))
    r, g, v = rows.cpu().numpy(), dy.float().cpu(), ye.float().cpu().numpy().astype(np.float64)
    for t in range(T):
        for j in range(k):
            if 0 <= r[t, j] < n:
                want[r[t, j]] = (weights[t, j].cpu() * g[t]).to(dtype)
                prod = g[t].numpy().astype(np.float64) * v[r[t, j]]
                dw[t, j], size[t, j] = prod.sum(), np.abs(prod).sum()
    assert torch.equal(dye.cpu(), want)
    assert (np.abs(d_weights.cpu().numpy() - dw) <= (d / 32 + 32) * 2.0 ** -24 * size).all()


@DTYPES
@pytest.mark.parametrize("T,k,d", [(37, 1, 4112), (50, 1, 80), (21, 2, 2064), (9, 3, 528), (11, 4, 272), (5, 8, 1040), (3, 11, 48)])
def test_rows_on_16_byte_boundaries(T, k, d, dtype):
    """Buffers that start 16 bytes past a 32-byte boundary, between guard zones: the same bits as on aligned buffers (sums run
    over the slots in order either way; dot products are held to their bar), guards intact."""
    rng = np.random.default_rng(T + d)
    E, n = 16, T * k
    experts = _experts(rng, T, k, E, 0.2)
    _, _, rows = _plan(experts, E)
    weights = torch.from_numpy(rng.random((T, k)).astype(np.float32)).cuda()
    shift = 16 // torch.empty(0, dtype=dtype).element_size()
    guards = []

    def place(r, content=None):
        flat = torch.full((2 * shift + r * d + 64,), 7.0, dtype=dtype, device="cuda")
        view = flat[shift:shift + r * d].view(r, d)
        assert view.data_ptr() % 32 == 16
        if content is not None:
            view.copy_(content)
        guards.append((flat, shift, r * d))
        return view

    draw = lambda r: torch.from_numpy(rng.normal(0, 1, (r, d)).astype(np.float32)).cuda().to(dtype)
    x, ye, dy = draw(T), draw(n), draw(T)
    xe, y, y1, dye, dw = torch.zeros_like(ye), torch.empty_like(x), torch.empty_like(x), torch.zeros_like(ye), torch.empty((T, k), device="cuda")
    B.fp8mlp_dispatch(x, rows, xe)
    B.fp8mlp_combine(ye, rows, weights, y)
    B.fp8mlp_combine(ye, rows, None, y1)
    B.fp8mlp_combine_backward(dy, ye, rows, weights, dye, dw)
    x_, ye_, dy_, xe_, dye_ = place(T, x), place(n, ye), place(T, dy), place(n, torch.zeros_like(ye)), place(n, torch.zeros_like(ye))
    yw_, y1_, dw_ = place(T), place(T), torch.empty_like(dw)
    B.fp8mlp_dispatch(x_, rows, xe_)
    B.fp8mlp_combine(ye_, rows, weights, yw_)
    B.fp8mlp_combine(ye_, rows, None, y1_)
    B.fp8mlp_combine_backward(dy_, ye_, rows, weights, dye_, dw_)
    for a, b in ((xe, xe_), (y, yw_), (y1, y1_), (dye, dye_)):
        assert torch.equal(a, b)
    r = rows.cpu().numpy()
    size = np.array([[np.abs(dy[t].double().cpu().numpy() * ye[r[t, j]].double().cpu().numpy()).sum() if r[t, j] >= 0 else 0.0
                      for j in range(k)] for t in range(T)])
    assert (np.abs((dw - dw_).cpu().numpy()) <= 2 * (d / 32 + 32) * 2.0 ** -24 * size).all()
    want, _ = R.combine(ye.float().cpu().numpy(), r, weights.cpu().numpy())
    step = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -23
    assert (np.abs(y.float().cpu().numpy() - want) <= (k * 2.0 ** -24 * 8 + 0.51 * step * np.abs(want))).all()
    for flat, s, count in guards:
        assert bool((flat[:s] == 7.0).all()) and bool((flat[s + count:] == 7.0).all())


def test_combine_gradient_against_differences():
    """<dy, combine(...)> is linear in each argument: differences of the 64-bit form are exact up to its rounding, so the
    kernel's gradients are held to their own fp32 bar."""
    rng = np.random.default_rng(11)
    T, k, E, d = 5, 3, 6, 32
    experts = _experts(rng, T, k, E)
    _, _, rows = _plan(experts, E)
    ye = rng.normal(0, 1, (T * k, d)).astype(np.float32)
    w = rng.random((T, k)).astype(np.float32)
    dy = rng.normal(0, 1, (T, d)).astype(np.float32)
    dev = lambda a: torch.from_numpy(a).cuda()
    dye, dw = torch.zeros((T * k, d), device="cuda"), torch.zeros((T, k), device="cuda")
    B.fp8mlp_combine_backward(dev(dy), dev(ye), rows, dev(w), dye, dw)
    r = rows.cpu().numpy()
    f = lambda ye_, w_: (R.combine(ye_, r, w_)[0] * dy.astype(np.float64)).sum()
    ye64, w64 = ye.astype(np.float64), w.astype(np.float64)
    for t in range(T):
        for j in range(k):
            up = w64.copy()
            up[t, j] += 1.0
            assert abs(float(dw[t, j]) - (f(ye64, up) - f(ye64, w64))) <= 1e-5
    for i in range(0, T * k, 4):
        for c in range(0, d, 7):
            up = ye64.copy()
            up[i, c] += 1.0
            assert abs(float(dye[i, c]) - (f(up, w64) - f(ye64, w64))) <= 1e-6


def test_row_offsets_beyond_32_bits():
    """Rows whose byte offset passes 2^32 (5.2 GB of rows): copies, sums and gradients at both ends of the buffer."""
    d, n, k = 32768, 80000, 2
    rows = torch.tensor([[0, n - 1], [n - 2, 40000], [65536, 1]], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(0)
    x = torch.from_numpy(rng.normal(0, 1, (3, d)).astype(np.float32)).cuda().bfloat16()
    xe = torch.empty((n, d), dtype=torch.bfloat16, device="cuda")
    B.fp8mlp_dispatch(x, rows, xe)
    for t in range(3):
        for j in range(k):
            assert torch.equal(xe[int(rows[t, j])], x[t])
    y = torch.empty_like(x)
    B.fp8mlp_combine(xe, rows, None, y)
    assert torch.equal(y, (x.float() * 2).bfloat16())
    w = torch.tensor([[0.5, 1.0], [2.0, 0.25], [1.0, 4.0]], device="cuda")
    dye, dw = torch.empty_like(xe), torch.empty((3, k), device="cuda")
    B.fp8mlp_combine_backward(x, xe, rows, w, dye, dw)
    for t in range(3):
        for j in range(k):
            assert torch.equal(dye[int(rows[t, j])], (w[t, j] * x[t].float()).bfloat16())
    norm2 = (x.double() ** 2).sum(-1)
    assert torch.allclose(dw.double(), norm2[:, None].expand(3, k), rtol=1e-4)


def test_other_stream_and_repeats():
    rng = np.random.default_rng(4)
    T, k, E, d = 900, 4, 16, 256
    experts = _experts(rng, T, k, E)
    _, _, rows = _plan(experts, E)
    ye = torch.from_numpy(rng.normal(0, 1, (T * k, d)).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.random((T, k)).astype(np.float32)).cuda()
    y0, y1 = torch.empty((T, d), device="cuda"), torch.empty((T, d), device="cuda")
    dye0, dye1, dw0, dw1 = torch.empty_like(ye), torch.empty_like(ye), torch.empty_like(w), torch.empty_like(w)
    B.fp8mlp_combine(ye, rows, w, y0)
    B.fp8mlp_combine_backward(y0, ye, rows, w, dye0, dw0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        late = torch.empty_like(ye)
        late.copy_(ye)
        B.fp8mlp_combine(late, rows, w, y1)
        B.fp8mlp_combine_backward(y1, late, rows, w, dye1, dw1)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y0, y1) and torch.equal(dye0, dye1) and torch.equal(dw0, dw1)


@pytest.mark.parametrize("T,k,E", [(1025, 1, 5), (2049, 3, 60), (4099, 5, 33), (8193, 2, 1000), (20011, 7, 257)])
def test_plan_with_ragged_warps(T, k, E):
    """Numbers of slots and experts that leave some lanes of a warp without work before each barrier of the cluster; repeated, the
    same bits."""
    rng = np.random.default_rng(T)
    experts = _experts(rng, T, k, E, 0.1)
    first = _plan(experts, E)
    for got, want in zip(first, R.plan(experts, E)):
        assert np.array_equal(got.cpu().numpy(), want)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(first, _plan(experts, E)))
