"""Without a GPU: what the expert and clipping entry points refuse, before anything is launched, and the plain
implementations that the GPU tests compare with against brute force and differences."""
import ctypes as C

import numpy as np
import pytest
import torch

import experts_reference as R
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


def test_route_refusals(lib):
    ok = dict(n_experts=8, top_k=2)
    route = lambda r, T=4, x=P, dt=B.F32, ld=8, bias=None, e=P, w=P: lib.fp8mlp_route(r, T, x, dt, ld, bias, e, w, None)
    for bad in (dict(n_experts=0), dict(n_experts=1025), dict(top_k=0), dict(top_k=9), dict(n_experts=64, top_k=33),
                dict(n_groups=0), dict(n_groups=3), dict(n_groups=4, top_groups=0), dict(n_groups=4, top_groups=5),
                dict(n_groups=8, top_groups=1)):
        assert route(B.new_router(**{**ok, **bad}), ld=2000) == B.ERR_SHAPE, bad
    for bad in (dict(score=2), dict(score=-1), dict(group_top=0), dict(group_top=3)):
        assert route(B.new_router(**{**ok, **bad})) == B.ERR_ARG, bad
    r = B.new_router(**ok)
    assert route(None) == B.ERR_ARG
    assert route(r, T=-1) == B.ERR_SHAPE and route(r, ld=7) == B.ERR_SHAPE
    assert route(r, dt=2) == B.ERR_ARG
    assert route(r, x=None) == B.ERR_ARG and route(r, e=None) == B.ERR_ARG and route(r, w=None) == B.ERR_ARG
    assert route(r, x=P + 2) == B.ERR_ALIGN and route(r, x=P + 1, dt=B.BF16) == B.ERR_ALIGN
    assert route(r, bias=P + 2) == B.ERR_ALIGN and route(r, e=P + 1) == B.ERR_ALIGN and route(r, w=P + 2) == B.ERR_ALIGN
    assert route(r, T=0, x=None, e=None, w=None, ld=0) == B.OK
    back = lambda r, T=4, x=P, dt=B.F32, ld=8, e=P, w=P, dx=2 * P, ldd=8: lib.fp8mlp_route_backward(r, T, x, dt, ld, e, w, dx, ldd, None)
    assert back(None) == B.ERR_ARG and back(r, dt=5) == B.ERR_ARG
    assert back(r, ld=7) == B.ERR_SHAPE and back(r, ldd=7) == B.ERR_SHAPE and back(r, T=-2) == B.ERR_SHAPE
    assert back(r, x=None) == B.ERR_ARG and back(r, dx=None) == B.ERR_ARG and back(r, e=None) == B.ERR_ARG and back(r, w=None) == B.ERR_ARG
    assert back(r, dx=P, x=P) == B.ERR_ARG             # not in place
    assert back(r, dx=P + 2) == B.ERR_ALIGN and back(r, w=P + 2) == B.ERR_ALIGN
    assert back(r, T=0) == B.OK
    bias = lib.fp8mlp_route_update_bias
    assert bias(0, P, 0.1, P, None) == B.ERR_SHAPE and bias(1025, P, 0.1, P, None) == B.ERR_SHAPE
    assert bias(8, None, 0.1, P, None) == B.ERR_ARG and bias(8, P, 0.1, None, None) == B.ERR_ARG
    assert bias(8, P + 2, 0.1, P, None) == B.ERR_ALIGN


def test_plan_refusals(lib):
    plan = lambda T=4, k=2, E=8, e=P, c=P, o=P, r=2 * P: lib.fp8mlp_dispatch_plan(T, k, E, e, c, o, r, None)
    assert plan(T=-1) == B.ERR_SHAPE and plan(k=0) == B.ERR_SHAPE and plan(k=33) == B.ERR_SHAPE
    assert plan(E=0) == B.ERR_SHAPE and plan(E=1025) == B.ERR_SHAPE and plan(T=2 ** 30, k=4) == B.ERR_SHAPE
    assert plan(e=None) == B.ERR_ARG and plan(c=None) == B.ERR_ARG and plan(o=None) == B.ERR_ARG and plan(r=None) == B.ERR_ARG
    assert plan(r=P) == B.ERR_ARG                      # rows is not experts
    assert plan(e=P + 2) == B.ERR_ALIGN and plan(c=P + 1) == B.ERR_ALIGN and plan(o=P + 2) == B.ERR_ALIGN and plan(r=P + 2) == B.ERR_ALIGN


def test_row_refusals(lib):
    disp = lambda T=4, k=2, d=32, dt=B.BF16, x=P, ld=32, r=P, xe=2 * P, n=8: lib.fp8mlp_dispatch(T, k, d, dt, x, ld, r, xe, n, None)
    comb = lambda T=4, k=2, d=32, dt=B.BF16, y=P, ld=32, r=P, ye=2 * P, n=8, w=P: lib.fp8mlp_combine(T, k, d, dt, ye, n, r, w, y, ld, None)
    back = lambda T=4, k=2, d=32, dt=B.BF16, y=P, ld=32, r=P, ye=2 * P, n=8, w=P, dye=3 * P, dw=P: lib.fp8mlp_combine_backward(
        T, k, d, dt, y, ld, ye, n, r, w, dye, dw, None)
    for call, token, expert in ((disp, "x", "xe"), (comb, "y", "ye"), (back, "y", "ye")):
        assert call(dt=2) == B.ERR_ARG
        assert call(T=-1) == B.ERR_SHAPE and call(n=-1) == B.ERR_SHAPE and call(T=2 ** 31) == B.ERR_SHAPE
        assert call(d=0) == B.ERR_SHAPE and call(d=24) == B.ERR_SHAPE and call(k=0) == B.ERR_SHAPE and call(k=33) == B.ERR_SHAPE
        assert call(ld=16) == B.ERR_SHAPE
        assert call(**{token: None}) == B.ERR_ARG and call(r=None) == B.ERR_ARG and call(**{expert: None}) == B.ERR_ARG
        assert call(**{token: P + 8}) == B.ERR_ALIGN and call(**{expert: P + 8}) == B.ERR_ALIGN and call(ld=36) == B.ERR_ALIGN
        assert call(r=P + 2) == B.ERR_ALIGN
        assert call(**{token: 2 * P}) == B.ERR_ARG     # token and expert rows are different buffers
        assert call(T=0) == B.OK
    assert comb(w=P + 2) == B.ERR_ALIGN
    assert back(w=None) == B.ERR_ARG and back(dw=None) == B.ERR_ARG and back(dye=None) == B.ERR_ARG
    assert back(dye=2 * P) == B.ERR_ARG                # dye is not ye
    assert back(dye=P + 8) == B.ERR_ALIGN and back(dw=P + 2) == B.ERR_ALIGN


def test_clip_refusals(lib):
    def grads(*entries):
        arr = (B._GradTensor * max(len(entries), 1))()
        for a, (g, out, n, dt) in zip(arr, entries):
            a.g, a.out, a.n, a.dtype = g, out, n, dt
        return arr, len(entries)

    good = (P, P, 16, B.F32)
    for call in (lib.fp8mlp_grad_norm, lib.fp8mlp_clip_grads):
        run = lambda lst, kind=B.NORM_L2, m=1.0, out=P, ws=P, call=call: call(lst[0], lst[1], kind, m, out, ws, None)
        assert run(grads(good), kind=2) == B.ERR_ARG and run(grads(good), kind=-1) == B.ERR_ARG
        assert run(grads(good), m=-1.0) == B.ERR_ARG and run(grads(good), m=float("nan")) == B.ERR_ARG
        assert run(grads(good), out=None) == B.ERR_ARG and run(grads(good), ws=None) == B.ERR_ARG
        assert run((None, 1)) == B.ERR_ARG and run((grads(good)[0], -1)) == B.ERR_ARG
        assert run(grads((P, P, 16, 7))) == B.ERR_ARG and run(grads((None, P, 16, B.F32))) == B.ERR_ARG
        assert run(grads((P, P, -1, B.F32))) == B.ERR_SHAPE
        assert run(grads((P + 2, P, 16, B.F32))) == B.ERR_ALIGN and run(grads((P + 1, P, 16, B.BF16))) == B.ERR_ALIGN
        assert run(grads(good), out=P + 2) == B.ERR_ALIGN and run(grads(good), ws=P + 8) == B.ERR_ALIGN
    clip = lib.fp8mlp_clip_grads
    lst = grads((P, None, 16, B.F32))
    assert clip(lst[0], 1, B.NORM_L2, 1.0, P, P, None) == B.ERR_ARG
    lst = grads((P, P + 2, 16, B.F32))
    assert clip(lst[0], 1, B.NORM_L2, 1.0, P, P, None) == B.ERR_ALIGN
    adam = lib.fp8mlp_adam_step_scaled
    arr = (B._AdamTensor * 1)()
    assert adam(arr, None, 1, None, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1, None) == B.ERR_ARG
    assert adam(arr, None, 1, P + 2, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1, None) == B.ERR_ALIGN
    assert adam(None, None, 1, P, 1e-3, 0.9, 0.95, 1e-8, 0.0, 1, None) == B.ERR_ARG


def test_binding_refuses_what_it_cannot_pass_on():
    r = B.new_router(8, 2)
    x = torch.zeros((4, 8))
    with pytest.raises(ValueError, match="logits"):
        B.fp8mlp_route(r, x, None, torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2)))
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        B.new_grad_list([torch.zeros(4, dtype=torch.float64)])
    with pytest.raises(ValueError, match="as many outputs"):
        B.new_grad_list([], [torch.zeros(4)])


def test_workspace_constant_matches_the_header():
    from pathlib import Path
    header = (Path(__file__).resolve().parent.parent / "include" / "fp8mlp.h").read_text()
    for name, value in (("NORM_WORKSPACE_BYTES", B.NORM_WORKSPACE_BYTES), ("MAX_EXPERTS", B.MAX_EXPERTS), ("MAX_TOP_K", B.MAX_TOP_K)):
        assert f"#define FP8MLP_{name} {value}\n" in header
    assert C.sizeof(B.Router) == 32 and C.sizeof(B._GradTensor) == 32


# ---------------------------------------------------------------- the plain implementations themselves

@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_reference_gradient_against_differences(kind, renorm):
    rng = np.random.default_rng(1)
    E, k, h = 12, 3, 1e-6
    for _ in range(5):
        x, dw = rng.normal(0, 2, E), rng.normal(0, 1, k)
        experts, w, _ = R.route_row(x, None, k, kind, renorm=renorm, scale=1.7)
        assert np.allclose(w, R.weights_of(x, experts, kind, renorm, 1.7), rtol=1e-14)
        grad = R.route_backward_row(x, experts, dw, kind, renorm, 1.7)
        for e in range(E):
            up, down = x.copy(), x.copy()
            up[e] += h
            down[e] -= h
            diff = (R.weights_of(up, experts, kind, renorm, 1.7) - R.weights_of(down, experts, kind, renorm, 1.7)) @ dw / (2 * h)
            assert abs(diff - grad[e]) < 1e-8


def test_reference_choice_by_hand():
    x = np.array([0.0, 3.0, 1.0, 3.0, -np.inf, 2.0])
    e, w, _ = R.route_row(x, None, 3, "sigmoid", renorm=False)
    assert list(e) == [1, 3, 5] and np.allclose(w, 1 / (1 + np.exp(-x[[1, 3, 5]])))
    e, _, _ = R.route_row(x, None, 2, "sigmoid", groups=3, top_groups=1, group_top=2)
    assert list(e) == [3, 2]                           # the pairs sum to 1.45, 1.68 and 0.88 (its masked expert adds nothing)
    e, _, _ = R.route_row(x, None, 2, "sigmoid", groups=3, top_groups=1, group_top=1)
    assert list(e) == [1, 0]                           # best members 0.95, 0.95, 0.88: the first of the equal two
    e, w, _ = R.route_row(np.full(4, -np.inf), None, 2, "softmax")
    assert list(e) == [-1, -1] and not w.any()
    e, w, _ = R.route_row(x, np.array([9.0, 0, 0, 0, 9.0, 0]), 2, "softmax")
    assert list(e) == [0, 1] and abs(w.sum() - 1) < 1e-12


def test_reference_plan_by_hand():
    counts, offsets, rows = R.plan(np.array([[2, 0], [-1, 2], [0, 1]]), 3)
    assert list(counts) == [2, 1, 2] and list(offsets) == [0, 2, 3, 5]
    assert rows.tolist() == [[3, 0], [-1, 4], [1, 2]]


def test_combine_gradient_is_not_written_over_its_input(lib):
    """With one expert per token dye and dy have the same shape; a block would overwrite rows of dy that others still read."""
    back = lambda dy, dye, n=4: lib.fp8mlp_combine_backward(4, 1, 32, B.BF16, dy, 32, 2 * P, n, P, P, dye, P, None)
    assert back(P, P) == B.ERR_ARG
    assert back(3 * P, 3 * P) == B.ERR_ARG


class _Elsewhere:
    """Looks like a contiguous tensor on a GPU; its pointer is not valid and no refused call follows it."""

    def __init__(self, shape, dtype, device):
        self.shape, self.dtype, self._device = torch.Size(shape), dtype, device
        self.device, self.is_cuda = f"cuda:{device}", True

    def numel(self):
        return self.shape.numel()

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    def is_contiguous(self):
        return True

    def get_device(self):
        return self._device

    def data_ptr(self):
        return P


def test_binding_refuses_tensors_of_another_gpu(monkeypatch):
    """One argument after the other on GPU 1 while GPU 0 is current."""
    monkeypatch.setattr(B, "_device", lambda: 0)
    f32, i32, bf16, u8 = torch.float32, torch.int32, torch.bfloat16, torch.uint8
    r = B.new_router(8, 2)
    slots, weights, logits, rows = ((4, 2), i32), ((4, 2), f32), ((4, 8), f32), ((4, 32), bf16)
    wide = ((8, 32), bf16)
    calls = [
        (lambda x, b, e, w: B.fp8mlp_route(r, x, b, e, w), [logits, ((8,), f32), slots, weights]),
        (lambda x, e, w, d: B.fp8mlp_route_backward(r, x, e, w, d), [logits, slots, weights, logits]),
        (lambda c, b: B.fp8mlp_route_update_bias(c, 1e-3, b), [((8,), i32), ((8,), f32)]),
        (lambda e, c, o, p: B.fp8mlp_dispatch_plan(e, 8, c, o, p), [slots, ((8,), i32), ((9,), i32), slots]),
        (B.fp8mlp_dispatch, [rows, slots, wide]),
        (B.fp8mlp_combine, [wide, slots, weights, rows]),
        (B.fp8mlp_combine_backward, [rows, wide, slots, weights, wide, weights]),
        (lambda g, o: B.new_grad_list([g], [o]), [logits, logits]),
    ]
    for call, args in calls:
        for away in range(len(args)):
            with pytest.raises(ValueError, match="cuda:1"):
                call(*[_Elsewhere(shape, dtype, int(i == away)) for i, (shape, dtype) in enumerate(args)])
    # a list made while its GPU was current, and the small buffers of a call
    grads = B.new_grad_list([_Elsewhere((4, 8), f32, 0)])
    small = [((2,), f32), ((B.NORM_WORKSPACE_BYTES,), u8)]
    for call in (B.fp8mlp_grad_norm, B.fp8mlp_clip_grads):
        for away in range(2):
            with pytest.raises(ValueError, match="cuda:1"):
                call(grads, B.NORM_L2, 1.0, *[_Elsewhere(shape, dtype, int(i == away)) for i, (shape, dtype) in enumerate(small)])
        with monkeypatch.context() as m:
            m.setattr(B, "_device", lambda: 1)
            with pytest.raises(ValueError, match="gradients"):
                call(grads, B.NORM_L2, 1.0, *[_Elsewhere(shape, dtype, 1) for shape, dtype in small])


@pytest.mark.parametrize("bad", [((1,), torch.float64, 0), ((1,), torch.bfloat16, 0), ((2,), torch.float32, 0), ((1,), torch.float32, 1)],
                         ids=["f64", "bf16", "norm and coefficient", "another GPU"])
def test_adam_coefficient_is_one_fp32_element(monkeypatch, bad):
    """The kernel reads one float; of the pair that the norm call fills that would be the norm."""
    monkeypatch.setattr(B, "_device", lambda: 0)
    with pytest.raises(ValueError, match="grad_scale"):
        B.fp8mlp_adam_step_scaled([], None, _Elsewhere(*bad), 1e-3, 0.9, 0.95, 1e-8, 0.0, 1)
