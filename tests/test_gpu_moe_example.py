"""The mixture-of-experts example: one layer's outputs and gradients against the unquantised layer in 64 bits, and a short
training run.  The experts' products are FP8 (E4M3 forward, E5M2 backward: relative steps of 2^-4 and 2^-3, errors that
average over a contraction), so outputs are held to 10 % of their norm and gradients to 20 % and a cosine above 0.97; routing
and clipping themselves are held to tight bounds in their own tests."""
import pytest
import torch

from examples.moe_training_step import MoeLayer, train
from paper_2409_12517_b200 import binding as B

pytestmark = pytest.mark.gpu


def _reference(layer, x, dy):
    """(y, dx, gradients) of the unquantised layer for the experts that were chosen, by automatic differentiation in fp64."""
    x = x.double().requires_grad_()
    params = [p.detach().double().clone().requires_grad_() for p in layer.params]
    chosen = layer.experts.long()
    s = torch.gather(torch.sigmoid(x @ params[0]), 1, chosen)
    w = s / s.sum(-1, keepdim=True)
    y = torch.zeros_like(x)
    for e in range(layer.E):
        W1, W2, W3 = params[1 + 3 * e: 4 + 3 * e]
        gate = x @ W2
        out = (gate * torch.sigmoid(gate) * (x @ W1)) @ W3
        y = y + out * (w * (chosen == e)).sum(-1, keepdim=True)
    y.backward(dy.double())
    return y.detach(), x.grad, [p.grad for p in params]


@pytest.mark.parametrize("E,k,groups", [(8, 2, 1), (16, 3, 4)])
def test_layer_against_the_unquantised_one(E, k, groups):
    T, d, f = 300, 128, 208
    gen = torch.Generator(device="cuda").manual_seed(3)
    layer = MoeLayer(d, f, E, k, T * k, n_groups=groups, top_groups=max(1, groups // 2), w_std=0.2, seed=1)
    try:
        x = torch.randn((T, d), generator=gen, device="cuda").bfloat16()
        dy = torch.randn((T, d), generator=gen, device="cuda").bfloat16()
        y = layer.forward(x)
        dx = layer.backward(dy)
        assert int(layer.counts.sum()) == T * k and layer.offsets[-1] == T * k
        ref_y, ref_dx, ref_grads = _reference(layer, x, dy)
        rel = lambda a, b: float((a.double() - b).norm() / b.norm())
        cos = lambda a, b: float((a.double() * b).sum() / (a.double().norm() * b.norm()))
        assert rel(y, ref_y) < 0.1
        assert rel(dx, ref_dx) < 0.2 and cos(dx, ref_dx) > 0.97
        for i, (g, r) in enumerate(zip(layer.grads, ref_grads)):
            if float(r.norm()) > 0:
                assert rel(g, r) < 0.2 and cos(g, r) > 0.97, f"parameter {i}"
        before = [p.clone() for p in layer.params]
        norm, coef = layer.step(max_norm=1.0).tolist()
        exact = float(torch.sqrt(sum((g.double() ** 2).sum() for g in layer.grads)))
        assert abs(norm - exact) <= 1e-6 * exact and abs(coef - min(1.0, 1.0 / (exact + 1e-6))) <= 1e-6
        assert all(not torch.equal(a, b) for a, b, g in zip(before, layer.params, layer.grads) if bool(g.any()))
        assert B.fp8mlp_status(layer.contexts[0]) == B.OK
    finally:
        layer.close()


def test_an_expert_that_no_token_chose():
    T, d, f, E = 40, 64, 96, 4
    layer = MoeLayer(d, f, E, 2, T * 2, seed=2)
    try:
        layer.bias[3] = -float("inf")                    # out of service
        x = torch.randn((T, d), device="cuda").bfloat16()
        layer.grads[1 + 9].fill_(5.0)
        y = layer.forward(x)
        layer.backward(torch.ones_like(y))
        assert int(layer.counts[3]) == 0 and not layer.grads[1 + 9].any()
        assert torch.isfinite(y).all()
    finally:
        layer.close()


def test_training_follows_the_unquantised_layer():
    """30 clipped steps beside the same steps of the unquantised layer in fp64 (its own parameters, plain Adam with exact
    moments, the FP8 layer's choice of experts): losses within 10 % of each other all the way, and both falling."""
    T, d, f, E, k, lr, max_norm = 256, 64, 96, 4, 2, 3e-3, 0.05
    gen = torch.Generator(device="cuda").manual_seed(7)
    layer = MoeLayer(d, f, E, k, T * k, seed=5)
    teacher = torch.randn((d, d), generator=gen, device="cuda") / d ** 0.5
    shadow = MoeLayer.__new__(MoeLayer)                  # parameters only
    shadow.E, shadow.params = E, [p.double() for p in layer.params]
    m, v = [torch.zeros_like(p) for p in shadow.params], [torch.zeros_like(p) for p in shadow.params]
    losses = []
    try:
        for step in range(1, 31):
            x = torch.randn((T, d), generator=gen, device="cuda").bfloat16()
            target = torch.tanh(x.float() @ teacher)
            y = layer.forward(x)
            diff = y.float() - target
            shadow.experts = layer.experts
            ref_y, _, _ = _reference(shadow, x, torch.zeros_like(y))
            ref_diff = ref_y - target.double()
            _, _, grads = _reference(shadow, x, 2.0 / ref_diff.numel() * ref_diff)
            layer.backward((2.0 / diff.numel() * diff).bfloat16())
            layer.step(lr, max_norm)
            norm = torch.sqrt(sum((g ** 2).sum() for g in grads))
            coef = torch.clamp(max_norm / (norm + 1e-6), max=1.0)
            for p, g, a, b in zip(shadow.params, grads, m, v):
                a.mul_(0.9).add_(g * coef, alpha=0.1)
                b.mul_(0.95).add_((g * coef) ** 2, alpha=0.05)
                p -= lr * (a / (1 - 0.9 ** step)) / (torch.sqrt(b / (1 - 0.95 ** step)) + 1e-8)
            losses.append((float(diff.square().mean()), float(ref_diff.square().mean())))
    finally:
        layer.close()
    for got, ref in losses:
        assert abs(got - ref) <= 0.1 * ref, losses
    for side in (0, 1):
        assert sum(l[side] for l in losses[-5:]) < sum(l[side] for l in losses[:5]), losses


def test_the_example_runs():
    losses = train(3, tokens=64, d=64, f=96, n_experts=4)
    assert len(losses) == 3 and all(0.0 < l < 10.0 for l in losses)


def test_the_chain_in_a_cuda_graph():
    """Routing, plan, dispatch, combine, their gradients and clipping captured once and replayed on new inputs: the same bits as
    the calls themselves."""
    T, E, k, d = 700, 64, 6, 256
    gen = torch.Generator(device="cuda").manual_seed(11)
    router = B.new_router(E, k, B.SCORE_SIGMOID, 8, 4, 2, True, 2.5)
    new = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device="cuda")
    logits, bias, x, dy = new(T, E), new(E), new(T, d, dtype=torch.bfloat16), new(T, d, dtype=torch.bfloat16)
    out = dict(experts=new(T, k, dtype=torch.int32), weights=new(T, k), counts=new(E, dtype=torch.int32),
               offsets=new(E + 1, dtype=torch.int32), rows=new(T, k, dtype=torch.int32), xe=new(T * k, d, dtype=torch.bfloat16),
               y=new(T, d, dtype=torch.bfloat16), dye=new(T * k, d, dtype=torch.bfloat16), dw=new(T, k), dx=new(T, d, dtype=torch.bfloat16),
               dlogits=new(T, E), norm_coef=new(2), clipped=new(T, E))
    lst, ws = B.new_grad_list([out["dlogits"]], [out["clipped"]]), B.new_norm_workspace()

    def chain():
        B.fp8mlp_route(router, logits, bias, out["experts"], out["weights"])
        B.fp8mlp_dispatch_plan(out["experts"], E, out["counts"], out["offsets"], out["rows"])
        B.fp8mlp_dispatch(x, out["rows"], out["xe"])
        B.fp8mlp_combine(out["xe"], out["rows"], out["weights"], out["y"])
        B.fp8mlp_combine_backward(dy, out["xe"], out["rows"], out["weights"], out["dye"], out["dw"])
        B.fp8mlp_combine(out["dye"], out["rows"], None, out["dx"])
        B.fp8mlp_route_backward(router, logits, out["experts"], out["dw"], out["dlogits"])
        B.fp8mlp_clip_grads(lst, B.NORM_L2, 0.5, out["norm_coef"], ws)

    def inputs():
        for t in (logits, x, dy):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        bias.copy_(0.05 * torch.randn(E, generator=gen, device="cuda"))

    inputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        chain()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            chain()
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        inputs()
        chain()
        want = {n: t.clone() for n, t in out.items()}
        for t in out.values():
            t.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        for n, t in out.items():
            assert torch.equal(t, want[n]), n
        # y = sum of the weights times x, up to the rounding of y
        total = want["weights"].sum(-1, keepdim=True) * x.float()
        assert torch.allclose(want["y"].float(), total, rtol=2.0 ** -7, atol=1e-6)


def _decode(codes, dtype, scale):
    return codes.view(dtype).double() / scale.double()


@pytest.mark.parametrize("max_norm", [0.05, 1e3], ids=["clipped", "not clipped"])
def test_moments_of_the_first_steps(max_norm):
    """The FP8 moments against exact ones of the same gradients from the first step on, an expert that joins in the third step
    included.  Per element, a code adds half a step: 2^-4 of an E4M3 value, 2^-3 of an E5M2 value, or half the smallest step
    (2^-10, 2^-17) over the scale; what the last step was off by is carried on with beta.  Parameters: a step moves them by at most
    about lr, from either moments, as long as no v is lost beside its m; three steps are held to 3 lr."""
    T, d, f, E, k, lr, beta1, beta2 = 256, 64, 96, 4, 2, 1e-3, 0.9, 0.95
    gen = torch.Generator(device="cuda").manual_seed(13)
    layer = MoeLayer(d, f, E, k, T * k, seed=6)
    try:
        layer.bias[3] = -float("inf")
        w = [p.double() for p in layer.params]
        exact = [[torch.zeros_like(p) for p in w] for _ in range(2)]
        off = [[torch.zeros_like(p) for p in w] for _ in range(2)]
        for step in range(1, 4):
            if step == 3:
                layer.bias[3] = 1.0
            x = torch.randn((T, d), generator=gen, device="cuda").bfloat16()
            layer.forward(x)
            layer.backward((torch.randn((T, d), generator=gen, device="cuda") / T).bfloat16())
            grads = [g.double() for g in layer.grads]
            _, coef = layer.step(lr, max_norm, bias_rate=0.0).tolist()
            assert (coef < 1.0) == (max_norm < 1.0)
            for i, (t, g) in enumerate(zip(layer.adam, grads)):
                shape = g.shape
                if step < 3 and i >= 1 + 9:
                    assert not g.any() and not t["m"].any() and not t["v"].any()
                for j, (beta, value, code, half, least, dtype) in enumerate((
                        (beta1, coef * g, "m", 2.0 ** -4, 2.0 ** -10, torch.float8_e4m3fn),
                        (beta2, (coef * g) ** 2, "v", 2.0 ** -3, 2.0 ** -17, torch.float8_e5m2))):
                    exact[j][i] = beta * exact[j][i] + (1 - beta) * value
                    scale = t[f"scale_{code}_in"]
                    got = _decode(t[code], dtype, scale).view(shape)
                    carried = beta * off[j][i]
                    allowed = carried + half * (exact[j][i].abs() + carried) + least / scale.double() + 1e-5 * exact[j][i].abs()
                    assert bool(((got - exact[j][i]).abs() <= allowed).all()), f"{code} of parameter {i}, step {step}"
                    off[j][i] = allowed
                assert not bool(((t["m"] & 0x7f) != 0)[t["v"] == 0].any()), "an m without its v"
                if g.any():
                    # the codes carry the moments, not a few of their largest elements
                    assert float((_decode(t["m"], torch.float8_e4m3fn, t["scale_m_in"]).view(shape) - exact[0][i]).norm()) < \
                        0.1 * float(exact[0][i].norm()), f"m of parameter {i}, step {step}"
                upd = (exact[0][i] / (1 - beta1 ** step)) / (torch.sqrt(exact[1][i] / (1 - beta2 ** step)) + 1e-8)
                w[i] = w[i] - lr * upd
                assert float((layer.params[i].double() - w[i]).abs().max()) <= 3 * lr, f"parameter {i}, step {step}"
    finally:
        layer.close()
