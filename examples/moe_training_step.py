"""A mixture-of-experts layer trained with FP8 SwiGLU blocks as its experts.

Every expert is one block of this library (its own context, scales and FP8 weights).  A training step is

    logits = x Wr                      library product (fp32)
    route  -> experts, weights         fp8mlp_route
    plan, dispatch -> xe               fp8mlp_dispatch_plan, fp8mlp_dispatch
    ye[e]  = block_e(xe[e])            fp8mlp_forward on each expert's rows
    y      = combine(ye, weights)      fp8mlp_combine
    and back: fp8mlp_combine_backward, fp8mlp_backward, fp8mlp_combine without weights, fp8mlp_route_backward,
    then fp8mlp_grad_norm over the 3 E + 1 gradients, the Adam pass with the clip coefficient
    (fp8mlp_adam_step_scaled), and the router's balance bias (fp8mlp_route_update_bias).

The rows of an expert are a host number (the block's token count), so a forward waits for the plan's E + 1 offsets once.

    python examples/moe_training_step.py [--steps 20]
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

if __package__ in (None, ""):
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
from paper_2409_12517_b200 import binding as B


class MoeLayer:
    def __init__(self, d: int, f: int, n_experts: int, top_k: int, max_tokens: int, score: int = B.SCORE_SIGMOID,
                 n_groups: int = 1, top_groups: int = 1, w_std: float = 0.05, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *shape: w_std * torch.randn(shape, generator=gen, device="cuda")
        self.d, self.f, self.E, self.k = d, f, n_experts, top_k
        self.router = B.new_router(n_experts, top_k, score, n_groups, top_groups, min(2, n_experts // n_groups), renormalise=True)
        self.bias = torch.zeros(n_experts, device="cuda")
        self.contexts = []
        for _ in range(n_experts):
            self.contexts.append(B.fp8mlp_create(max_tokens, d, f, B.SMOOTH | B.SAVE_FOR_BWD))
        self.scales = [B.new_scales(f) for _ in range(n_experts)]
        self.amax = [B.new_amax(f) for _ in range(n_experts)]
        # the router, then W1, W2, W3 of every expert
        self.params = [randn(d, n_experts)]
        for _ in range(n_experts):
            self.params += [randn(d, f), randn(d, f), randn(f, d)]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.grad_list = B.new_grad_list(self.grads)
        self.norm_coef, self.workspace = torch.zeros(2, device="cuda"), B.new_norm_workspace()
        one, zero = (lambda: torch.ones(1, device="cuda")), (lambda: torch.zeros(1, device="cuda"))
        codes = lambda p: torch.zeros(p.numel(), dtype=torch.uint8, device="cuda")
        self.adam = [dict(w=p, g=g, m=codes(p), v=codes(p), scale_m_in=one(), scale_v_in=one(), scale_m_out=one(), scale_v_out=one(),
                          amax_m=zero(), amax_v=zero()) for p, g in zip(self.params, self.grads)]
        self.steps = 0

    def close(self):
        for ctx in self.contexts:
            B.fp8mlp_destroy(ctx)
        self.contexts = []

    def weights_of(self, e: int):
        return self.params[1 + 3 * e: 4 + 3 * e]

    def forward(self, x):
        """x: [T, d] bf16 -> y [T, d] bf16; keeps what backward needs."""
        T = x.shape[0]
        self.x = x
        self.logits = x.float() @ self.params[0]
        self.experts = torch.empty((T, self.k), dtype=torch.int32, device="cuda")
        self.weights = torch.empty((T, self.k), device="cuda")
        B.fp8mlp_route(self.router, self.logits, self.bias, self.experts, self.weights)
        self.counts = torch.empty(self.E, dtype=torch.int32, device="cuda")
        offsets = torch.empty(self.E + 1, dtype=torch.int32, device="cuda")
        self.rows = torch.empty((T, self.k), dtype=torch.int32, device="cuda")
        B.fp8mlp_dispatch_plan(self.experts, self.E, self.counts, offsets, self.rows)
        xe = torch.empty((T * self.k, self.d), dtype=torch.bfloat16, device="cuda")
        B.fp8mlp_dispatch(x, self.rows, xe)
        self.offsets = offsets.tolist()                  # waits for the plan; the copy of the rows goes on meanwhile
        self.ye = torch.empty_like(xe)
        for e, (begin, end) in enumerate(zip(self.offsets, self.offsets[1:])):
            if end > begin:
                B.fp8mlp_forward(self.contexts[e], end - begin, xe[begin:end], *self.weights_of(e), B.SCALE_FROM_CURRENT_AMAX,
                                 self.scales[e], self.amax[e], self.ye[begin:end])
        y = torch.empty_like(x)
        B.fp8mlp_combine(self.ye, self.rows, self.weights, y)
        return y

    def backward(self, dy):
        """dy: [T, d] bf16 -> dx [T, d] bf16; fills self.grads."""
        dye = torch.empty_like(self.ye)
        d_weights = torch.empty_like(self.weights)
        B.fp8mlp_combine_backward(dy, self.ye, self.rows, self.weights, dye, d_weights)
        dxe = torch.empty_like(dye)
        for e, (begin, end) in enumerate(zip(self.offsets, self.offsets[1:])):
            grads = self.grads[1 + 3 * e: 4 + 3 * e]
            if end > begin:
                B.fp8mlp_backward(self.contexts[e], end - begin, dye[begin:end], B.SCALE_FROM_CURRENT_AMAX, self.scales[e],
                                  self.amax[e], dxe[begin:end], *grads)
            else:
                for g in grads:                          # an expert that no token chose
                    g.zero_()
        dx = torch.empty_like(dy)
        B.fp8mlp_combine(dxe, self.rows, None, dx)
        d_logits = torch.empty_like(self.logits)
        B.fp8mlp_route_backward(self.router, self.logits, self.experts, d_weights, d_logits)
        torch.matmul(self.x.float().T, d_logits, out=self.grads[0])
        return (dx.float() + d_logits @ self.params[0].T).bfloat16()

    def choose_moment_scales(self, beta1: float, beta2: float):
        """The scales that this step writes its moments with: delayed, from the maxima of the last step, with room for moments
        that grow; a tensor without a gradient so far starts from a bound of this step's, for no element of the clipped
        gradients is larger than their norm.

        m gets more room than v.  E4M3 keeps values down to 2^-18.8 of its largest, E5M2 down to 2^-32.8, in terms of the
        gradient 2^-16.4; with these factors an element's v outlasts its m, where an m without its v would make a step of many
        times the learning rate."""
        bound = self.norm_coef[:1] * self.norm_coef[1:]
        for t in self.adam:
            top_m = torch.where(t["amax_m"] > 0, 16 * t["amax_m"], 8 * (1 - beta1) * bound)
            top_v = torch.where(t["amax_v"] > 0, 4 * t["amax_v"], (1 - beta2) * bound ** 2)
            B.fp8mlp_scale_from_amax(top_m, B.E4M3, t["scale_m_out"])
            B.fp8mlp_scale_from_amax(top_v, B.E5M2, t["scale_v_out"])

    def step(self, lr: float = 1e-3, max_norm: float = 1.0, bias_rate: float = 1e-3, beta1: float = 0.9, beta2: float = 0.95):
        """Clipped Adam step on all parameters, and the router's balance bias.  Returns (norm, coefficient), on the device."""
        self.steps += 1
        B.fp8mlp_grad_norm(self.grad_list, B.NORM_L2, max_norm, self.norm_coef, self.workspace)
        self.choose_moment_scales(beta1, beta2)
        for i in range(0, len(self.adam), 8):
            B.fp8mlp_adam_step_scaled(self.adam[i:i + 8], None, self.norm_coef[1:], lr, beta1, beta2, 1e-8, 0.0, self.steps)
        for t in self.adam:                              # what the codes were written with
            t["scale_m_in"].copy_(t["scale_m_out"])
            t["scale_v_in"].copy_(t["scale_v_out"])
        B.fp8mlp_route_update_bias(self.counts, bias_rate, self.bias)
        return self.norm_coef


def train(steps: int, tokens: int = 512, d: int = 256, f: int = 704, n_experts: int = 8, top_k: int = 2, lr: float = 1e-3,
          max_norm: float = 0.05, seed: int = 0, report=None):
    """Fits the layer to a fixed random map; returns the losses."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    layer = MoeLayer(d, f, n_experts, top_k, tokens * top_k, seed=seed)
    teacher = torch.randn((d, d), generator=gen, device="cuda") / d ** 0.5
    losses = []
    try:
        for step in range(steps):
            x = torch.randn((tokens, d), generator=gen, device="cuda").bfloat16()
            target = torch.tanh(x.float() @ teacher)
            y = layer.forward(x)
            diff = y.float() - target
            layer.backward((2.0 / diff.numel() * diff).bfloat16())
            norm, coef = layer.step(lr, max_norm).tolist()
            losses.append(float(diff.square().mean()))
            if report is not None:
                report(f"step {step:3d}  loss {losses[-1]:.4f}  gradient norm {norm:.4f}  clip {coef:.3f}  rows of the experts "
                       f"{layer.counts.tolist()}")
    finally:
        layer.close()
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=20)
    parser.add_argument("--tokens", type=int, default=512)
    args = parser.parse_args()
    train(args.steps, tokens=args.tokens, report=print)
