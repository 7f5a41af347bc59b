"""Workloads of the mixture-of-experts and gradient-clipping operators: routing, dispatch, combine, clip.

Every case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` makes one pass through an
operator - in elementary torch operations, or (own = True) through this package - and `exact` evaluates the definition in
64 bits.  Kinds of case, by `op`:
  route           logits -> chosen experts and their weights
  route_backward  gradients of the weights -> gradients of the logits
  dispatch        chosen experts -> counts, offsets, rows; token rows copied into expert order
  dispatch_backward  rows in expert order -> summed gradient of the token rows
  combine         expert outputs -> weighted sum for each token
  combine_backward   gradient of that sum -> gradients of the expert outputs and of the weights
  norm            global gradient norm and clip coefficient (the Adam pass applies the coefficient)
  clip            the same, and the scaled gradients
"""
import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases

def _router(T, E, k, score, bias=False, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0, dtype="f32"):
    return dict(T=T, E=E, k=k, score=score, bias=bias, groups=groups, top_groups=top_groups, group_top=group_top,
                renorm=renorm, scale=scale, dtype=dtype)


def listed():
    return [
        # one token of a served model: latency of the router alone
        dict(name="route_one_token", op="route",
             **_router(1, 256, 8, "sigmoid", True, 8, 4, 2, True, 2.5)),
        # a training batch of 16384 tokens over many small experts, limited to four of eight groups
        dict(name="route_16k_256_experts", op="route",
             **_router(16384, 256, 8, "sigmoid", True, 8, 4, 2, True, 2.5)),
        # softmax weights kept as they are (dense gradient), odd counts, bf16 logits as a bf16 product leaves them
        dict(name="route_backward_softmax_odd", op="route_backward",
             **_router(2047, 60, 4, "softmax", renorm=False, dtype="bf16")),
        # the backward pass of the training batch above
        dict(name="route_backward_16k", op="route_backward",
             **_router(16384, 256, 8, "sigmoid", True, 8, 4, 2, True, 2.5)),
        # a few tokens of a served model at the 7B width
        dict(name="dispatch_4_tokens", op="dispatch", T=4, d=4096, E=256, k=8, drop=0.0, dtype="bf16"),
        # a training batch at the 7B width, two of eight experts
        dict(name="dispatch_16k", op="dispatch", T=16384, d=4096, E=8, k=2, drop=0.0, dtype="bf16"),
        # its backward pass with more experts per token, and padding tokens that go nowhere
        dict(name="dispatch_backward_2k_padded", op="dispatch_backward", T=2048, d=4096, E=64, k=6, drop=0.1, dtype="bf16"),
        # ragged small batch at the small width
        dict(name="combine_odd", op="combine", T=509, d=512, E=60, k=4, drop=0.1, dtype="bf16"),
        # combine and its backward pass in training at the 7B width
        dict(name="combine_8k", op="combine", T=8192, d=4096, E=64, k=6, drop=0.0, dtype="bf16"),
        dict(name="combine_backward_8k", op="combine_backward", T=8192, d=4096, E=64, k=6, drop=0.0, dtype="bf16"),
        # gradients of 16 small experts (256 x 704), their router and some vectors of odd length, bf16
        dict(name="clip_16_experts_bf16", op="clip", d=256, f=704, E=16, extra=12, dtype="bf16", norm="l2"),
        # gradients of one 7B MLP block with a router, fp32 as the weight-gradient kernels leave them
        dict(name="clip_7b_block", op="clip", d=4096, f=11008, E=1, extra=7, dtype="f32", norm="l2"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random) -> dict:
    op = rng.choice(["route", "route", "route_backward", "route_backward", "dispatch", "dispatch", "dispatch_backward",
                     "combine", "combine", "combine_backward", "norm", "clip", "clip"])
    if op.startswith("route"):
        T, dtype = _log(rng, 1, 32768), rng.choice(["f32", "f32", "bf16"])
        groups = rng.choice([1, 1, 4, 8])
        if groups == 1:
            E = _log(rng, 4, 512)
            case = _router(T, E, min(E, rng.randint(1, 10)), rng.choice(["softmax", "sigmoid"]), rng.random() < 0.4)
        else:
            per = rng.randint(2, 32)
            top_groups = rng.randint(1, groups)
            case = _router(T, groups * per, min(top_groups * per, rng.randint(1, 10)), rng.choice(["softmax", "sigmoid"]),
                           rng.random() < 0.6, groups, top_groups, rng.choice([1, 2]))
        case.update(renorm=rng.random() < 0.6, scale=rng.choice([1.0, 1.0, 2.5]), dtype=dtype)
        return dict(op=op, **case)
    if op in ("norm", "clip"):
        d, f = rng.choice([(256, 704), (512, 1536), (512, 1536), (1024, _log(rng, 1024, 4096)), (4096, 11008)])
        E = 1 if d == 4096 else _log(rng, 1, 8 if d == 1024 else 64 if op == "norm" else 16)
        return dict(op=op, d=d, f=f, E=E, extra=rng.randint(0, 12), dtype=rng.choice(["f32", "f32", "bf16", "mixed"]),
                    norm="inf" if rng.random() < 0.2 else "l2")
    d = 16 * _log(rng, 8, 512)
    k = rng.randint(1, 8)
    T = _log(rng, 1, 100_000_000 // (d * (k + 1)) if op != "combine_backward" else 80_000_000 // (d * (k + 1)))
    return dict(op=op, T=T, d=d, E=max(k, _log(rng, 4, 256)), k=k, drop=rng.choice([0.0, 0.0, 0.1, 0.5]),
                dtype="f32" if rng.random() < 0.25 else "bf16")


def work(case: dict) -> dict:
    op = case["op"]
    if op.startswith("route"):
        T, E, k, b = case["T"], case["E"], case["k"], 4 if case["dtype"] == "f32" else 2
        if op == "route":
            return {"bytes": T * E * b + 8 * T * k + (4 * E if case["bias"] else 0), "flops": 10 * T * E}
        # the softmax gradient is dense where the weights are not renormalised; otherwise only the chosen logits count
        dense = case["score"] == "softmax" and not case["renorm"]
        return {"bytes": T * E * b + (T * E * b if dense else T * k * b) + 8 * T * k, "flops": 10 * T * (E if dense else k)}
    if op in ("norm", "clip"):
        n, total = 0, 0
        for shape, dt in _gradient_shapes(case):
            numel = math.prod(shape)
            n += numel
            total += numel * (4 if dt == "f32" else 2)
        return {"bytes": total * (2 if op == "clip" else 1) + 8, "flops": n * (3 if op == "clip" else 2)}
    T, d, k, b = case["T"], case["d"], case["k"], 4 if case["dtype"] == "f32" else 2
    n = int(T * (1.0 - case["drop"])) * k
    if op == "dispatch":
        return {"bytes": (T * d + n * d) * b + 8 * T * k + 8 * case["E"], "flops": T * k}
    if op == "dispatch_backward":
        return {"bytes": (T * d + n * d) * b + 4 * T * k, "flops": n * d}
    if op == "combine":
        return {"bytes": (T * d + n * d) * b + 8 * T * k, "flops": 2 * n * d}
    return {"bytes": (T * d + 2 * n * d) * b + 12 * T * k, "flops": 3 * n * d}


# ---------------------------------------------------------------- inputs

def _gradient_shapes(case):
    """W1, W2 [d, f] and W3 [f, d] of every expert, the router [d, E], and some odd small tensors (norm gains, biases)."""
    kinds = {"f32": ("f32", "f32"), "bf16": ("bf16", "bf16"), "mixed": ("bf16", "f32")}[case["dtype"]]
    d, f = case["d"], case["f"]
    shapes = []
    for _ in range(case["E"]):
        shapes += [((d, f), kinds[0]), ((d, f), kinds[0]), ((f, d), kinds[0])]
    shapes.append(((d, max(case["E"], 8)), kinds[1]))
    shapes += [((1 + 37 * i * i,), kinds[1]) for i in range(case["extra"])]
    return shapes


def _choice_values(case, x, bias):
    """Scores and the values that the selection compares, in the precision of x."""
    if case["score"] == "softmax":
        e = torch.exp(x - x.amax(-1, keepdim=True))
        s = e / e.sum(-1, keepdim=True)
    else:
        s = 1 / (1 + torch.exp(-x))
    return s, (s if bias is None else s + bias)


def _select(case, c):
    """The chosen experts in falling order of c, ties to the lowest index, within the best groups."""
    T, E = c.shape
    G = case["groups"]
    if G > 1:
        per = c.view(T, G, E // G)
        value = torch.sort(per, dim=-1, descending=True, stable=True).values[..., :min(case["group_top"], E // G)].sum(-1)
        best = torch.sort(value, dim=-1, descending=True, stable=True).indices[:, :case["top_groups"]]
        keep = torch.zeros((T, G), dtype=torch.bool, device=c.device)
        keep[torch.arange(T, device=c.device)[:, None], best] = True
        c = torch.where(keep[:, :, None], per, torch.full_like(per, -math.inf)).view(T, E)
    return torch.sort(c, dim=-1, descending=True, stable=True).indices[:, :case["k"]]


def _close_calls(case, x, bias):
    """Rows whose selection (in 64 bits) is decided by less than 1e-5 of the value: equal logits aside, which every
    precision ties alike, a rounding could decide these, and then neither result is the wrong one."""
    _, c = _choice_values(case, x.double(), None if bias is None else bias.double())
    T, E = c.shape
    G = case["groups"]
    slack = 1e-6 if case["bias"] else 0.0       # a bias can cancel a score: its rounding stays

    def near(v, n):
        top = torch.sort(v, dim=-1, descending=True).values[:, :n + 1]
        gap, size = top[:, :-1] - top[:, 1:], top[:, :-1].abs()
        return ((gap <= 1e-5 * size + slack) & (gap > 1e-14 * size)).any(-1)

    close = torch.zeros(T, dtype=torch.bool, device=x.device)
    kept = c
    if G > 1:
        per = c.view(T, G, E // G)
        value = torch.sort(per, dim=-1, descending=True).values[..., :min(case["group_top"], E // G)].sum(-1)
        close |= near(value, case["top_groups"]) if case["top_groups"] < G else close
        best = torch.sort(value, dim=-1, descending=True, stable=True).indices[:, :case["top_groups"]]
        keep = torch.zeros((T, G), dtype=torch.bool, device=c.device)
        keep[torch.arange(T, device=c.device)[:, None], best] = True
        kept = torch.where(keep[:, :, None], per, torch.full_like(per, -1e30)).view(T, E)
    return close | near(kept, min(case["k"], E - 1))


def _logits(case, gen):
    """Router logits: a spread of a few units, with some experts favoured over the whole batch."""
    T, E, dt = case["T"], case["E"], _DTYPES[case["dtype"]]
    favour = 0.5 * torch.randn(E, generator=gen, device="cuda")
    bias = 0.05 * torch.randn(E, generator=gen, device="cuda") if case["bias"] else None
    make = lambda n: (1.2 * torch.randn((n, E), generator=gen, device="cuda") + favour).to(dt)
    x = make(T)
    for _ in range(12):
        redo = torch.nonzero(_close_calls(case, x, bias)).flatten()
        if redo.numel() == 0:
            break
        x[redo] = make(redo.numel())
    return x, bias


def _random_experts(case, gen):
    """k different experts for each token, uneven in their load; dropped (padding) tokens have none (-1)."""
    T, E, k = case["T"], case["E"], case["k"]
    noise = torch.randn((T, E), generator=gen, device="cuda") + 0.7 * torch.randn(E, generator=gen, device="cuda")
    experts = torch.topk(noise, k, dim=-1).indices.to(torch.int32)
    n_drop = T - int(T * (1.0 - case["drop"]))
    if n_drop:
        experts[torch.randperm(T, generator=gen, device="cuda")[:n_drop]] = -1
    return experts.contiguous()


def _rows_of(experts, E):
    """(counts, offsets, rows, order) by stable sorting: rows in order of expert, then token, then slot; order is the slot
    of each row, unused slots last."""
    flat = experts.reshape(-1)
    key, order = torch.sort(torch.where(flat >= 0, flat, torch.full_like(flat, E)), stable=True)
    offsets = torch.searchsorted(key, torch.arange(E + 1, device=flat.device, dtype=key.dtype)).to(torch.int32)
    rows = torch.empty_like(flat)
    rows[order] = torch.arange(flat.numel(), device=flat.device, dtype=torch.int32)
    rows = torch.where(flat >= 0, rows, torch.full_like(rows, -1))
    return offsets[1:] - offsets[:-1], offsets, rows.view(experts.shape), order


def prepare(case: dict, seed: int) -> dict:
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    st = {"case": case}
    if op.startswith("route"):
        T, k = case["T"], case["k"]
        st["logits"], st["bias"] = _logits(case, gen)
        st["experts"] = torch.empty((T, k), dtype=torch.int32, device="cuda")
        st["weights"] = torch.empty((T, k), dtype=torch.float32, device="cuda")
        if op == "route_backward":
            _, c = _choice_values(case, st["logits"].float(), st["bias"])
            st["experts"] = _select(case, c).to(torch.int32).contiguous()
            st["d_weights"] = 1e-3 * torch.randn((T, k), generator=gen, device="cuda")
            st["d_logits"] = torch.empty_like(st["logits"])
    elif op in ("norm", "clip"):
        st["grads"] = []
        for shape, dt in _gradient_shapes(case):
            spread = 1e-3 * math.exp(torch.randn(1, generator=gen, device="cuda").item())
            st["grads"].append((spread * torch.randn(shape, generator=gen, device="cuda")).to(_DTYPES[dt]))
        st["outs"] = [torch.empty_like(g) for g in st["grads"]] if op == "clip" else None
        biggest = max(float(g.float().abs().max()) for g in st["grads"])
        st["max_norm"] = 1.0 if case["norm"] == "l2" else 0.5 * biggest
        st["norm_coef"] = torch.empty(2, dtype=torch.float32, device="cuda")
    else:
        T, d, E, k, dt = case["T"], case["d"], case["E"], case["k"], _DTYPES[case["dtype"]]
        st["experts"] = _random_experts(case, gen)
        randn = lambda n, scale=1.0: (scale * torch.randn((n, d), generator=gen, device="cuda")).to(dt)
        if op == "dispatch":
            st["x"] = randn(T)
            st["counts"] = torch.empty(E, dtype=torch.int32, device="cuda")
            st["offsets"] = torch.empty(E + 1, dtype=torch.int32, device="cuda")
            st["rows"] = torch.empty((T, k), dtype=torch.int32, device="cuda")
            st["xe"] = torch.zeros((T * k, d), dtype=dt, device="cuda")
        else:
            st["rows"] = _rows_of(st["experts"], E)[2].contiguous()
            w = torch.rand((T, k), generator=gen, device="cuda") + 0.05
            st["weights"] = w / w.sum(-1, keepdim=True)
            st["ye"] = randn(T * k)
            if op == "combine_backward":
                st["dy"] = randn(T, 1e-3)
                st["dye"] = torch.zeros((T * k, d), dtype=dt, device="cuda")
                st["d_weights"] = torch.empty((T, k), dtype=torch.float32, device="cuda")
            else:
                st["y"] = torch.empty((T, d), dtype=dt, device="cuda")
    if own:
        from paper_2409_12517_b200 import binding as B
        if op.startswith("route"):
            st["router"] = B.new_router(case["E"], case["k"], score=B.SCORE_SOFTMAX if case["score"] == "softmax" else B.SCORE_SIGMOID,
                                        n_groups=case["groups"], top_groups=case["top_groups"], group_top=case["group_top"],
                                        renormalise=case["renorm"], scale=case["scale"])
        elif op in ("norm", "clip"):
            st["list"] = B.new_grad_list(st["grads"], st["outs"])
            st["workspace"] = B.new_norm_workspace()
    return st


# ---------------------------------------------------------------- one pass

def run(state: dict):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    from paper_2409_12517_b200 import binding as B
    case, op = st["case"], st["case"]["op"]
    if op == "route":
        B.fp8mlp_route(st["router"], st["logits"], st["bias"], st["experts"], st["weights"])
        return st["experts"], st["weights"]
    if op == "route_backward":
        B.fp8mlp_route_backward(st["router"], st["logits"], st["experts"], st["d_weights"], st["d_logits"])
        return st["d_logits"]
    if op == "dispatch":
        B.fp8mlp_dispatch_plan(st["experts"], case["E"], st["counts"], st["offsets"], st["rows"])
        B.fp8mlp_dispatch(st["x"], st["rows"], st["xe"])
        return st["counts"], st["offsets"], st["rows"], st["xe"]
    if op == "dispatch_backward":
        B.fp8mlp_combine(st["ye"], st["rows"], None, st["y"])
        return st["y"]
    if op == "combine":
        B.fp8mlp_combine(st["ye"], st["rows"], st["weights"], st["y"])
        return st["y"]
    if op == "combine_backward":
        B.fp8mlp_combine_backward(st["dy"], st["ye"], st["rows"], st["weights"], st["dye"], st["d_weights"])
        return st["dye"], st["d_weights"]
    kind = B.NORM_L2 if case["norm"] == "l2" else B.NORM_INF
    if op == "norm":
        B.fp8mlp_grad_norm(st["list"], kind, st["max_norm"], st["norm_coef"], st["workspace"])
        return st["norm_coef"]
    B.fp8mlp_clip_grads(st["list"], kind, st["max_norm"], st["norm_coef"], st["workspace"])
    return [st["norm_coef"], *st["outs"]]


def _run_plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "route":
        s, c = _choice_values(case, st["logits"].float(), st["bias"])
        experts = _select(case, c)
        w = torch.gather(s, 1, experts)
        if case["renorm"]:
            w = w / w.sum(-1, keepdim=True)
        return experts.to(torch.int32), w * case["scale"]
    if op == "route_backward":
        x = st["logits"].float()
        s, _ = _choice_values(case, x, None)
        experts, dw = st["experts"].long(), st["d_weights"] * case["scale"]
        chosen = torch.gather(s, 1, experts)
        if case["renorm"]:
            total = chosen.sum(-1, keepdim=True)
            dw = (dw - (dw * chosen).sum(-1, keepdim=True) / total) / total
        ds = torch.zeros_like(s)
        ds[torch.arange(case["T"], device=s.device)[:, None], experts] = dw
        if case["score"] == "softmax":
            dx = s * (ds - (ds * s).sum(-1, keepdim=True))
        else:
            dx = ds * s * (1 - s)
        return dx.to(st["logits"].dtype)
    if op == "dispatch":
        counts, offsets, rows, order = _rows_of(st["experts"], case["E"])
        filled = torch.arange(order.numel(), device=order.device) < offsets[-1]
        xe = torch.where(filled[:, None], st["x"][order // case["k"]], torch.zeros((), dtype=st["x"].dtype, device="cuda"))
        return counts, offsets, rows, xe
    if op == "combine_backward":
        dy, rows = st["dy"].float(), st["rows"].long()
        n = st["ye"].shape[0]
        dye = torch.zeros((n + 1, case["d"]), dtype=st["ye"].dtype, device="cuda")     # the last row takes the unused slots
        dw = torch.zeros_like(st["weights"])
        for j in range(case["k"]):
            r, used = rows[:, j], rows[:, j] >= 0
            dye[torch.where(used, r, torch.full_like(r, n))] = (st["weights"][:, j:j + 1] * dy).to(dye.dtype)
            dot = (dy * st["ye"][r.clamp(min=0)].float()).sum(-1)
            dw[:, j] = torch.where(used, dot, torch.zeros_like(dot))
        return dye[:n], dw
    if op in ("combine", "dispatch_backward"):
        rows = st["rows"].long()
        y = torch.zeros((case["T"], case["d"]), dtype=torch.float32, device="cuda")
        for j in range(case["k"]):
            part = st["ye"][rows[:, j].clamp(min=0)].float()
            w = (rows[:, j:j + 1] >= 0).float()
            y += part * (w * st["weights"][:, j:j + 1] if op == "combine" else w)
        return y.to(st["ye"].dtype)
    if case["norm"] == "l2":
        norm = torch.sqrt(torch.stack([(g.float() * g.float()).sum() for g in st["grads"]]).sum())
    else:
        norm = torch.stack([g.float().abs().max() for g in st["grads"]]).max()
    coef = torch.clamp(st["max_norm"] / (norm + 1e-6), max=1.0)
    both = torch.stack([norm, coef])
    if op == "norm":
        return both
    return [both, *[(g.float() * coef).to(g.dtype) for g in st["grads"]]]


# ---------------------------------------------------------------- the definitions in 64 bits

def _first_largest(c, n):
    """Indices of the n largest of each row, one after the other, the lowest index among equals."""
    at = torch.arange(c.shape[1], device=c.device)
    left, found = c.clone(), []
    for _ in range(n):
        best = torch.where(left == left.amax(-1, keepdim=True), at, c.shape[1]).amin(-1, keepdim=True)
        found.append(best)
        left.scatter_(1, best, -math.inf)
    return torch.cat(found, dim=1)


def exact(case: dict, seed: int):
    st = prepare(case, seed)
    op = case["op"]
    f64 = torch.float64
    if op.startswith("route"):
        x = st["logits"].to(f64)
        if case["score"] == "softmax":
            s = torch.exp(x - torch.logsumexp(x, -1, keepdim=True))
        else:
            s = torch.sigmoid(x)
        if op == "route":
            c = s if st["bias"] is None else s + st["bias"].to(f64)
            G, per = case["groups"], case["E"] // case["groups"]
            if G > 1:
                grouped = c.view(case["T"], G, per)
                best = grouped.amax(-1)
                if case["group_top"] == 2 and per > 1:
                    best = best + torch.kthvalue(grouped, per - 1, dim=-1).values
                keep = _first_largest(best, case["top_groups"])
                c = c.masked_fill(torch.ones((case["T"], G), dtype=torch.bool, device="cuda").scatter_(1, keep, False)
                                  .repeat_interleave(per, dim=1), -math.inf)
            idx = _first_largest(c, case["k"])
            w = torch.gather(s, 1, idx)
            if case["renorm"]:
                w = w / w.sum(-1, keepdim=True)
            return idx.to(torch.int32), case["scale"] * w
        idx, dw = st["experts"].long(), st["d_weights"].to(f64) * case["scale"]
        p = torch.gather(s, 1, idx)
        if case["renorm"]:
            r = p / p.sum(-1, keepdim=True)
            at = r * (dw - (dw * r).sum(-1, keepdim=True))          # s_j times the gradient of s_j
            at = at if case["score"] == "softmax" else at * torch.gather(torch.sigmoid(-x), 1, idx)
            return torch.zeros_like(s).scatter_(1, idx, at)
        if case["score"] == "sigmoid":
            return torch.zeros_like(s).scatter_(1, idx, dw * p * torch.gather(torch.sigmoid(-x), 1, idx))
        return torch.zeros_like(s).scatter_(1, idx, dw * p) - s * (dw * p).sum(-1, keepdim=True)
    if op in ("norm", "clip"):
        if case["norm"] == "l2":
            norm = math.sqrt(sum(float(g.to(f64).square().sum()) for g in st["grads"]))
        else:
            norm = max(float(g.to(f64).abs().max()) for g in st["grads"])
        coef = min(1.0, st["max_norm"] / (norm + 1e-6))
        both = torch.tensor([norm, coef], dtype=f64, device="cuda")
        return both if op == "norm" else [both, *[g.to(f64) * coef for g in st["grads"]]]
    T, k, d = case["T"], case["k"], case["d"]
    if op == "dispatch":
        slot = torch.arange(T * k, device="cuda")
        expert = st["experts"].flatten().long()
        slot = slot[expert >= 0]
        slot = slot[torch.argsort(expert[slot] * (T * k) + slot)]
        xe = torch.zeros((T * k, d), dtype=f64, device="cuda")
        xe[:slot.numel()] = st["x"].to(f64)[slot // k]
        return None, None, None, xe         # the others are whole numbers
    rows = st["rows"].long()
    used = rows >= 0
    if op == "combine_backward":
        dye = torch.zeros((T * k, d), dtype=f64, device="cuda")
        dw = torch.zeros((T, k), dtype=f64, device="cuda")
        for t0 in range(0, T, 2048):                                # in blocks of tokens: the products are large in 64 bits
            m, r = used[t0:t0 + 2048], rows[t0:t0 + 2048]
            dy = st["dy"][t0:t0 + 2048].to(f64)
            per_slot = dy[:, None, :].expand(-1, k, -1)
            dye[r[m]] = per_slot[m] * st["weights"][t0:t0 + 2048][m].to(f64)[:, None]
            dw[t0:t0 + 2048][m] = (per_slot[m] * st["ye"][r[m]].to(f64)).sum(-1)
        return dye, dw
    y = torch.zeros((T, d), dtype=f64, device="cuda")
    w = st["weights"].to(f64) if op == "combine" else torch.ones((T, k), dtype=f64, device="cuda")
    for t0 in range(0, T, 2048):
        m, r = used[t0:t0 + 2048], rows[t0:t0 + 2048].clamp(min=0)
        y[t0:t0 + 2048] = torch.einsum("tk,tkd->td", w[t0:t0 + 2048] * m, st["ye"][r].to(f64))
    return y
