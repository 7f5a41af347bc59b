"""Plain implementations, in 64 bits and by loops, of expert routing, dispatch, combine and gradient clipping: what the
kernels' tests compare with.  Written from the formulas in include/fp8mlp.h; nothing here is shared with the kernels."""
import numpy as np


def scores(x, kind):
    """x: [E] float64 -> s.  kind: "softmax" or "sigmoid"."""
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        if kind == "softmax":
            e = np.exp(x - x.max()) if not np.isnan(x).any() else np.full_like(x, np.nan)
            s = e / e.sum()
        else:
            s = np.where(x >= 0, 1 / (1 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1 + np.exp(-np.abs(x))))
        # scores are fp32 values: below its normal range they keep few digits, and then none
        return np.where(s < 2.0 ** -126, s.astype(np.float32).astype(np.float64), s)


def route_row(x, bias, k, kind, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0):
    """One token: (experts [k], weights [k], margin).  margin: the smallest relative distance, among the comparisons that
    decided something, between two values that are not equal (a rounding can turn what is closer than its error)."""
    x = np.asarray(x, np.float64)
    E = x.size
    s = scores(x, kind)
    c = s if bias is None else s + np.asarray(bias, np.float64)
    free = ~np.isneginf(x) & ~np.isnan(c) & ~np.isneginf(c)
    margin = np.inf

    def near(a, b):
        return np.inf if a == b or np.isinf(a) or np.isinf(b) else abs(a - b) / max(abs(a), abs(b), 1e-3 if bias is not None else 0.0)

    if groups > 1:
        per = E // groups
        value = np.full(groups, -np.inf)
        for g in range(groups):
            members = sorted((c[e] for e in range(g * per, (g + 1) * per) if free[e]), reverse=True)
            if members:
                value[g] = sum(members[:group_top])
        order = sorted(range(groups), key=lambda g: (-value[g], g))
        for a in order[:top_groups]:                   # every kept group with every other: equal ones may hide a near one
            margin = min([margin] + [near(value[a], value[b]) for b in order[top_groups:]])
        for g in order[top_groups:]:
            free[g * per:(g + 1) * per] = False
    order = sorted((e for e in range(E) if free[e]), key=lambda e: (-c[e], e))
    for i, a in enumerate(order[:k]):
        margin = min([margin] + [near(c[a], c[b]) for b in order[i + 1:]])
    experts = (order + [-1] * k)[:k]
    chosen = np.array([s[e] if e >= 0 else 0.0 for e in experts])
    total = chosen.sum()
    w = chosen if not renorm else (chosen / total if total != 0 else np.zeros(k))
    return np.array(experts, np.int32), scale * w, margin


def weights_of(x, experts, kind, renorm, scale):
    """The weights as a function of the logits for a fixed choice (what the gradient differentiates)."""
    s = scores(x, kind)
    chosen = np.array([s[e] if 0 <= e < len(x) else 0.0 for e in experts])
    if renorm:
        chosen = chosen / chosen.sum() if chosen.sum() != 0 else np.zeros_like(chosen)
    return scale * chosen


def route_backward_row(x, experts, dw, kind, renorm, scale):
    """Gradient of sum_j dw_j w_j with respect to x, by the quotient rule on w and the Jacobian of the scores."""
    x = np.asarray(x, np.float64)
    E = x.size
    s = scores(x, kind)
    used = [j for j, e in enumerate(experts) if 0 <= e < E]
    ds = np.zeros(E)
    if not used:
        return ds
    idx = np.array([experts[j] for j in used])
    d = scale * np.asarray(dw, np.float64)[used]
    if renorm:
        total = s[idx].sum()
        d = np.zeros_like(d) if total == 0 else d / total - (d * s[idx]).sum() / total ** 2
    ds[idx] = d
    if kind == "softmax":
        return s * (ds - (ds * s).sum())
    return ds * s * (1 - s)


def plan(experts, E):
    """(counts, offsets, rows) from the definition: rows in order of expert, then of slot."""
    flat = np.asarray(experts).reshape(-1)
    counts = np.array([(flat == e).sum() for e in range(E)], np.int32)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows = np.full(flat.size, -1, np.int32)
    for e in range(E):
        at = np.nonzero(flat == e)[0]
        rows[at] = offsets[e] + np.arange(at.size)
    return counts, offsets, rows.reshape(np.shape(experts))


def combine(ye, rows, weights):
    """(y, sum of the absolute products) in 64 bits."""
    ye = np.asarray(ye, np.float64)
    T, k = rows.shape
    y, size = np.zeros((T, ye.shape[1])), np.zeros((T, ye.shape[1]))
    for t in range(T):
        for j in range(k):
            if 0 <= rows[t, j] < ye.shape[0]:
                term = (1.0 if weights is None else float(weights[t, j])) * ye[rows[t, j]]
                y[t] += term
                size[t] += np.abs(term)
    return y, size


def clip(grads, max_norm, kind):
    """(norm, coefficient) of a list of arrays."""
    flat = [np.asarray(g, np.float64).ravel() for g in grads]
    if kind == "l2":
        norm = np.sqrt(sum((g * g).sum() for g in flat)) if flat else 0.0
    else:
        norm = max([np.abs(g).max() for g in flat if g.size], default=0.0)
    return float(norm), float(np.minimum(1.0, max_norm / (norm + 1e-6)))
