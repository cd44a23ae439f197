"""Plain 64-bit forms of the operators of an experts block, and seeded inputs for their tests."""
from __future__ import annotations

import numpy as np
import torch

from paper_2307_00228_b200 import binding as B

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8, E4M3: 2.0 ** -4}   # a rounding is off by at most this, relative


def norm_reference(x, residual, weight, eps):
    s = x.double() + (residual.double() if residual is not None else 0)
    y = s / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    return s, y * weight.double() if weight is not None else y


def route_reference(d: B.RouteDesc, logits: np.ndarray, bias: np.ndarray | None):
    """Row by row, from the header's text."""
    n, E = logits.shape
    ids, ws = np.full((n, d.top_k), -1, np.int64), np.zeros((n, d.top_k))
    l = logits.astype(np.float64)
    l = np.where(np.isnan(l), -np.inf, np.minimum(l, np.finfo(np.float32).max))
    for v in range(n):
        open_ = l[v] > -np.inf
        score = np.zeros(E)
        with np.errstate(over="ignore"):
            if d.score == "softmax":
                z = np.exp(l[v][open_] - (l[v][open_].max() if open_.any() else 0))
                score[open_] = z / z.sum()
            else:
                score[open_] = 1 / (1 + np.exp(-l[v][open_]))
        key = np.where(open_, l[v] if bias is None else score + bias.astype(np.float64), -np.inf)
        key = np.where(np.isnan(key), -np.inf, key)
        if d.n_groups > 1:
            size = E // d.n_groups
            worth = np.full(d.n_groups, -np.inf)
            for g in range(d.n_groups):
                best = np.sort(key[g * size:(g + 1) * size])[::-1]
                best = best[best > -np.inf][:d.group_best]
                if best.size == 0:
                    continue
                if bias is None and d.group_best == 2:
                    best = np.sort(score[g * size:(g + 1) * size])[::-1][:best.size]
                worth[g] = best.sum()
            keep = sorted(range(d.n_groups), key=lambda g: (-worth[g], g))[:d.group_k]
            for g in range(d.n_groups):
                if g not in keep:
                    key[g * size:(g + 1) * size] = -np.inf
        order = sorted(range(E), key=lambda e: (-key[e], e))[:d.top_k]
        for j, e in enumerate(order):
            if key[e] > -np.inf:
                ids[v, j], ws[v, j] = e, score[e]
        if d.renormalise:
            t = ws[v].sum()
            ws[v] = ws[v] / t if t > 0 else 0
    return ids, ws * d.weight_scale


def act64(v, name):
    if name == "relu":
        return v.clamp_min(0)
    if name == "elu":
        return torch.where(v > 0, v, torch.expm1(v.clamp_max(0)))
    if name == "silu":
        return v * torch.sigmoid(v)
    return v


def experts_case(seed, n, E, k, a, h, o, dtype, gated=False, act="relu", biased=True, eight=False, masked=0.0, repeat=False, skew=None, device="cpu"):
    """Inputs on the CPU: x, x_scale, W1, w1_scale, b1, W2, b2, ids, weights."""
    g = torch.Generator().manual_seed(seed)
    n1 = h * (2 if gated else 1) if h else o
    c = {"n": n, "E": E, "k": k, "a": a, "h": h, "o": o, "dtype": dtype, "gated": gated, "act": act, "eight": eight}
    x, w1 = torch.randn(n, a, generator=g), (2 * torch.rand(E, a, n1, generator=g) - 1) * (6 / (a + n1)) ** 0.5
    c["x_scale"] = c["w1_scale"] = None
    if eight:
        c["x_scale"] = x.abs().amax(1).clamp_min(1e-3) / 448 if n else torch.zeros(0)
        c["w1_scale"] = (w1.abs().amax(1) / 448).contiguous()
        c["x"], c["W1"] = (x / c["x_scale"][:, None]).to(E4M3), (w1 / c["w1_scale"][:, None, :]).to(E4M3)
    else:
        c["x"], c["W1"] = x.to(dtype), w1.to(dtype)
    c["b1"] = 0.2 * torch.randn(E, n1, generator=g) if biased else None
    c["W2"] = ((2 * torch.rand(E, h, o, generator=g) - 1) * (6 / (h + o)) ** 0.5).to(dtype) if h else None
    c["b2"] = 0.2 * torch.randn(E, o, generator=g) if biased and h else None
    if skew is not None:      # share of the places that all go to expert 0
        ids = torch.where(torch.rand(n, k, generator=g) < skew, 0, torch.randint(0, E, (n, k), generator=g))
    elif repeat or k > E:
        ids = torch.randint(0, E, (n, k), generator=g)
    else:
        ids = torch.rand(n, E, generator=g).argsort(1)[:, :k]
    ids[torch.rand(n, k, generator=g) < masked] = -1
    c["ids"], c["weights"] = ids.to(torch.int32).contiguous(), torch.rand(n, k, generator=g)
    return c


def experts_desc(c, device="cuda"):
    dev = lambda t: None if t is None else t.to(device)   # noqa: E731
    return B.ExpertsDesc(n_experts=c["E"], top_k=c["k"], in_dim=c["a"], hidden_dim=c["h"], out_dim=c["o"], feat_dtype=c["dtype"], W1=dev(c["W1"]),
                         b1=dev(c["b1"]), W2=dev(c["W2"]), b2=dev(c["b2"]), act=c["act"], gated=c["gated"], w1_scale=dev(c["w1_scale"]))


def experts_reference(c, device="cpu"):
    """(result, magnitude of its terms) in 64 bits: the magnitude is sum_j |w_j| (sum_h |hidden_h| |W2_h| + |b2|), with what the first product's
    terms add to it for one product."""
    up = lambda t: None if t is None else t.to(device).double()   # noqa: E731
    x, W1, W2, b1, b2, ws = (up(c[k]) for k in ("x", "W1", "W2", "b1", "b2", "weights"))
    if c["eight"]:
        x, W1 = x * up(c["x_scale"])[:, None], W1 * up(c["w1_scale"])[:, None, :]
    ids = c["ids"].to(device).long()
    out = torch.zeros(c["n"], c["o"], dtype=torch.float64, device=device)
    mag = torch.zeros_like(out)
    for e in range(c["E"]):
        v, j = (ids == e).nonzero(as_tuple=True)
        if v.numel() == 0:
            continue
        h, m = x[v] @ W1[e], x[v].abs() @ W1[e].abs()
        if b1 is not None:
            h, m = h + b1[e], m + b1[e].abs()
        if c["gated"]:
            gate, u = act64(h[:, :c["h"]], c["act"]), h[:, c["h"]:]
            m = m[:, :c["h"]] * u.abs() + gate.abs() * m[:, c["h"]:]
            h = gate * u
        else:
            h = act64(h, c["act"])
        first = m   # what the first product's own rounding scales with
        if c["h"]:
            m = (h.abs() + first) @ W2[e].abs()
            h = h @ W2[e]
            if b2 is not None:
                h, m = h + b2[e], m + b2[e].abs()
        out.index_put_((v,), ws[v, j, None] * h, accumulate=True)
        mag.index_put_((v,), ws[v, j, None].abs() * (m if c["h"] else m + h.abs()), accumulate=True)
    return out, mag


def run_experts(c, device="cuda", stream=None, desc=None, workspace=None):
    d = experts_desc(c) if desc is None else desc
    dev = lambda t: None if t is None else t.to(device)   # noqa: E731
    out = torch.full((c["n"], c["o"]), float("nan"), dtype=c["dtype"], device=device)
    ws = torch.full((B.it_experts_workspace_bytes(d, c["n"]),), 0xff, dtype=torch.uint8, device=device) if workspace is None else workspace
    B.it_experts_forward(d, dev(c["x"]), dev(c["ids"]), dev(c["weights"]), out, ws, x_scale=dev(c["x_scale"]), stream=stream)
    B.it_experts_check(ws)
    return out


def experts_tolerance(c, out, mag):
    """Bound of |result - reference|.  Accumulation in fp32: at most K * 2^-23 of the magnitudes for either product, wherever a sum is cut (a
    tensor core may truncate: a whole step); the activation's own error is below 2e-6 of its argument's magnitude.  bf16: the stored
    hidden row is off by 2^-8, and the result by 2^-8 of itself."""
    depth = (c["a"] + (c["h"] or 0) + c["k"] + 16) * 2.0 ** -23 + 4e-6
    half = HALF[c["dtype"]]
    return mag * (depth + (half if c["h"] and c["dtype"] == BF16 else 0)) * 1.01 + out.abs() * half


def check_experts(c, got, device="cpu"):
    ref, mag = experts_reference(c, device)
    err = (got.to(device).double() - ref).abs()
    tol = experts_tolerance(c, ref, mag)
    assert torch.isfinite(got).all()
    assert (err <= tol).all(), (err / tol.clamp_min(1e-300)).max().item()
    # and as a whole, against an indexing mistake that a row of large terms would hide: rounding errors are independent, so in the 2-norm
    # they stay below their bound for single entries: two roundings of 2^-8 for bf16 (hidden row, result), accumulation for fp32
    rel = (err.norm() / ref.norm().clamp_min(1e-30)).item()
    assert rel <= (1e-2 if c["dtype"] == BF16 else 2e-5), rel
