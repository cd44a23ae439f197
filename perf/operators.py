"""The mixture-of-experts block that may stand between two layers, as cases that can be timed and compared.

A block is: residual addition and root-mean-square norm of every vertex state (`it_residual_norm`), the choice of experts per
vertex (`it_route`, on the logits of a dense layer), and the chosen experts' products, weighted and added up
(`it_experts_forward`).  Every case is one call of one of the three.  Sizes run from a single vertex, scored on request, to all
vertices of the larger graphs of this repository's workloads; widths are those of its layers (64 to 768 columns).

A case is a dict of plain values:
  kind      "norm" | "route" | "experts"
  dtype     storage type of states, weights and outputs ("f32" | "bf16")
  n         vertices
  norm:     dim; residual: a second operand is added, and the sum is stored; eight: the output is e4m3 with a scale per row
  route:    experts, top_k; score ("softmax" | "sigmoid"); bias: a balance bias; groups, group_k, group_best; renorm; scale;
            masked: share of logits that are minus infinity (and of rows where all are)
  experts:  experts, top_k, dims "in-hidden-out" ("in-out": one product); act; gated; biased: products have a bias;
            eight: states and first weights are e4m3; masked: share of places that name no expert
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
EPS = 1e-5


def listed():
    return [
        # One vertex whose 768-column text embedding is normalised on request: a latency.
        dict(name="norm_one", kind="norm", dtype="bf16", n=1, dim=768, residual=True, eight=False),
        # Raw features of 100 columns, an odd number of vertices, fp32.
        dict(name="norm_f32_odd", kind="norm", dtype="f32", n=610_001, dim=100, residual=True, eight=False),
        # States that go on to experts in 8 bits.
        dict(name="norm_eight", kind="norm", dtype="bf16", n=1_000_003, dim=256, residual=True, eight=True),
        # Every vertex of the attention workload's graph between two of its layers.
        dict(name="norm_large", kind="norm", dtype="bf16", n=5_000_000, dim=128, residual=True, eight=False),
        # A handful of vertices scored on request, sigmoid scores with a balance bias.
        dict(name="route_few", kind="route", dtype="f32", n=7, experts=64, top_k=4, score="sigmoid", bias=True, groups=1, group_k=1, group_best=1,
             renorm=True, scale=1.0, masked=0.0),
        # All vertices of a graph over a few experts, two each.
        dict(name="route_top2", kind="route", dtype="bf16", n=2_000_000, experts=16, top_k=2, score="softmax", bias=False, groups=1, group_k=1, group_best=1,
             renorm=True, scale=1.0, masked=0.0),
        # Many experts in groups, a balance bias, some experts closed to some vertices.
        dict(name="route_groups", kind="route", dtype="f32", n=200_003, experts=256, top_k=8, score="sigmoid", bias=True, groups=8, group_k=4, group_best=2,
             renorm=True, scale=2.5, masked=0.05),
        # One vertex through its two experts: weights read once, nothing else matters.
        dict(name="experts_one", kind="experts", dtype="bf16", n=1, experts=16, top_k=2, dims="256-1024-256", act="relu", gated=False, biased=True,
             eight=False, masked=0.0),
        # A small graph in fp32.
        dict(name="experts_f32", kind="experts", dtype="f32", n=20_001, experts=8, top_k=2, dims="64-256-64", act="elu", gated=False, biased=True,
             eight=False, masked=0.0),
        # All vertices of a large graph through two of sixteen experts.
        dict(name="experts_large", kind="experts", dtype="bf16", n=1_000_000, experts=16, top_k=2, dims="128-512-128", act="relu", gated=False, biased=True,
             eight=False, masked=0.0),
        # Typed vertices: one matrix per type, states in 8 bits, some vertices of no type.
        dict(name="experts_typed_eight", kind="experts", dtype="bf16", n=1_500_001, experts=8, top_k=1, dims="256-256", act="relu", gated=False, biased=True,
             eight=True, masked=0.02),
        # Wide states (text embeddings) through four of thirty-two gated experts.
        dict(name="experts_wide", kind="experts", dtype="bf16", n=40_003, experts=32, top_k=4, dims="768-1024-768", act="silu", gated=True, biased=False,
             eight=False, masked=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "route", "experts", "experts"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "norm":
        dim = 16 * _log(rng, 1, 64) if rng.random() < 0.7 else 8 * rng.randrange(1, 200)
        eight = dim % 16 == 0 and rng.random() < 0.4
        return dict(kind=kind, dtype=dtype, n=_log(rng, 1, 320_000_000 // max(dim, 64)), dim=dim, residual=rng.random() < 0.7, eight=eight)
    if kind == "route":
        experts = rng.choice([2, 5, 8, 12, 16, 32, 60, 64, 100, 128, 160, 256])
        top_k = min(experts, rng.choice([1, 2, 2, 3, 4, 6, 8]))
        groups = rng.choice([g for g in (1, 1, 2, 4, 8) if experts % g == 0 and experts // g >= 4 or g == 1])
        group_k = rng.randrange(1, groups + 1)
        while group_k * (experts // groups) < top_k:
            group_k += 1
        return dict(kind=kind, dtype=dtype, n=_log(rng, 1, 40_000_000 // max(experts, 16)), experts=experts, top_k=top_k, score=rng.choice(["softmax", "sigmoid"]),
                    bias=rng.random() < 0.5, groups=groups, group_k=group_k, group_best=rng.choice([1, 2]), renorm=rng.random() < 0.7,
                    scale=rng.choice([1.0, 1.0, 2.5]), masked=rng.choice([0.0, 0.0, 0.1]))
    experts = rng.choice([2, 4, 7, 8, 16, 16, 32, 64])
    top_k = min(experts, rng.choice([1, 2, 2, 3, 4]))
    eight = dtype == "bf16" and rng.random() < 0.35
    step = 16 if eight else 8
    width = lambda lo, hi: step * _log(rng, lo // step, hi // step)   # noqa: E731
    a, c = width(32, 512), width(32, 512)
    two = rng.random() < 0.7
    hidden = width(64, 1024) if two else 0
    gated = two and rng.random() < 0.4
    per = 2 * (a * hidden * (2 if gated else 1) + hidden * c if two else a * c)   # flops of one place
    most = min(1_000_000, int(1.2e11 if dtype == "f32" else 4e11) // (per * top_k))
    return dict(kind=kind, dtype=dtype, n=_log(rng, 1, max(2, most)), experts=experts, top_k=top_k, dims="%d-%d-%d" % (a, hidden, c) if two else "%d-%d" % (a, c),
                act=rng.choice(["none", "relu", "elu", "silu"]), gated=gated, biased=rng.random() < 0.7, eight=eight, masked=rng.choice([0.0, 0.0, 0.1]))


# ----------------------------------------------------------------------------- inputs
def _widths(case):
    d = [int(v) for v in case["dims"].split("-")]
    return (d[0], d[1], d[2]) if len(d) == 3 else (d[0], 0, d[1])


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 17)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)   # noqa: E731
    uniform = lambda *shape: torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)   # noqa: E731
    n, t = case["n"], DTYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"] == "norm":
        s["x"] = normal(n, case["dim"]).to(t)   # what a layer adds
        s["residual"] = (2 * normal(n, case["dim"])).to(t) if case["residual"] else None   # the stream it is added to
        s["weight"] = 1 + 0.2 * normal(case["dim"])
        return s
    if case["kind"] == "route":
        e = case["experts"]
        s["logits"] = (1.5 * normal(n, e)).to(t)
        if case["masked"]:
            s["logits"][uniform(n, e) < case["masked"]] = -math.inf
            s["logits"][uniform(n) < case["masked"] / 10] = -math.inf
        s["bias"] = 0.05 * normal(e) if case["bias"] else None
        return s
    e, k = case["experts"], case["top_k"]
    a, hidden, c = _widths(case)
    n1 = (2 * hidden if case["gated"] else hidden) or c
    glorot = lambda fi, fo: (2 * uniform(e, fi, fo) - 1) * math.sqrt(6 / (fi + fo))   # noqa: E731
    s["x"], s["x_scale"] = normal(n, a).to(t), None
    s["w1"], s["w1_scale"] = glorot(a, n1), None
    if case["eight"]:   # one scale per vertex and per column of an expert
        big = s["x"].float().abs().amax(1).clamp_min(1e-20) / 448
        s["x"], s["x_scale"] = (s["x"].float() / big[:, None]).to(E4M3), big
        big = s["w1"].abs().amax(1).clamp_min(1e-20) / 448
        s["w1"], s["w1_scale"] = (s["w1"] / big[:, None, :]).to(E4M3), big.contiguous()
    else:
        s["w1"] = s["w1"].to(t)
    s["b1"] = 0.1 * (2 * uniform(e, n1) - 1) if case["biased"] else None
    s["w2"] = glorot(hidden, c).to(t) if hidden else None
    s["b2"] = 0.1 * (2 * uniform(e, c) - 1) if case["biased"] and hidden else None
    score = normal(n, e) + 0.7 * normal(e)   # some experts are met more often than others
    w, ids = torch.topk(score, k, dim=1)
    s["ids"] = ids.to(torch.int32).contiguous()
    s["weights"] = torch.softmax(w, 1).contiguous()
    if case["masked"]:
        none = uniform(n, k) < case["masked"]
        s["ids"][none] = -1
        s["weights"][none] = 0
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# ----------------------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"norm": _own_norm, "route": _own_route, "experts": _own_experts}[kind](state)
    return {"norm": _norm, "route": _route, "experts": _experts}[kind](state)


def _own_norm(s):
    from paper_2307_00228_b200 import binding as B
    if "desc" not in s:   # what a program keeps: the description and its output buffers
        c, x = s["case"], s["x"]
        s["desc"] = B.NormDesc(dim=c["dim"], feat_dtype=x.dtype, weight=s["weight"], eps=EPS, out_dtype=E4M3 if c["eight"] else x.dtype)
        s["out"] = torch.empty(x.shape, dtype=E4M3 if c["eight"] else x.dtype, device=x.device)
        s["scales"] = torch.empty(c["n"], device=x.device) if c["eight"] else None
        s["sum"] = torch.empty_like(x) if c["residual"] else None
    B.it_residual_norm(s["desc"], s["x"], s["out"], residual=s["residual"], sum_out=s["sum"], scales=s["scales"])
    return [v for v in (s["out"], s["scales"], s["sum"]) if v is not None]


def _own_route(s):
    from paper_2307_00228_b200 import binding as B
    if "desc" not in s:
        c, x = s["case"], s["logits"]
        s["desc"] = B.RouteDesc(n_experts=c["experts"], top_k=c["top_k"], logit_dtype=x.dtype, score=c["score"], balance_bias=s["bias"], n_groups=c["groups"],
                                group_k=c["group_k"], group_best=c["group_best"], renormalise=c["renorm"], weight_scale=c["scale"])
        s["ids"] = torch.empty(c["n"], c["top_k"], dtype=torch.int32, device=x.device)
        s["weights"] = torch.empty(c["n"], c["top_k"], device=x.device)
    B.it_route(s["desc"], s["logits"], s["ids"], s["weights"])
    return [s["ids"], s["weights"]]


def _own_experts(s):
    from paper_2307_00228_b200 import binding as B
    if "desc" not in s:
        c, x = s["case"], s["x"]
        a, hidden, o = _widths(c)
        s["desc"] = B.ExpertsDesc(n_experts=c["experts"], top_k=c["top_k"], in_dim=a, hidden_dim=hidden, out_dim=o, act=c["act"], gated=c["gated"],
                                  feat_dtype=DTYPES[c["dtype"]], W1=s["w1"], b1=s["b1"], W2=s["w2"], b2=s["b2"], w1_scale=s["w1_scale"])
        s["out"] = torch.empty(c["n"], o, dtype=DTYPES[c["dtype"]], device=x.device)
        s["workspace"] = torch.empty(B.it_experts_workspace_bytes(s["desc"], c["n"]), dtype=torch.uint8, device=x.device)
    B.it_experts_forward(s["desc"], s["x"], s["ids"], s["weights"], s["out"], s["workspace"], x_scale=s["x_scale"])
    return s["out"]


def _norm(s):
    v = s["x"].float()
    if s["residual"] is not None:
        v = v + s["residual"].float()
    y = v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * s["weight"]
    if s["case"]["eight"]:
        scale = (y.abs().amax(1) / 448).clamp_min(2.0 ** -126)
        out = [(y / scale[:, None]).clamp(-448, 448).to(E4M3), scale]
    else:
        out = [y.to(s["x"].dtype)]
    return out + ([v.to(s["x"].dtype)] if s["residual"] is not None else [])


def _route(s):
    """In 64 bits: the choice goes by scores that may lie next to each other.  Ties go to the lowest index (stable sorts)."""
    c = s["case"]
    l = s["logits"].double()
    n, e = l.shape
    open_ = l > -math.inf
    if c["score"] == "softmax":
        p = torch.where(open_, torch.exp(l - l.amax(1, keepdim=True).clamp_min(-1e300)), 0.0)
        score = p / p.sum(1, keepdim=True).clamp_min(1e-300)
    else:
        score = 1 / (1 + torch.exp(-l))
    # without a bias the order of the scores is that of the logits
    key = score + s["bias"].double() if s["bias"] is not None else score
    key = torch.where(open_, key, -math.inf)
    if c["groups"] > 1:
        size = e // c["groups"]
        in_group = key.view(n, c["groups"], size)
        best = torch.sort(in_group, dim=2, descending=True).values[:, :, :c["group_best"]]
        group = torch.where(best > -math.inf, best, 0.0).sum(2)
        group = torch.where(best[:, :, 0] > -math.inf, group, -math.inf)
        kept = torch.sort(group, dim=1, descending=True, stable=True).indices[:, :c["group_k"]]
        chosen = torch.zeros_like(group, dtype=torch.bool).scatter_(1, kept, True)
        key = torch.where(chosen[:, :, None], in_group, -math.inf).reshape(n, e)
    top = torch.sort(key, dim=1, descending=True, stable=True)
    none = top.values[:, :c["top_k"]] == -math.inf
    ids = top.indices[:, :c["top_k"]]
    w = torch.where(none, 0.0, score.gather(1, ids))
    if c["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return [torch.where(none, -1, ids).to(torch.int32), (w * c["scale"]).float()]


def _act(v, act):
    if act == "relu":
        return v.clamp_min(0)
    if act == "elu":
        return torch.where(v > 0, v, torch.expm1(v.clamp_max(0)))
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return v


def _experts(s):
    """The places sorted by expert, each expert's rows padded to the longest, and one batched product over the experts."""
    c, ids, k = s["case"], s["ids"].long(), s["case"]["top_k"]
    a, hidden, o = _widths(c)
    n, e = c["n"], c["experts"]
    flat = torch.where(ids < 0, e, ids).view(-1)
    order = torch.sort(flat, stable=True).indices
    count = torch.bincount(flat, minlength=e + 1)
    first = torch.cumsum(count, 0) - count
    longest = max(1, int(count[:e].max()))   # a program with elementary operations has to know it on the host
    place = torch.arange(longest, device=flat.device)
    real = place[None, :] < count[:e, None]
    slot = order[(first[:e, None] + place[None, :]).clamp_max(n * k - 1)]
    x = s["x"].float() if s["x_scale"] is None else s["x"].float() * s["x_scale"][:, None]
    w1 = s["w1"].float() if s["w1_scale"] is None else s["w1"].float() * s["w1_scale"][:, None, :]
    h = torch.bmm(x[torch.div(slot, k, rounding_mode="floor")], w1)
    if s["b1"] is not None:
        h = h + s["b1"][:, None, :]
    h = _act(h[:, :, :hidden], c["act"]) * h[:, :, hidden:] if c["gated"] else _act(h, c["act"])
    if hidden:
        h = torch.bmm(h, s["w2"].float())
        if s["b2"] is not None:
            h = h + s["b2"][:, None, :]
    y = torch.zeros(n * k, o, device=flat.device)
    y[slot[real]] = h[real]
    y = y * s["weights"].view(-1, 1)
    return y.view(n, k, o).sum(1).to(DTYPES[c["dtype"]])


# ----------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    n, size = case["n"], 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norm":
        d = case["dim"]
        reads = n * d * size * (2 if case["residual"] else 1) + 4 * d
        writes = (n * (d + 4) if case["eight"] else n * d * size) + (n * d * size if case["residual"] else 0)
        return {"bytes": reads + writes, "flops": n * d * (6 if case["residual"] else 5)}
    if case["kind"] == "route":
        return {"bytes": n * (case["experts"] * size + case["top_k"] * 8) + (4 * case["experts"] if case["bias"] else 0),
                "flops": n * case["experts"] * (4 + case["top_k"])}
    a, hidden, o = _widths(case)
    n1 = (2 * hidden if case["gated"] else hidden) or o
    places, met = n * case["top_k"] * (1 - case["masked"]), min(case["experts"], n * case["top_k"])
    one = 1 if case["eight"] else size
    weights = met * (a * n1 * one + hidden * o * size)
    return {"bytes": n * (a * one + o * size + case["top_k"] * 8 + (4 if case["eight"] else 0)) + weights, "flops": places * 2 * (a * n1 + hidden * o)}


# ----------------------------------------------------------------------------- from the definitions, in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "norm":
        v = s["x"].double() + (0 if s["residual"] is None else s["residual"].double())
        y = v / (v.square().sum(1, keepdim=True) / case["dim"] + EPS).sqrt() * s["weight"].double()
        out = [y]
        if case["eight"]:   # the values that the 8 bits round, and their scale
            scale = y.abs().max(1).values / 448
            out = [y / scale[:, None], scale]
        return out + ([v] if case["residual"] else [])
    if case["kind"] == "route":
        return _exact_route(case, s)
    k = case["top_k"]
    a, hidden, o = _widths(case)
    out = torch.zeros(case["n"], o, dtype=torch.float64, device="cuda")
    for j in range(k):
        for e in range(case["experts"]):
            rows = (s["ids"][:, j] == e).nonzero().flatten()
            for part in rows.split(1 << 18):
                x, w = s["x"][part].double(), s["w1"][e].double()
                if case["eight"]:
                    x, w = x * s["x_scale"][part, None].double(), w * s["w1_scale"][e].double()
                h = x @ w
                if case["biased"]:
                    h += s["b1"][e].double()
                g = h[:, :hidden] if case["gated"] else h
                if case["act"] == "relu":
                    g = torch.relu(g)
                elif case["act"] == "elu":
                    g = torch.where(g > 0, g, torch.exp(g.clamp_max(0)) - 1)
                elif case["act"] == "silu":
                    g = g * torch.sigmoid(g)
                if case["gated"]:
                    g = g * h[:, hidden:]
                if hidden:
                    g = g @ s["w2"][e].double()
                    if case["biased"]:
                        g += s["b2"][e].double()
                out[part] += s["weights"][part, j, None].double() * g
    return out


def _exact_route(case, s):
    import numpy as np
    l = s["logits"].double().cpu().numpy()
    n, e = l.shape
    if n * e > 120_000_000:
        return None
    with np.errstate(over="ignore", invalid="ignore"):
        if case["score"] == "softmax":
            m = l.max(1, keepdims=True)
            z = np.exp(l - np.where(np.isfinite(m), m, 0.0))
            total = z.sum(1, keepdims=True)
            score = z / np.where(total > 0, total, 1.0)
        else:
            score = 1.0 / (1.0 + np.exp(-l))
    key = score if s["bias"] is None else score + s["bias"].double().cpu().numpy()
    shut = np.isneginf(l)
    key[shut] = -np.inf
    if case["groups"] > 1:
        size = e // case["groups"]
        rank = -np.sort(-key.reshape(n, case["groups"], size), axis=2)[:, :, :case["group_best"]]
        any_ = rank[:, :, 0] > -np.inf
        group = np.where(any_, np.where(np.isneginf(rank), 0.0, rank).sum(2), -np.inf)
        out_of = np.argsort(-group, axis=1, kind="stable")[:, case["group_k"]:]
        shut_group = np.zeros_like(any_)
        np.put_along_axis(shut_group, out_of, True, axis=1)
        key = np.where(np.repeat(shut_group, size, axis=1), -np.inf, key)
    ids = np.argsort(-key, axis=1, kind="stable")[:, :case["top_k"]]
    none = np.isneginf(np.take_along_axis(key, ids, axis=1))
    w = np.where(none, 0.0, np.take_along_axis(score, ids, axis=1))
    if case["renorm"]:
        total = w.sum(1, keepdims=True)
        w = w / np.where(total > 0, total, 1.0)
    return [torch.from_numpy(np.where(none, -1, ids).astype(np.int32)), torch.from_numpy(w * case["scale"])]
