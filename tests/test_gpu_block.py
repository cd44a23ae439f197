"""The operators of an experts block together, between two layers of a graph: residual norm, logits by a dense layer, choice, experts."""
import numpy as np
import pytest
import torch

from paper_2307_00228_b200 import binding as B
from block_util import BF16, E4M3, F32, experts_reference, norm_reference, route_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "eight"])
@pytest.mark.parametrize("n", [1, 900])
def test_block_between_two_layers(kind, n):
    dtype = F32 if kind == "f32" else BF16
    g = torch.Generator().manual_seed(n)
    r = lambda *s: torch.randn(s, generator=g)   # noqa: E731
    dim, hidden, E, k, e = 64, 128, 8, 2, 6 * n
    indptr = torch.arange(0, e + 1, 6, dtype=torch.int64).cuda()
    indices = torch.randint(0, n, (e,), generator=g, dtype=torch.int32).cuda()
    graph = B.it_graph_create(indptr, indices)
    B.it_split_hubs(graph, 0)
    layer = B.LayerDesc(op="mean", act="relu", in_dim=dim, out_dim=dim, W=(r(2 * dim, dim) / 11).to(dtype).cuda())
    gate = B.LayerDesc(op="dense", act="none", in_dim=dim, out_dim=E, W=(r(dim, E) / 4).to(dtype).cuda())
    ws = torch.empty(max(B.it_workspace_bytes(graph, [layer]), B.it_workspace_bytes(graph, [gate])), dtype=torch.uint8, device="cuda")
    x, w_norm = r(n, dim).to(dtype).cuda(), (1 + 0.1 * r(dim)).cuda()
    W1, W2 = (r(E, dim, hidden) / 8), (r(E, hidden, dim) / 11).to(dtype)
    scale1 = (W1.abs().amax(1) / 448).contiguous() if kind == "eight" else None
    W1 = (W1 / scale1[:, None, :]).to(E4M3) if kind == "eight" else W1.to(dtype)
    h = torch.empty_like(x)
    B.it_layer_forward(graph, layer, x, h, ws)
    B.it_graph_check(graph)
    # what follows is compared stage by stage, each on the library's own input to it
    norm, s = torch.empty_like(x), torch.empty_like(x)
    B.it_residual_norm(B.NormDesc(dim=dim, feat_dtype=dtype, weight=w_norm), h, norm, residual=x, sum_out=s)
    logits = torch.empty(n, E, dtype=dtype, device="cuda")
    B.it_layer_forward(graph, gate, norm, logits, ws)
    ids, w = torch.empty(n, k, dtype=torch.int32, device="cuda"), torch.empty(n, k, device="cuda")
    rd = B.RouteDesc(n_experts=E, top_k=k, logit_dtype=dtype)
    B.it_route(rd, logits, ids, w)
    xin, x_scale = norm, None
    if kind == "eight":
        xin, x_scale = torch.empty(n, dim, dtype=E4M3, device="cuda"), torch.empty(n, device="cuda")
        B.it_residual_norm(B.NormDesc(dim=dim, feat_dtype=dtype, weight=w_norm, out_dtype=E4M3), h, xin, residual=x, scales=x_scale)
    d = B.ExpertsDesc(n_experts=E, top_k=k, in_dim=dim, hidden_dim=hidden, out_dim=dim, feat_dtype=dtype, W1=W1.cuda(), W2=W2.cuda(), act="relu",
                      w1_scale=None if scale1 is None else scale1.cuda())
    ews = torch.empty(B.it_experts_workspace_bytes(d, n), dtype=torch.uint8, device="cuda")
    y = torch.empty_like(x)
    B.it_experts_forward(d, xin, ids, w, y, ews, x_scale=x_scale)
    B.it_experts_check(ews)
    out = torch.empty_like(x)
    B.it_residual_norm(B.NormDesc(dim=dim, feat_dtype=dtype, weight=w_norm), y, out, residual=s)
    half = torch.finfo(dtype).eps / 2
    _, want = norm_reference(h, x, w_norm, 1e-5)
    assert ((norm.double() - want).abs() <= want.abs() * (half + 2e-6)).all()
    rid, rw = route_reference(rd, logits.float().cpu().numpy(), None)
    assert np.array_equal(ids.cpu().numpy(), rid) and np.allclose(w.cpu().numpy(), rw, rtol=1e-5)
    c = {"n": n, "E": E, "k": k, "a": dim, "h": hidden, "o": dim, "dtype": dtype, "gated": False, "act": "relu", "eight": kind == "eight", "x": xin, "x_scale": x_scale,
         "W1": W1, "w1_scale": scale1, "b1": None, "W2": W2, "b2": None, "ids": ids, "weights": w}
    ref, mag = experts_reference(c, "cuda")
    assert ((y.double() - ref).abs() <= mag * (half + 4e-5) + ref.abs() * half).all()
    _, want = norm_reference(y, s, w_norm, 1e-5)
    assert ((out.double() - want).abs() <= want.abs() * (half + 2e-6)).all()


def test_kernels_are_counted_and_profiled():
    x = torch.randn(100, 64, device="cuda")
    before = B.it_kernel_launch_count()
    B.it_profile_begin()
    B.it_residual_norm(B.NormDesc(dim=64, feat_dtype=F32), x, torch.empty_like(x))
    stats = {s["name"]: s for s in B.it_profile_end()}
    assert B.it_kernel_launch_count() == before + 1
    assert stats["residual_norm"]["launches"] == 1 and stats["residual_norm"]["algo_bytes"] == 2 * 100 * 64 * 4


@pytest.mark.parametrize("rounds", [12])
def test_arrays_written_by_the_call_before(rounds):
    """A kernel of these calls may start while the one before it still runs: the norm writes, each time something else, what the next call takes as its balance
    bias, as the first weights, their bias or their scales."""
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    E, n, a, o = 16, 60, 64, 64
    many = 1500
    norm = B.NormDesc(dim=64, feat_dtype=F32)
    one = B.NormDesc(dim=E, feat_dtype=F32)
    logits, logits2 = r(n, E), r(n, 64)
    bias, bias2 = torch.zeros(E, device="cuda"), torch.zeros(64, device="cuda")
    W1, b1 = torch.zeros(E, a, o, device="cuda"), torch.zeros(E, o, device="cuda")
    eight_W1, eight_scale = (r(E, a, o) * 50).to(E4M3), torch.zeros(E, o, device="cuda")
    routes = [(B.RouteDesc(n_experts=E, top_k=2, logit_dtype=F32, score="sigmoid", balance_bias=bias), logits, bias, one),
              (B.RouteDesc(n_experts=64, top_k=6, logit_dtype=F32, score="sigmoid", balance_bias=bias2), logits2, bias2, norm)]
    full = B.ExpertsDesc(n_experts=E, top_k=2, in_dim=a, out_dim=o, feat_dtype=F32, W1=W1, b1=b1)
    eight = B.ExpertsDesc(n_experts=E, top_k=2, in_dim=a, out_dim=o, feat_dtype=BF16, W1=eight_W1, w1_scale=eight_scale)
    ids, w = torch.randint(0, E, (many, 2), generator=g, device="cuda", dtype=torch.int32), torch.rand(many, 2, generator=g, device="cuda")
    x, x8, xs = r(many, a), (r(many, a) * 50).to(E4M3), torch.full((many,), 0.02, device="cuda")
    ws = torch.empty(max(B.it_experts_workspace_bytes(d, many) for d in (full, eight)), dtype=torch.uint8, device="cuda")

    def calls(sources, wait):
        """Every array from its source, then the call that takes it; `wait`: the GPU is waited for in between."""
        got = []
        b1.zero_()   # (the first products take it before it is written)
        sync = torch.cuda.synchronize if wait else lambda: None
        for (d, l, to, nd), src in zip(routes, sources):
            i, v = torch.empty(n, d.top_k, dtype=torch.int32, device="cuda"), torch.empty(n, d.top_k, device="cuda")
            B.it_residual_norm(nd, src, to.view(1, -1)); sync()
            B.it_route(d, l, i, v); sync()
            got += [i, v]
        for count in (n // 4, many):
            out, out8 = torch.empty(count, o, device="cuda"), torch.empty(count, o, dtype=BF16, device="cuda")
            B.it_residual_norm(norm, sources[2], W1.view(-1, 64)); sync()
            B.it_experts_forward(full, x[:count], ids[:count], w[:count], out, ws); sync()
            got.append(out.clone())
            B.it_residual_norm(norm, sources[3], b1); sync()
            B.it_experts_forward(full, x[:count], ids[:count], w[:count], out, ws); sync()
            B.it_residual_norm(norm, sources[3], eight_scale); sync()
            B.it_experts_forward(eight, x8[:count], ids[:count], w[:count], out8, ws, x_scale=xs[:count]); sync()
            got += [out, out8]
        return got

    every = [[r(1, E), r(1, 64), r(E * a, 64), r(E, 64)] for _ in range(rounds)]
    want = [calls(s, True) for s in every]
    for _ in range(3):
        got = [calls(s, False) for s in every]
        torch.cuda.synchronize()
        for a_, b_ in zip(got, want):
            for p, q in zip(a_, b_):
                assert torch.equal(p, q)


@pytest.mark.parametrize("field,value", [("act", 3), ("feat_dtype", 2), ("weight_dtype", 2), ("act_edge", 3)])
def test_a_layer_refuses_what_only_the_block_takes(field, value):
    """SiLU and 8-bit states: refused by the call itself, and nothing is written."""
    indptr = torch.arange(0, 33, 4, dtype=torch.int64, device="cuda")
    graph = B.it_graph_create(indptr, torch.zeros(32, dtype=torch.int32, device="cuda"))
    B.it_split_hubs(graph, 0)
    layer = B.LayerDesc(op="mean", act="none", in_dim=16, out_dim=16, W=torch.ones(32, 16, device="cuda"))
    if field == "act_edge":
        B.it_graph_set_edge_features(graph, torch.ones(32, 4, device="cuda"))
        layer = B.LayerDesc(op="mean", act="none", in_dim=16, out_dim=16, W=torch.ones(32, 16, device="cuda"), edge_dim=4, msg_dim=16, W_edge=torch.ones(20, 16, device="cuda"))
    ws = torch.empty(B.it_workspace_bytes(graph, [layer]), dtype=torch.uint8, device="cuda")
    x, out = torch.ones(8, 16, device="cuda"), torch.full((8, 16), 7.0, device="cuda")
    c = layer.to_c()
    setattr(c, field, value)
    with pytest.raises(B.ItError, match="IT_ERR_INVALID_ARG|IT_ERR_UNSUPPORTED"):
        B.it_layer_forward(graph, c, x, out, ws)
    assert (out == 7).all()
    B.it_layer_forward(graph, layer, x, out, ws)
    assert not (out == 7).all()
