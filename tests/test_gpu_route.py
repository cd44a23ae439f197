"""it_route against its definition in 64 bits: the choice exactly, the weights to their rounding."""
import numpy as np
import pytest
import torch

from paper_2307_00228_b200 import binding as B
from block_util import BF16, F32, route_reference

pytestmark = pytest.mark.gpu

# weights: expf 2 ulp, the rounded difference from the top (|x| < 20) 10 ulp, a sum of 8 to 32 experts a lane and 5 steps across lanes at half
# an ulp each, two products and a division; twice where the sum of the chosen divides
RTOL = 2 * (2 + 10 + 19 + 3) * 2.0 ** -23


def _run(d, logits, stream=None):
    n = logits.shape[0]
    ids = torch.full((n + 1, d.top_k), 77, dtype=torch.int32, device="cuda")
    w = torch.full((n + 1, d.top_k), 77.0, device="cuda")
    B.it_route(d, logits, ids[:n], w[:n], stream=stream)
    if stream is not None:
        stream.synchronize()
    assert (ids[n] == 77).all() and (w[n] == 77).all()   # rows behind the last are left
    return ids[:n].cpu().numpy(), w[:n].cpu().numpy()


def _check(d, logits, bias=None):
    ids, w = _run(d, logits)
    rid, rw = route_reference(d, logits.float().cpu().numpy(), None if bias is None else bias.cpu().numpy())
    assert np.array_equal(ids, rid), np.argwhere(ids != rid)[:5]
    assert np.allclose(w, rw, rtol=RTOL, atol=1e-30)


def _logits(seed, n, e, dtype, masked=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    l = (1.5 * torch.randn(n, e, generator=g, device="cuda")).to(dtype)
    if masked:
        l[torch.rand(n, e, generator=g, device="cuda") < masked] = -float("inf")
    return l


EXPERTS = [1, 2, 5, 8, 9, 16, 17, 32, 33, 60, 64, 100, 128, 200, 256, 300, 512, 1000, 1024]


@pytest.mark.parametrize("e", EXPERTS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
def test_choice_and_weights(e, dtype, score, biased):
    for n, k, renorm in ((1, 1, True), (33, min(e, 2), False), (70, min(e, 8), True), (5, min(e, 32), True)):
        l = _logits(e + n, n, e, dtype, masked=0.0 if n == 33 else 0.1)
        bias = 0.1 * torch.randn(e, generator=torch.Generator().manual_seed(e)).cuda() if biased else None
        _check(B.RouteDesc(n_experts=e, top_k=k, logit_dtype=dtype, score=score, balance_bias=bias, renormalise=renorm, weight_scale=1.0 if renorm else 2.5), l, bias)


@pytest.mark.parametrize("e,groups,group_k", [(8, 2, 1), (16, 4, 2), (64, 8, 3), (60, 5, 2), (256, 8, 4), (96, 32, 7), (512, 16, 4), (1024, 1024, 9), (128, 64, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("score,biased", [("softmax", False), ("sigmoid", True), ("softmax", True)])
def test_groups(e, groups, group_k, dtype, score, biased):
    for best in (1, 2):
        for masked in (0.0, 0.4):
            l = _logits(e + best, 41, e, dtype, masked)
            l[3] = -float("inf")
            bias = 0.1 * torch.randn(e, generator=torch.Generator().manual_seed(e)).cuda() if biased else None
            d = B.RouteDesc(n_experts=e, top_k=min(8, e // groups * group_k), logit_dtype=dtype, score=score, balance_bias=bias, n_groups=groups, group_k=group_k,
                            group_best=best)
            _check(d, l, bias)


@pytest.mark.parametrize("e", [4, 16, 64, 256, 700])
@pytest.mark.parametrize("biased", [False, True])
def test_ties_go_to_the_lowest_index(e, biased):
    l = torch.randint(0, 3, (50, e), generator=torch.Generator().manual_seed(e)).to(BF16).cuda()
    bias = torch.zeros(e, device="cuda") if biased else None
    _check(B.RouteDesc(n_experts=e, top_k=min(e, 6), logit_dtype=BF16, balance_bias=bias), l, bias)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("e", [12, 64, 256])
def test_keys_closer_than_32_bits_resolve(score, e):
    """A bias that makes all keys of the row nearly equal: they differ by its rounding to fp32 alone."""
    for seed in range(12):
        l = torch.randn(1, e, generator=torch.Generator().manual_seed(seed))
        s = torch.softmax(l.double(), 1) if score == "softmax" else torch.sigmoid(l.double())
        bias = (0.5 - s[0]).float()
        d = B.RouteDesc(n_experts=e, top_k=5, logit_dtype=F32, score=score, balance_bias=bias.cuda())
        _check(d, l.cuda(), bias)


@pytest.mark.parametrize("e", [6, 48])
def test_values_that_close_an_expert(e):
    l = _logits(1, 12, e, F32)
    l[0] = -float("inf")
    l[1] = float("nan")
    l[2, :] = float("nan"); l[2, 3] = 0.5
    l[3, 2] = float("inf"); l[3, 4] = float("inf")
    l[4, 1:] = -float("inf")
    l[5] = 3e38; l[5, 1] = -3e38
    l[6] = torch.finfo(F32).min
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            d = B.RouteDesc(n_experts=e, top_k=3, logit_dtype=F32, score=score, renormalise=renorm)
            _check(d, l)
    bias = torch.zeros(e); bias[1] = -float("inf"); bias[2] = float("nan")
    _check(B.RouteDesc(n_experts=e, top_k=3, logit_dtype=F32, score="sigmoid", balance_bias=bias.cuda()), l, bias)


def test_peaked_rows():
    """Scores far below the largest: their rounding comes from the difference of the logits."""
    l = 25 * torch.randn(300, 64, generator=torch.Generator().manual_seed(2))
    bias = torch.zeros(64)
    d = B.RouteDesc(n_experts=64, top_k=8, logit_dtype=F32, balance_bias=bias.cuda())
    ids, _ = _run(d, l.cuda())
    rid, _ = route_reference(d, l.numpy(), bias.numpy())
    assert np.array_equal(ids, rid)


def test_unaligned_rows_and_views():
    base = _logits(4, 3001, 24, BF16).flatten()
    l = base[1:1 + 2000 * 24].view(2000, 24)   # rows that start at odd elements
    _check(B.RouteDesc(n_experts=24, top_k=4, logit_dtype=BF16), l)


def test_many_rows_are_the_same_every_time():
    l = _logits(5, 300_001, 16, BF16)
    d = B.RouteDesc(n_experts=16, top_k=2, logit_dtype=BF16)
    a, b = _run(d, l), _run(d, l)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    rid, rw = route_reference(d, l[-700:].float().cpu().numpy(), None)
    assert np.array_equal(a[0][-700:], rid) and np.allclose(a[1][-700:], rw, rtol=RTOL)


def test_other_stream_and_captured_replays():
    l = _logits(6, 500, 32, F32)
    d = B.RouteDesc(n_experts=32, top_k=4, logit_dtype=F32)
    want = _run(d, l)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = _run(d, l, stream=s)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    ids, w, lin = torch.zeros(500, 4, dtype=torch.int32, device="cuda"), torch.zeros(500, 4, device="cuda"), torch.zeros_like(l)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.it_route(d, lin, ids, w)
    for sign in (1, -1):
        lin.copy_(sign * l)
        graph.replay()
        want = _run(d, sign * l)
        assert np.array_equal(ids.cpu().numpy(), want[0]) and np.array_equal(w.cpu().numpy(), want[1])


def test_no_rows():
    l = torch.empty(0, 8, device="cuda")
    B.it_route(B.RouteDesc(n_experts=8, top_k=2, logit_dtype=F32), l, torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda"))


def test_offsets_past_32_bits():
    n, e = (1 << 31) // 16 + 100, 16
    l = torch.zeros(n, e, dtype=BF16, device="cuda")
    l[-50:] = _logits(7, 50, e, BF16)
    d = B.RouteDesc(n_experts=e, top_k=1, logit_dtype=BF16)
    ids, w = torch.empty(n, 1, dtype=torch.int32, device="cuda"), torch.empty(n, 1, device="cuda")
    B.it_route(d, l, ids, w)
    rid, rw = route_reference(d, l[-60:].float().cpu().numpy(), None)
    assert np.array_equal(ids[-60:].cpu().numpy(), rid) and np.allclose(w[-60:].cpu().numpy(), rw, rtol=RTOL)
    assert (ids[:1000] == 0).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("e", [4, 20, 32, 60, 64, 256, 700])
def test_a_key_behind_the_border_may_be_the_least_exact(score, e):
    """Two keys of tiny scores at the border of the choice, and behind them one of a score near 1 and a bias near -1, which 32 bits know far less
    exactly: its exact key passes the others' in some rows and not in others."""
    a, b, c, d, n = 3, 1, 0, 2, 201
    l = np.full((n, e), -60.0, np.float32)
    l[:, [a, b]], l[:, d] = -40.0, 0.0
    l[:, c] = np.float32(5.2739234) + np.float32(4.7683716e-7) * (np.arange(n, dtype=np.float32) - n // 2)
    for q in range(12):
        bias = np.full(e, -8.0, np.float32)
        bias[a] = np.float32(0.01) + np.float32(q * 1.1e-8)
        bias[b] = bias[a] - np.float32(7.45e-9)
        bias[c] = np.float32(0.01) - np.float32(1 / (1 + np.exp(-np.float64(l[n // 2, c]))))   # (a softmax over c, d and next to nothing is that sigmoid)
        bias = torch.from_numpy(bias)
        for k in (1, 2):
            _check(B.RouteDesc(n_experts=e, top_k=k, logit_dtype=F32, score=score, balance_bias=bias.cuda(), renormalise=False), torch.from_numpy(l).cuda(), bias)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("e,size", [(16, 4), (40, 4), (64, 8), (60, 5), (256, 32), (96, 3), (1024, 64)])
def test_groups_whose_best_two_nearly_cancel(score, e, size):
    """The worth of a group is a sum of two keys; large biases of opposite sign leave a small one, which 32 bits know by the size of the keys alone."""
    g, n = e // size, 64
    rng = np.random.default_rng(e)
    for magnitude in (3.0, 40.0, 1000.0):
        bias = np.full(e, -1e6, np.float32).reshape(g, size)
        for i in range(g):
            big = np.float32(magnitude * (1 + 0.1 * rng.random()))
            two = rng.choice(size, 2, replace=False)
            bias[i, two[0]], bias[i, two[1]] = big, -big
        bias = bias.reshape(e)
        step = np.spacing(np.float32(magnitude))   # scores differ by a few steps of the keys
        l = (10 * step * (e if score == "softmax" else 1) * rng.normal(size=(n, e))).astype(np.float32)
        bias = torch.from_numpy(bias)
        for group_k in (1, g - 1):
            d = B.RouteDesc(n_experts=e, top_k=2, logit_dtype=F32, score=score, balance_bias=bias.cuda(), n_groups=g, group_k=group_k, group_best=2, renormalise=False)
            _check(d, torch.from_numpy(l).cuda(), bias)


@pytest.mark.parametrize("scale", [1.0, 2.5])
@pytest.mark.parametrize("e,k,groups", [(2, 1, 1), (8, 2, 1), (16, 4, 1), (30, 3, 1), (32, 8, 1), (60, 4, 1), (64, 6, 8), (60, 6, 5), (256, 8, 1), (256, 8, 8), (700, 20, 1)])
@pytest.mark.parametrize("score,biased", [("sigmoid", False), ("sigmoid", True), ("softmax", True)])
def test_weights_of_scores_that_32_bits_do_not_hold(score, biased, e, k, groups, scale):
    """The chosen share a weight of 1 between them however small their scores are, also where e^-90 and e^-700 are 0 in 32 bits."""
    g = torch.Generator().manual_seed(e + k)
    depth = torch.tensor([0.0, 20, 60, 80, 85, 86, 87, 87.5, 88, 88.3, 88.5, 88.7, 89, 90, 95, 100, 103, 104, 110, 130, 200, 400, 600, 680])
    n = depth.numel()
    l = 12 * torch.rand(n, e, generator=g) - depth[:, None]
    bias = None
    if score == "softmax":   # one expert far above, which the bias keeps out: the chosen lie `depth` below it
        l[:, e // 2] = 12.0
    if biased:
        bias = 3 * torch.rand(e, generator=g)
        bias[e // 2] = -9.0
    groups = groups if e > 2 else 1
    d = B.RouteDesc(n_experts=e, top_k=k, logit_dtype=F32, score=score, balance_bias=None if bias is None else bias.cuda(), n_groups=groups, group_k=max(1, groups // 2),
                    group_best=2, weight_scale=scale)
    _check(d, l.cuda(), bias)
    _, w = _run(d, l.cuda())
    assert np.allclose(w.sum(1), scale, rtol=1e-5)


def test_scores_that_64_bits_do_not_hold_are_0():
    """As in 64 bits, where 1 / (1 + e^-l) ends at a logit of -709.78 and e^-x at x = 745: weight 0, whatever the others are."""
    l = torch.tensor([[-709.9, -720.0, -800.0], [-1e4, -3e38, -720.0], [-600.0, -601.0, -700.0]])
    ids, w = _run(B.RouteDesc(n_experts=3, top_k=2, logit_dtype=F32, score="sigmoid"), l.cuda())
    assert (ids == [[0, 1], [2, 0], [0, 1]]).all()
    assert (w[:2] == 0).all() and np.allclose(w[2], [1 / (1 + np.exp(-1)), 1 / (1 + np.exp(1))], rtol=RTOL)
    bias = torch.tensor([-9.0, 0.25, 0.0])
    l = torch.tensor([[0.0, -746.0, -747.0], [0.0, -700.0, -701.0], [30.0, -800.0, 0.0]])
    ids, w = _run(B.RouteDesc(n_experts=3, top_k=2, logit_dtype=F32, balance_bias=bias.cuda()), l.cuda())
    assert (ids == [1, 2]).all()
    assert (w[0] == 0).all() and np.allclose(w[1], [1 / (1 + np.exp(-1)), 1 / (1 + np.exp(1))], rtol=RTOL) and (w[2] == [0, 1]).all()
