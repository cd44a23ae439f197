"""it_residual_norm against its formula in 64 bits."""
import math

import pytest
import torch

from paper_2307_00228_b200 import binding as B
from block_util import BF16, E4M3, F32, HALF, norm_reference

pytestmark = pytest.mark.gpu


def _inputs(seed, n, dim, dtype, residual=True, weight=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    return (r(n, dim).to(dtype), (2 * r(n, dim)).to(dtype) if residual else None, 1 + 0.3 * r(dim) if weight else None)


def _tol(dim):
    # the sum of squares: a chain of at most max(32, dim / 256) + 13 additions of positive terms (halved by the root), the operands'
    # sum twice, reciprocal root 2 ulp = 2^-22, two products, the product of the mean
    return (0.5 * (max(32, dim / 256) + 13) + 2 + 4 + 3) * 2.0 ** -24


def _run(x, residual, weight, eight=False, want_sum=True, eps=1e-5, stream=None):
    d = B.NormDesc(dim=x.shape[1], feat_dtype=x.dtype, weight=weight, eps=eps, out_dtype=E4M3 if eight else None)
    out = torch.empty(x.shape, dtype=E4M3 if eight else x.dtype, device="cuda")
    scales = torch.empty(x.shape[0], device="cuda") if eight else None
    sum_out = torch.empty_like(x) if want_sum else None
    B.it_residual_norm(d, x, out, residual=residual, sum_out=sum_out, scales=scales, stream=stream)
    return out, scales, sum_out


def _check(x, residual, weight, out, scales, sum_out, eps=1e-5):
    s, y = norm_reference(x, residual, weight, eps)
    tol = _tol(x.shape[1])
    if sum_out is not None:
        plain = x.float() + residual.float() if residual is not None else x.float()
        assert torch.equal(sum_out, plain.to(x.dtype))
    if scales is None:
        assert ((out.double() - y).abs() <= y.abs() * (tol + HALF[x.dtype] * (1 + tol))).all()
        return
    want = (y.abs().amax(1) / 448).clamp_min(2.0 ** -126)
    assert ((scales.double() - want).abs() <= want * (tol + 2.0 ** -23)).all()
    got = out.double() * scales.double()[:, None]
    step = torch.maximum(y.abs() * HALF[E4M3], scales.double()[:, None] * 2.0 ** -10)   # half a step, of a subnormal too
    assert ((got - y).abs() <= step * (1 + 1e-5) + y.abs() * (2 * tol + 2.0 ** -22)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [8, 16, 24, 40, 64, 104, 128, 200, 256, 264, 512, 768, 1024, 1032, 2048, 20000])
@pytest.mark.parametrize("n", [1, 3, 130])
def test_against_formula(dtype, dim, n):
    x, r, w = _inputs(dim * 7 + n, n, dim, dtype)
    _check(x, r, w, *_run(x, r, w))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [16, 48, 64, 112, 128, 256, 768, 1024, 1040, 4096])
@pytest.mark.parametrize("n", [1, 5, 133])
def test_eight_bits(dtype, dim, n):
    x, r, w = _inputs(dim * 11 + n, n, dim, dtype)
    out, scales, sum_out = _run(x, r, w, eight=True)
    _check(x, r, w, out, scales, sum_out)
    assert (out.float().abs().amax(1) == 448).all()   # the largest entry of a row takes the type's largest value


@pytest.mark.parametrize("residual,weight,want_sum", [(False, True, False), (True, False, False), (False, False, True), (True, True, False)])
@pytest.mark.parametrize("dim", [64, 1536])
def test_optional_operands(residual, weight, want_sum, dim):
    x, r, w = _inputs(3, 77, dim, BF16, residual, weight)
    _check(x, r, w, *_run(x, r, w, want_sum=want_sum))


def test_many_rows():
    x, r, w = _inputs(5, 200_003, 64, BF16)
    _check(x, r, w, *_run(x, r, w))


@pytest.mark.parametrize("dim", [64, 1040])
@pytest.mark.parametrize("eight", [False, True])
def test_zeros_infinities_and_nan_stay_in_their_rows(dim, eight):
    x, _, w = _inputs(6, 9, dim, BF16, residual=False)
    x[1] = 0
    x[3, 5] = float("inf")
    x[5, 2] = float("nan")
    x[7] = 1e-30
    out, scales, _ = _run(x, None, w, eight=eight, want_sum=False)
    f = out.float()
    assert (f[1] == 0).all()
    assert f[3].isnan().any() and f[5].isnan().all()
    if eight:
        assert scales[1] == 2.0 ** -126 and scales[5].isnan()
    rows = [0, 2, 4, 6, 8]
    _check(x[rows], None, w, out[rows], scales[rows] if eight else None, None)


@pytest.mark.parametrize("dim", [128, 2048])
def test_outputs_over_their_inputs(dim):
    x, r, w = _inputs(8, 50, dim, F32)
    want, _, want_sum = _run(x, r, w)
    d = B.NormDesc(dim=dim, feat_dtype=F32, weight=w)
    x1, r1 = x.clone(), r.clone()
    B.it_residual_norm(d, x1, x1, residual=r1, sum_out=r1)
    assert torch.equal(x1, want) and torch.equal(r1, want_sum)
    x2, r2 = x.clone(), r.clone()
    B.it_residual_norm(d, x2, r2, residual=r2, sum_out=x2)
    assert torch.equal(r2, want) and torch.equal(x2, want_sum)


def test_rows_behind_the_last_are_left():
    x, r, w = _inputs(9, 40, 64, BF16)
    out, s = torch.full_like(x, 7), torch.full_like(x, 7)
    d = B.NormDesc(dim=64, feat_dtype=BF16, weight=w)
    B.it_residual_norm(d, x[:37], out[:37], residual=r[:37], sum_out=s[:37])
    assert (out[37:] == 7).all() and (s[37:] == 7).all() and not (out[36] == 7).all()


def test_offsets_past_32_bits():
    n, dim = (1 << 31) // 256 + 5, 256
    x = torch.ones(n, dim, dtype=BF16, device="cuda")
    x[-3:] = torch.arange(dim, device="cuda").to(BF16)
    out = torch.zeros_like(x)
    B.it_residual_norm(B.NormDesc(dim=dim, feat_dtype=BF16), x, out)
    _check(x[-9:], None, None, out[-9:], None, None)
    _check(x[:9], None, None, out[:9], None, None)


def test_other_stream_and_captured_replays():
    x, r, w = _inputs(10, 300, 96, BF16)
    want = _run(x, r, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = _run(x, r, w, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0])
    d = B.NormDesc(dim=96, feat_dtype=BF16, weight=w)
    out, sum_out, xin = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.it_residual_norm(d, xin, out, residual=r, sum_out=sum_out)
    for scale in (1.0, 0.5):
        xin.copy_(x * scale)
        graph.replay()
        again = _run((x * scale), r, w)
        assert torch.equal(out, again[0]) and torch.equal(sum_out, again[2])


def test_no_rows():
    x = torch.empty(0, 64, dtype=BF16, device="cuda")
    assert B.it_residual_norm(B.NormDesc(dim=64, feat_dtype=BF16), x, torch.empty_like(x)).shape == (0, 64)
    assert math.isclose(HALF[BF16], torch.finfo(BF16).eps / 2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [16, 256, 1040, 2064])
@pytest.mark.parametrize("eight", [False, True])
def test_rows_beyond_the_range_of_their_squares(dim, dtype, eight):
    """What the header says of infinities, NaN, squares that overflow or vanish, and eps = 0."""
    x, _, w = _inputs(12, 8, dim, dtype, residual=False)
    w = w.abs() + 0.1
    x[1, 3] = -float("inf")
    x[2, dim - 1] = float("nan")
    x[3, 7] = 3e19
    x[4] = 1e-30
    x[5] = 0
    x[5, 2] = -1e-30
    out, scales, _ = _run(x, None, w, eight=eight, want_sum=False, eps=0.0)
    f = out.float()
    others = [i for i in range(dim) if i != 3]
    if eight:
        assert f[1].isnan().all() and scales[1].isnan() and f[2].isnan().all() and scales[2].isnan()
        assert (f[3] == 0).all() and scales[3] == 2.0 ** -126
    else:
        assert f[1, 3].isnan() and (f[1, others] == 0).all() and f[2].isnan().all() and (f[3] == 0).all()
        assert (f[4] == float("inf")).all()
        assert f[5, 2] == -float("inf") and f[5, others[3:]].isnan().all()
    rows = [0, 6, 7]
    _check(x[rows], None, w, out[rows], scales[rows] if eight else None, None, eps=0.0)
