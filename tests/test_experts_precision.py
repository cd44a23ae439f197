"""How exactly it_experts_forward multiplies fp32: 2-norms of the error against 64 bits."""
import pytest
import torch

from block_util import F32, experts_case, experts_reference, run_experts


def bound(*Ks):
    """For a chain of products with Ks terms.  A tensor core adds 16 terms at a time and may cut off what it adds by a whole step, 2^-23 of the sum, in runs of
    up to 512 terms; the sums of the runs are added to nearest, half a step each.  Four steps for what the six products leave out (three products of 2^-24),
    the bias and the rounding of a result."""
    return sum((min(K, 512) / 16 + (K + 511) // 512 / 2 + 4) * 2.0 ** -23 for K in Ks)


def error(c, got):
    ref, _ = experts_reference(c, "cuda")
    return ((got.double() - ref).norm() / ref.norm()).item()


@pytest.mark.gpu
@pytest.mark.parametrize("K,o,n,k", [(1024, 264, 1500, 2), (1032, 64, 700, 1), (4096, 520, 900, 1), (16384, 72, 600, 2), (65536, 64, 1000, 1)])
def test_long_sums_are_as_exact_as_short_ones(K, o, n, k):
    c = experts_case(K + o, n, 3, k, K, 0, o, F32, act="none", biased=True)
    got = run_experts(c)
    assert error(c, got) <= bound(K)
    assert torch.equal(run_experts(c), got)


@pytest.mark.gpu
@pytest.mark.parametrize("a,h,o,gated", [(64, 16384, 64, False), (8192, 1024, 16, True), (2048, 2056, 136, True)])
def test_long_sums_of_both_products(a, h, o, gated):
    """(gated: the relative errors of the two factors add up)"""
    c = experts_case(a + h, 700, 2, 2, a, h, o, F32, act="none", gated=gated, biased=False)
    assert error(c, run_experts(c)) <= bound(a, h) + (bound(a) if gated else 0)


# ----------------------------------------------------------------------------- six products, none of them missing
def split3(v):
    """fp32 as three bf16 parts, cut off: 8 bits each."""
    parts = []
    for _ in range(3):
        top = (v.view(torch.int32) & -65536).view(F32)
        parts.append(top.double())
        v = v - top
    return parts


def product_of_parts(x, w, missing=None):
    """The sum of the six products in 64 bits, or of the five others."""
    a, b = split3(x), split3(w)
    return sum(a[i] @ b[j] for i, j in SIX if (i, j) != missing)


SIX = [(2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0)]
SHORT = [(64, 0, 64), (256, 0, 128), (64, 256, 64), (128, 128, 128)]


@pytest.mark.parametrize("shape", SHORT, ids=str)
@pytest.mark.parametrize("missing", [None, *SIX], ids=str)
def test_the_bound_tells_a_missing_product(shape, missing):
    a, h, o = shape
    c = experts_case(a + h, 400, 1, 1, a, h, o, F32, act="none", biased=False)
    x = c["x"]
    for first, w in enumerate((c["W1"], c["W2"])):
        if w is None:
            continue
        want, got = x.double() @ w[0].double(), product_of_parts(x, w[0], missing)
        rel = ((got - want).norm() / want.norm()).item()
        if missing is None:
            assert rel <= 4 * 2.0 ** -24
        else:
            assert rel > 1.5 * bound(*((a, h) if h else (a,))), rel
        x = want.float()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHORT, ids=str)
@pytest.mark.parametrize("n,k", [(5, 2), (3000, 1), (2500, 3)])
def test_short_sums_keep_every_product(shape, n, k):
    a, h, o = shape
    c = experts_case(a + h + n, n, 5, k, a, h, o, F32, act="none", biased=False)
    assert error(c, run_experts(c)) <= bound(*((a, h) if h else (a,)))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [5, 3000])
def test_short_sums_keep_every_product_gated(n):
    """Each of the two factors, and the second product."""
    c = experts_case(n, n, 5, 2, 64, 128, 64, F32, act="none", gated=True, biased=False)
    assert error(c, run_experts(c)) <= bound(64, 64, 128)


@pytest.mark.gpu
@pytest.mark.parametrize("a,h,o,gated", [(512, 1024, 512, True), (512, 512, 64, True), (384, 384, 384, True), (320, 520, 136, True), (512, 512, 512, False), (512, 0, 256, False),
                                         (264, 0, 64, False), (1024, 2048, 72, False)])
@pytest.mark.parametrize("k", [1, 2])
def test_as_exact_as_plain_fp32(a, h, o, gated, k):
    """What the tensor cores cut off adds up over the factors of a gate and the products that follow one another, where roundings to nearest partly cancel: the result
    stays within one and a half times the error of the same products in plain fp32."""
    c = experts_case(a + h + o, 2000, 3, k, a, h, o, F32, act="none", gated=gated, biased=False)
    x, ids, w, W1 = (c[i].cuda() for i in ("x", "ids", "weights", "W1"))
    before, torch.backends.cuda.matmul.allow_tf32 = torch.backends.cuda.matmul.allow_tf32, False
    plain = torch.zeros(2000, o, device="cuda")
    for j in range(k):
        for e in range(3):
            v = (ids[:, j] == e).nonzero().flatten()
            y = x[v] @ W1[e]
            if gated:
                y = y[:, :h] * y[:, h:]
            if h:
                y = y @ c["W2"][e].cuda()
            plain[v] += w[v, j, None] * y
    torch.backends.cuda.matmul.allow_tf32 = before
    assert error(c, run_experts(c)) <= 1.5 * error(c, plain)
