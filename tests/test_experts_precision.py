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
