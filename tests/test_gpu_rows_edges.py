"""Operators on whole sets of rows where their calls could go wrong: lists that leave blocks empty, limits of waits, extreme magnitudes,
overlapping and unaligned arguments. Against the formulas in 64 bits; tolerances count roundings (u = 2^-24)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def P(wpsgd_lib):
    import paper_1708_04801_b200 as pkg

    return pkg


# ---- short lists: one cluster of blocks ------------------------------------------------------------------------------------
@pytest.mark.parametrize("tensors", [1, 2, 7, 16])
def test_norms_of_short_lists_call_after_call(P, tensors):
    # with fewer chunks than blocks, the blocks without any reach the exchange of sums at once: every call finds all sums
    g = torch.Generator().manual_seed(tensors)
    grads = [torch.randn(500 + 3 * i, generator=g).cuda() for i in range(tensors)]
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))
    with P.Context(1, 8) as ctx:
        lists = P.GradList(grads)
        norms = torch.cat([ctx.grad_norm(lists) for _ in range(2000)])
        ctx.check()
    # squares of at most 16 elements a thread in fp32 (products and additions: 16 u), half of it in the root, rounded once; the rest in fp64
    assert bool((norms == norms[0]).all()) and abs(float(norms[0]) - want) <= 10 * U * want
