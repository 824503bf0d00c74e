"""What a vocabulary's gradient is added to keeps its subnormal numbers, at every size."""
import pytest
import torch

import paper_1910_10929_b200 as dgs
from test_vocabulary_gpu import grad, problem

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,width,words", [(40, 64, 300), (300, 64, 3000), (300, 264, 5000), (20_000, 40, 300), (130, 31, 1000)])
def test_subnormal_numbers_that_are_added_to(rows, width, words, dtype):
    hidden, table, target, dloss = problem(rows, width, words, dtype, 51)
    g = torch.Generator(device=DEV).manual_seed(1)
    bits = torch.randint(0, 1 << 23, (words, width), generator=g, device=DEV, dtype=torch.int32)
    bits = torch.where(torch.rand(words, width, generator=g, device=DEV) < 0.5, bits, bits | -(1 << 31))
    before = bits.view(torch.float32)
    lse = dgs.vocabulary_loss(hidden, table, target).lse
    # nothing is added: every bit stays (-0 + 0 is 0)
    _, dw = grad(hidden, table, torch.full_like(target, -1), lse, dloss, before)
    got = dw.contiguous().view(torch.int32)
    assert bool(((got == bits) | ((bits == -(1 << 31)) & (got == 0))).all())
    # a gradient that is subnormal itself: sums of f32 numbers below 2^-126 are exact
    small = dloss * (2.0 ** -130 / float(dloss.max()))
    _, alone = grad(hidden, table, target, lse, small)
    assert bool((alone != 0).any())
    _, dw = grad(hidden, table, target, lse, small, before)
    want = before.double() + alone.double()
    assert bool(((dw.double() - want).abs() <= 2.0 ** -149 + want.abs() * 2.0 ** -24).all())
