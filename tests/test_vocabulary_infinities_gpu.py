"""Words that are impossible: an infinity in the vocabulary whose logits are -inf takes the word out of the softmax, in every type and with or without tensor cores."""
import pytest
import torch

import paper_1910_10929_b200 as dgs
from test_vocabulary_gpu import check_grad, check_loss, problem

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,width,words", [(40, 64, 300), (300, 64, 300), (300, 200, 3000), (9, 16, 100), (500, 17, 1000)])
def test_words_of_minus_infinity_have_no_probability(rows, width, words, dtype):
    hidden, table, target, dloss = problem(rows, width, words, dtype, 31, by=0.5)
    hidden = hidden.abs() + 2.0 ** -6
    hidden[: rows // 2] = (hidden[: rows // 2] * 16).round() / 16 + 0.0625          # few digits: numbers whose second parts are 0
    gone = torch.tensor([7, words // 2, words - 1], device=DEV)
    target = torch.where((target[:, None] == gone).any(1), 0, target)
    keep = torch.ones(words, dtype=torch.bool, device=DEV)
    keep[gone] = False
    rest, at = table[keep], torch.where(target >= 0, (torch.cumsum(keep, 0) - 1)[target.clamp(min=0)], target)      # the vocabulary without those words
    dirty = table.clone()
    dirty[gone[0]] = -INF                                                           # a whole row, and two with one such number beside a large one
    dirty[gone[1:], 3] = -INF
    dirty[gone[1:], 5] = 60000.0
    got = dgs.vocabulary_loss(hidden, dirty, target)
    check_loss(hidden, rest, at, got)
    dw = torch.full((words * width,), 9.0, device=DEV)
    dgs.vocabulary_loss_grad(hidden, dirty, target, got.lse, dloss, dw)             # dhidden is NaN, by the formula: 0 * inf
    assert dgs.operator_status(DEV) == 0
    dw = dw.view(words, width)
    assert not dw[~keep].any()
    check_grad(hidden, rest, at, got.lse, dloss, dgs.vocabulary_loss_grad(hidden, rest, at, got.lse, dloss), dw[keep])
    # one number alone: dhidden's other columns
    table[gone[0]], table[gone[0], 3] = 0.0, -INF
    got = dgs.vocabulary_loss(hidden, table, target)
    dh = dgs.vocabulary_loss_grad(hidden, table, target, got.lse, dloss)
    others = torch.arange(width, device=DEV) != 3
    more = torch.arange(words, device=DEV) != gone[0]
    at = torch.where(target > gone[0], target - 1, target)
    same = dgs.vocabulary_loss_grad(hidden, table[more], at, got.lse, dloss)
    check_grad(hidden, table[more], at, got.lse, dloss, torch.where(others, dh, same), None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [40, 300])
def test_infinities_that_are_no_impossible_words(rows, dtype):
    hidden, table, target, dloss = problem(rows, 64, 300, dtype, 32)
    target[0] = 11
    table[11] = -INF
    hidden[0] = hidden[0].abs() + 0.5                                               # its own target is impossible
    hidden[1] = -hidden[0]                                                          # a logit of +inf
    hidden[2] = torch.where(torch.arange(64, device=DEV) % 2 == 0, 1.0, -1.0)       # inf - inf
    hidden[3, 5] = 0.0                                                              # inf * 0
    target[1:4] = 5
    got = dgs.vocabulary_loss(hidden, table, target)
    assert float(got.loss[0]) == INF and bool(torch.isfinite(got.lse[0]))
    assert bool(torch.isnan(got.loss[1:4]).all()) and bool(torch.isnan(got.lse[1:4]).all())


@pytest.mark.parametrize("rows", [40, 300])
def test_large_numbers_beside_an_infinity_stay_what_they_are(rows):
    """f32: numbers past fp16's largest in a row and column that hold an infinity too."""
    g = torch.Generator(device=DEV).manual_seed(5)
    hidden = torch.rand(rows, 40, generator=g, device=DEV) * 2.0 ** -20 + 2.0 ** -22
    table = torch.randn(300, 40, generator=g, device=DEV) * 2.0 ** 20
    target = torch.randint(1, 300, (rows,), generator=g, device=DEV)
    dirty = table.clone()
    dirty[0, 7] = -INF
    dirty[0, 8] = 2.0 ** 22
    keep = torch.arange(300, device=DEV) > 0
    got = dgs.vocabulary_loss(hidden, dirty, target)
    check_loss(hidden, table[keep], target - 1, got)
    dloss = torch.rand(rows, generator=g, device=DEV)
    dw = torch.empty(300 * 40, device=DEV)
    dgs.vocabulary_loss_grad(hidden, dirty, target, got.lse, dloss, dw)
    same = dgs.vocabulary_loss_grad(hidden, table[keep].contiguous(), target - 1, got.lse, dloss)
    check_grad(hidden, table[keep], target - 1, got.lse, dloss, same, dw.view(300, 40)[1:])
    # dhidden's other columns: s of the word is 0
    alone = table.clone()
    alone[0, 7] = -INF
    dh = dgs.vocabulary_loss_grad(hidden, alone, target, dgs.vocabulary_loss(hidden, alone, target).lse, dloss)
    others = torch.arange(40, device=DEV) != 7
    assert bool(torch.isfinite(dh[:, others]).all())
