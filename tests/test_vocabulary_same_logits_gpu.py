"""Loss and gradient form the same logits, bit by bit, where both go with tensor cores or both without: of a word that is certain beyond f32's reach the loss' own lse is the
word's logit, so that exp(z - lse) - 1 and with it the whole gradient is 0 and not a rounding of two sums."""
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [40, 300])                          # without tensor cores and with them
@pytest.mark.parametrize("width", [64, 100, 128, 192, 304, 384, 576, 640, 768, 896, 1000])
def test_a_certain_word_leaves_no_gradient(rows, width, dtype):
    g = torch.Generator(device=DEV).manual_seed(width)
    words = 500
    table = torch.randn(words, width, generator=g, device=DEV).to(dtype)
    target = torch.randint(0, words, (rows,), generator=g, device=DEV)
    hidden = table[target] * 8                                       # a power of two: exact
    z = hidden.double() @ table.double().T
    best = z.gather(1, target[:, None])
    # the others' exponentials are 0 in f32, whatever the sums' roundings; targets whose words lie too near to others are left out
    target = target.masked_fill((best - z.scatter(1, target[:, None], float("-inf")).amax(1, keepdim=True) < 128)[:, 0], -1)
    assert int((target >= 0).sum()) > rows / 2
    loss, lse = dgs.vocabulary_loss(hidden, table, target)
    assert not loss.any()
    dw = torch.full((words * width,), 7.0, device=DEV)
    dh = dgs.vocabulary_loss_grad(hidden, table, target, lse, torch.rand(rows, generator=g, device=DEV) + 0.5, dw)
    assert dgs.operator_status(DEV) == 0
    assert not dh.any() and not dw.any()
