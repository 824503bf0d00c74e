"""Which of a vocabulary's few-row calls go with tensor cores, told by their workspaces: no GPU needed."""
import pytest

import paper_1910_10929_b200 as dgs

P = 1 << 36
BF16, F32 = dgs.DGS_TYPE_BF16, dgs.DGS_TYPE_F32


def up(v, by=256):
    return -(-v // by) * by


def with_tensor_cores(rows, width, words, kind):
    """(loss, gradient): without tensor cores a loss keeps 8 bytes for each row and CTA (of 32 words at a time, at most 592) beside 4 for each row, and a gradient a part of dhidden for each
    CTA (of 8 words, 32 where they are many, at most 296)."""
    h, w = dgs.dgs_matrix(P, rows, width, width, kind), dgs.dgs_matrix(2 * P, words, width, width, kind)
    passes = -(-words // 32)
    ctas = -(-passes // -(-passes // 592))
    tiles = min(-(-words // (8 if words <= 1184 else 32)), 296)
    return (dgs.dgs_vocabulary_loss_bytes(h, w) != up(ctas * rows * 8) + up(rows * 4), dgs.dgs_vocabulary_loss_grad_bytes(h, w) != up(tiles * rows * width * 4))


@pytest.mark.parametrize("rows,width,words,kind", [(64, 16, 80000, BF16), (64, 16, 20000, BF16), (37, 64, 20000, BF16), (64, 16, 80000, F32), (64, 64, 20000, F32), (65, 16, 1000, BF16), (64, 768, 50257, F32)])
def test_narrow_words_go_with_tensor_cores_where_they_are_many(rows, width, words, kind):
    assert with_tensor_cores(rows, width, words, kind) == (True, True)


@pytest.mark.parametrize("rows,width,words,kind", [(1, 16, 5000, BF16), (37, 512, 1000, F32), (64, 16, 500, BF16), (8, 768, 5000, BF16), (1, 64, 20000, F32), (8, 300, 5000, F32)])
def test_few_products_go_without(rows, width, words, kind):
    assert with_tensor_cores(rows, width, words, kind) == (False, False)
