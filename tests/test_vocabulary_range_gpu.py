"""Hidden states and vocabularies near the ends of f32's range whose logits and gradients lie within it: powers of two that are taken out and put back must not leave the range on the way."""
import pytest
import torch

import paper_1910_10929_b200 as dgs
from test_vocabulary_gpu import check_grad, check_loss, cut, logits, problem

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# without tensor cores; with them; partial results of dW (many rows, few words)
SIZES = [(40, 32, 300), (300, 32, 3000), (20_000, 40, 300)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("by", [115, 60, -60, -110])
@pytest.mark.parametrize("rows,width,words", SIZES)
def test_large_times_small(rows, width, words, by, dtype):
    hidden, table, target, dloss = problem(rows, width, words, dtype, 41, by=1.0)
    h, w = hidden * 2.0 ** by, table * 2.0 ** -by                    # logits as before
    got = dgs.vocabulary_loss(h, w, target)
    check_loss(h, w, target, got)
    for scale in (0, -by // 2):                                      # dW about as large as h, and half way back
        g = dloss * 2.0 ** scale
        dw = torch.empty(words * width, device=DEV)
        dh = dgs.vocabulary_loss_grad(h, w, target, got.lse, g, dw)
        assert dgs.operator_status(DEV) == 0
        # dhidden is as large as the vocabulary times dloss: where its terms' magnitudes add up to more than f32 holds nothing is asked, and below f32's normal numbers each of the words'
        # additions may be off by half of 2^-149
        live = target >= 0
        z, dz = logits(h, w)
        x = z - got.lse.double()[:, None]
        p = torch.exp(x)
        y = torch.zeros_like(p)
        y[live] = y[live].scatter_(1, target[live][:, None], 1.0)
        factor = torch.where(live, g.double(), 0.0)[:, None]
        s = factor * (p - y)
        ds = factor * (p * (1.1 * dz + x.abs() * 2.0 ** -22 + 3 * 2.0 ** -22) + y * 2.0 ** -23) + s.abs() * 2.0 ** -21 + float(g.max()) * 2.0 ** -38
        info, want, size = torch.finfo(dtype), s @ w.double(), s.abs() @ w.double().abs()
        near = ds @ w.double().abs() + size * (cut(2 * words) + 2.0 ** -21) + want.abs() * (info.eps / 2) * (1 + 2.0 ** -8) + info.smallest_normal * info.eps + words * 2.0 ** -150
        assert bool((((dh.double() - want).abs() <= near) | (size + near > torch.finfo(torch.float32).max)).all())
        # dW likewise; rows' additions below the normal numbers
        m = torch.where(live[:, None], h.double(), 0.0)
        want, size = s.T @ m, s.abs().T @ m.abs()
        near = ds.T @ m.abs() + size * (cut(2 * rows) + 2.0 ** -21) + want.abs() * 3 * 2.0 ** -24 + rows * 2.0 ** -150 + 2.0 ** -149
        assert bool(((dw.view(words, width).double() - want).abs() <= near).all())


@pytest.mark.parametrize("rows,width,words", SIZES)
def test_one_large_column_and_a_small_loss(rows, width, words):
    hidden, table, target, dloss = problem(rows, width, words, torch.bfloat16, 42, by=1.0)
    hidden[:, 3] = hidden[:, 3] * 2.0 ** 120
    table[:, 3] = 0.0                                                # no part in the logits
    dloss = dloss * 2.0 ** -60
    got = dgs.vocabulary_loss(hidden, table, target)
    dw = torch.empty(words * width, device=DEV)
    dh = dgs.vocabulary_loss_grad(hidden, table, target, got.lse, dloss, dw)
    assert bool(torch.isfinite(dw).all())
    check_grad(hidden, table, target, got.lse, dloss, dh, dw.view(words, width))
