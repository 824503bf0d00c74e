"""The hidden states' gradient of a vocabulary's loss is rounded once, at its end: of 16-bit types it is off by half a step of its own value and by f32's errors, no more.

Tolerances: half a step exactly (2^-9 of the power of two at or below the value for bfloat16, 2^-12 for fp16), beside what s carries (its logit's error, the exponential, 22 bits, 2^-38 of the
largest dloss) and what its sums cut off, element by element as in test_vocabulary_gpu.py."""
import pytest
import torch

import paper_1910_10929_b200 as dgs
from test_vocabulary_gpu import cut, grad, logits, problem

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,width,words", [(40, 16, 300), (300, 16, 300), (130, 40, 2049), (700, 8, 777), (5000, 24, 1000)])
def test_hidden_gradient_is_rounded_once(rows, width, words, dtype):
    hidden, table, target, dloss = problem(rows, width, words, dtype, 21)
    for want_dw in (True, False):
        lse = dgs.vocabulary_loss(hidden, table, target).lse
        got, _ = grad(hidden, table, target, lse, dloss, want_dw=want_dw)
        live = target >= 0
        w, g = table.double(), torch.where(live, dloss.double(), 0.0)[:, None]
        z, dz = logits(hidden, table)
        x = z - lse.double()[:, None]
        p = torch.exp(x)
        y = torch.zeros_like(p)
        y[live] = y[live].scatter_(1, target[live][:, None], 1.0)
        s = g * (p - y)
        ds = g * (p * (1.1 * dz + x.abs() * 2.0 ** -22 + 3 * 2.0 ** -22) + y * 2.0 ** -23) + s.abs() * 2.0 ** -21 + float(g.max()) * 2.0 ** -38
        want = s @ w
        near = ds @ w.abs() + (s.abs() @ w.abs()) * (cut(2 * words) + 2.0 ** -23) + want.abs() * 3 * 2.0 ** -24
        info = torch.finfo(dtype)
        step = torch.exp2(torch.floor(torch.log2((want.abs() + near).clamp(min=info.smallest_normal)))) * info.eps
        assert bool(((got.double() - want).abs() <= step / 2 + near).all())
