"""Activations at every finite number of the 16-bit types, subnormal ones included, against 64-bit activations."""
import pytest
import torch

import paper_1910_10929_b200 as dgs
from test_checkpoint_gpu import act64, half_step

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def numbers(dtype):
    x = torch.arange(1 << 16, device=DEV).to(torch.int16).view(dtype)
    return torch.where(torch.isfinite(x), x, 0.0).view(64, 1024)


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_activation_of_every_number(dtype, act):
    x = numbers(dtype)
    y = dgs.Checkpoint(*x.shape, device=DEV).save(x, act)
    want, u = act64(act, x.double())
    # in f32, relative to the result: 16 roundings of 2^-24 and those of the exponent (3 |u| of them, for erfc's argument 2 x^2, each counted as 4), then one
    # rounding to the type, half a subnormal step at least.  Where the score itself is subnormal in f32 (|u| > 87, x < 105 there) half a step of it, times x: 2^-143.
    rel = (16 + 4 * (x.double() ** 2 if act == "gelu" else u.abs()).clamp(max=400)) * 2.0 ** -24
    bound = want.abs() * rel * (1 + torch.finfo(dtype).eps) + half_step(dtype, want) + 2.0 ** -140
    off = (y.double() - want).abs()
    assert bool((off <= bound).all()), [(float(a), float(b), float(c)) for a, b, c in zip(x[off > bound][:5], y[off > bound][:5], want[off > bound][:5])]
