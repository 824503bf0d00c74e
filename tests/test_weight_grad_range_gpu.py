"""Weight gradients at the ends of their types and sizes: gradients next to nothing."""
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("rows", [1, 600])               # few rows, and by the tensor cores
def test_f32_gradients_next_to_nothing(rows):
    """Three bfloat16 numbers add up to a float of at least 2^-110; below, what lies under bfloat16's last bit, 2^-133, may be missing, and no more."""
    g = torch.Generator(device=DEV).manual_seed(0)
    e = torch.randint(-149, -99, (1 << 14,), generator=g, device=DEV)
    d = (torch.ldexp(torch.rand(1 << 14, generator=g, device=DEV, dtype=torch.float64) + 1, e)).float()
    d[::2] *= -1
    h = torch.tensor([1.0, -1.0, 2.0, 64.0], device=DEV)
    x, dy = torch.zeros(rows, 4, device=DEV), torch.zeros(rows, 1 << 14, device=DEV)
    x[-1], dy[-1] = h, d
    c = dgs.Checkpoint(rows, 4, device=DEV)
    c.save(x)
    dw, db = torch.full((1 << 14, 4), float("nan"), device=DEV), torch.full((1 << 14,), float("nan"), device=DEV)
    c.weight_grad(dy, dw, db)
    cut = torch.where(d.abs() < 2.0 ** -110, 2.0 ** -133, 0.0).double()
    # a product with h, a power of two, is a float wherever d is
    assert bool(((dw.double() - d.double()[:, None] * h.double()).abs() <= cut[:, None] * h.abs().double()).all())
    assert bool(((db.double() - d.double()).abs() <= cut).all())
    assert dgs.operator_status(DEV) == 0
