"""Calls on views of more than two dimensions: the parts of a fused projection, a batch's rows apart, whatever lies evenly spaced."""
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_parts_of_a_fused_projection(dtype):
    g = torch.Generator(device=DEV).manual_seed(0)
    whole = torch.randint(-7, 8, (2, 40, 3 * 33), generator=g, device=DEV).to(dtype)
    x, dy, free = whole.split(33, dim=2)
    assert not x.is_contiguous()
    c = dgs.Checkpoint(80, 33, device=DEV)
    y = c.save(x, "relu")
    assert y.shape == x.shape and torch.equal(y, x.clamp(min=0)) and torch.equal(c.load().view(2, 40, 33), x.float())
    dx = c.activation_grad(dy, "relu")
    assert torch.equal(dx, dy * (x > 0))
    dw, db = torch.zeros(33, 33, device=DEV), torch.zeros(33, device=DEV)
    c.weight_grad(dy, dw, db)
    d = dy.reshape(80, 33).double()
    assert torch.equal(dw.double(), d.T @ x.reshape(80, 33).double()) and torch.equal(db.double(), d.sum(0))
    kept = whole.clone()
    c.load(out=free)                                     # written in place, and nothing beside it
    assert torch.equal(free.float(), x.float()) and torch.equal(whole[..., :66], kept[..., :66])
    a, b = dgs.route_experts(x, 4), dgs.route_experts(x.reshape(80, 33), 4)
    for p, q in zip(a, b):
        assert torch.equal(p, q)
    assert torch.equal(dgs.route_experts_grad(x, a.expert, a.weight), dgs.route_experts_grad(x.reshape(80, 33), a.expert, a.weight).view(2, 40, 33))
    assert dgs.operator_status(DEV) == 0
