"""Results that torch's differentiation does not see are not handed out in silence."""
import warnings

import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_result_that_is_cut_off_warns():
    z = torch.randn(10, 8, device=DEV, requires_grad=True)
    c = dgs.Checkpoint(10, 8, device=DEV)
    with pytest.warns(UserWarning, match="route_experts returns is cut off"):
        r = dgs.route_experts(z, 2)
    assert not r.weight.requires_grad
    with pytest.warns(UserWarning, match="Checkpoint.save returns is cut off"):
        y = c.save(z, "silu")
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        c.save(z)                                        # holds z, which stays what it is to torch
        with torch.no_grad():
            assert torch.equal(dgs.route_experts(z, 2).weight, r.weight) and torch.equal(c.save(z, "silu"), y)
        assert torch.equal(dgs.route_experts(z.detach(), 2).weight, r.weight)
        # a backward pass of one's own: torch records nothing there
        class Route(torch.autograd.Function):
            @staticmethod
            def forward(ctx, z):
                r = dgs.route_experts(z, 2)
                ctx.save_for_backward(z, r.expert)
                return r.weight

            @staticmethod
            def backward(ctx, dweight):
                return dgs.route_experts_grad(*ctx.saved_tensors, dweight)
        w = Route.apply(z)
        (w * torch.arange(2, device=DEV)).sum().backward()
    want = torch.autograd.grad((torch.softmax(z.double().gather(1, r.expert.long()), 1) * torch.arange(2, device=DEV)).sum(), z)[0]
    # p (g - sum g p) of two weights: each at most 1, off by the 48 roundings of a weight and a few more
    assert float((z.grad.double() - want.double()).abs().max()) < 2 * 64 * 2.0 ** -24
