"""What the torch-backed calls of a worker's own operators make of their arguments: no GPU needed."""
import pytest
import torch

from paper_1910_10929_b200 import operators


def test_a_router_is_made_from_the_values_that_arguments_have_now():
    scale, k, renormalise = torch.tensor(1.5), torch.tensor(2), torch.tensor(True)
    make = lambda: operators._router(k, "softmax", 1, 1, 1, renormalise, scale)   # noqa: E731
    r = make()
    assert (r.k, r.renormalise, r.scale) == (2, 1, 1.5)
    scale.fill_(0.25)
    k.fill_(3)
    renormalise.fill_(False)
    r = make()
    assert (r.k, r.renormalise, r.scale) == (3, 0, 0.25)
    for bad in (0, -1, 1.5, 1 << 31):
        with pytest.raises(ValueError):
            operators._router(bad, "softmax", 1, 1, 1, True, 1.0)
    with pytest.raises(ValueError):
        operators._router(2, "relu", 1, 1, 1, True, 1.0)
