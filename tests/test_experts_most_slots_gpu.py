"""As many slots as there can be: tokens * k just below 2^31, with a k that does not divide it."""
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_slots_just_below_2_31():
    k = 3
    tokens = ((1 << 31) - 1) // k                                    # 2147483646 slots
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty(tokens, 1, dtype=torch.bfloat16, device=DEV)
    for part in x.split(1 << 26):
        part.normal_(generator=g)
    order = torch.arange(tokens * k, dtype=torch.int32, device=DEV)
    place = order.view(tokens, k)
    y = dgs.gather_experts(x, order, place)
    assert y.shape == (tokens * k, 1)
    at = torch.cat([torch.arange(40, device=DEV), torch.randint(0, tokens * k, (1000,), generator=g, device=DEV), tokens * k - 1 - torch.arange(40, device=DEV)])
    assert torch.equal(y[at], x[at // k])
    out = dgs.gather_experts_grad(y, place)
    t = at // k
    # three times a bfloat16 number, rounded once
    assert torch.equal(out[t], (x[t].double() * 3).to(torch.bfloat16))
    assert dgs.operator_status(DEV) == 0
    more = tokens + 1
    with pytest.raises(dgs.DgsError) as e:
        dgs.dgs_experts_gather(dgs.dgs_matrix(x.data_ptr(), more, 0, 1, dgs.DGS_TYPE_BF16), order.data_ptr(), place.data_ptr(), k,
                               dgs.dgs_matrix(y.data_ptr(), more * k, 1, 1, dgs.DGS_TYPE_BF16))
    assert e.value.code == dgs.DGS_EINVAL
