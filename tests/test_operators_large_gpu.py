"""The operators where offsets pass 32 bits: more than 2^32 values in a checkpoint, a gradient, the logits.  Only the first and last rows and columns are
worked out beside them."""
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS, COLS = 66_001, 65_568          # 4.33e9 values
NEED = 60 << 30


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < NEED:
        pytest.skip("needs 60 GB of device memory")
    yield
    torch.cuda.empty_cache()


def test_a_checkpoint_of_more_than_32_bits():
    g = torch.Generator(device=DEV).manual_seed(0)
    x = torch.zeros(ROWS, COLS, dtype=torch.bfloat16, device=DEV)
    x.random_(-7, 8, generator=g)
    c = dgs.Checkpoint(ROWS, COLS, device=DEV)
    assert c.save(x, "relu", out=x) is x                 # in place; what is held is x before
    held = c.load(torch.bfloat16)
    ends = torch.tensor([0, 1, 32_750, ROWS - 2, ROWS - 1], device=DEV)
    assert torch.equal(x[ends], held[ends].clamp(min=0)) and bool((held[ends] < 0).any())
    dx = c.activation_grad(x, "relu", out=x)
    assert torch.equal(dx[ends], held[ends].clamp(min=0))
    del x, dx
    dy = torch.zeros(ROWS, 24, dtype=torch.bfloat16, device=DEV)
    dy.random_(-3, 4, generator=g)
    dw = torch.zeros(24 * COLS, device=DEV)
    c.weight_grad(dy, dw)
    cols = torch.tensor([0, 1, 40_000, COLS - 1], device=DEV)
    want = dy.double().T @ held[:, cols].double()        # whole numbers below 2^24: exact
    assert torch.equal(dw.view(24, COLS)[:, cols].double(), want)
    assert dgs.operator_status(DEV) == 0


@pytest.mark.parametrize("cols", [COLS, COLS - 1])       # read as it is, and brought onto 16 bytes first
def test_a_gradient_of_more_than_32_bits(cols):
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randint(-7, 8, (ROWS, 32), generator=g, device=DEV).float()
    c = dgs.Checkpoint(ROWS, 32, device=DEV)
    c.save(x)
    dy = torch.zeros(ROWS, cols, dtype=torch.bfloat16, device=DEV)
    dy.random_(-3, 4, generator=g)
    dw, db = torch.zeros(cols * 32, device=DEV), torch.zeros(cols, device=DEV)
    c.weight_grad(dy, dw, db)
    at = torch.tensor([0, 7, 33_333, cols - 1], device=DEV)
    part = dy[:, at].double()
    assert torch.equal(dw.view(cols, 32)[at].double(), part.T @ x.double()) and torch.equal(db[at].double(), part.sum(0))
    assert dgs.operator_status(DEV) == 0


def test_logits_of_more_than_32_bits():
    tokens, experts = 4_200_001, 1024
    z = torch.zeros(tokens, experts, dtype=torch.bfloat16, device=DEV)
    z.normal_()
    r = dgs.route_experts(z, 1)
    ends = torch.tensor([0, 1, 2_100_000, tokens - 1], device=DEV)
    best = z[ends].float()
    first = (best == best.amax(1, keepdim=True)).int().argmax(1)      # the lowest index of the largest
    assert torch.equal(r.expert[ends, 0].long(), first)
    assert int(r.offsets[-1]) == tokens
    assert torch.equal(r.order[r.place[ends, 0].long()].long(), ends)
    dw = torch.zeros(tokens, 1, device=DEV)
    dw[-1] = 1.0
    dz = dgs.route_experts_grad(z, r.expert, dw, renormalise=False, out=z)
    assert float(dz[-1].float().abs().sum()) > 0 and not bool(dz[-2].any())
