"""The bindings by the library's own names, for rows to the experts and back and the vocabulary's loss: the torch-backed calls' results."""
import pytest
import torch

import paper_1910_10929_b200 as dgs
from test_experts_gpu import lists
from test_vocabulary_gpu import problem

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KIND = {torch.float32: dgs.DGS_TYPE_F32, torch.bfloat16: dgs.DGS_TYPE_BF16, torch.float16: dgs.DGS_TYPE_FP16}


def matrix(t):
    return dgs.dgs_matrix(t.data_ptr(), t.shape[0], t.stride(0), t.shape[1], KIND[t.dtype])


@pytest.mark.parametrize("dtype", list(KIND))
def test_rows_to_the_experts_and_back(dtype):
    g = torch.Generator(device=DEV).manual_seed(1)
    order, place = lists(50, 3, 7, 1, 0.2)
    x, dout = (torch.randn(50, 72, generator=g, device=DEV).to(dtype) for _ in range(2))
    weight = torch.rand(50, 3, generator=g, device=DEV)
    stream = torch.cuda.current_stream(DEV).cuda_stream
    y, out, dx, dy = torch.empty(150, 72, dtype=dtype, device=DEV), torch.empty_like(x), torch.empty_like(x), torch.empty(150, 72, dtype=dtype, device=DEV)
    dweight = torch.empty(50, 3, device=DEV)
    dgs.dgs_experts_gather(matrix(x), order.data_ptr(), place.data_ptr(), 3, matrix(y), stream)
    dgs.dgs_experts_combine(matrix(y), weight.data_ptr(), place.data_ptr(), 3, matrix(out), stream)
    dgs.dgs_experts_combine_grad(matrix(dout), matrix(y), weight.data_ptr(), order.data_ptr(), place.data_ptr(), 3, matrix(dy), dweight.data_ptr(), stream)
    dgs.dgs_experts_combine(matrix(dy), 0, place.data_ptr(), 3, matrix(dx), stream)
    assert torch.equal(y, dgs.gather_experts(x, order, place)) and torch.equal(out, dgs.combine_experts(y, weight, place))
    a, b = dgs.combine_experts_grad(dout, y, weight, order, place)
    assert torch.equal(dy, a) and torch.equal(dweight, b) and torch.equal(dx, dgs.gather_experts_grad(dy, place))
    with pytest.raises(dgs.DgsError) as e:
        dgs.dgs_experts_gather(matrix(x), order.data_ptr(), place.data_ptr(), 2, matrix(y), stream)
    assert e.value.code == dgs.DGS_EINVAL and "dgs_experts_gather" in str(e.value)


@pytest.mark.parametrize("dtype", list(KIND))
@pytest.mark.parametrize("rows,words", [(20, 300), (300, 2000)])
def test_the_vocabularys_loss(rows, words, dtype):
    hidden, table, target, dloss = problem(rows, 40, words, dtype, 61)
    stream = torch.cuda.current_stream(DEV).cuda_stream
    h, w = matrix(hidden), matrix(table)
    loss, lse, dw, dh = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.ones(words * 40, device=DEV), torch.empty_like(hidden)
    need = dgs.dgs_vocabulary_loss_bytes(h, w), dgs.dgs_vocabulary_loss_grad_bytes(h, w)
    work = torch.empty(max(need), dtype=torch.uint8, device=DEV)
    dgs.dgs_vocabulary_loss(h, w, target.data_ptr(), dgs.DGS_TARGET_I64, loss.data_ptr(), lse.data_ptr(), work.data_ptr(), need[0], stream)
    dgs.dgs_vocabulary_loss_grad(h, w, target.data_ptr(), lse.data_ptr(), dloss.data_ptr(), 1, matrix(dh), dw.data_ptr(), dgs.DGS_TARGET_I64 | dgs.DGS_LOSS_ADD,
                                 work.data_ptr(), need[1], stream)
    got = dgs.vocabulary_loss(hidden, table, target)
    again = torch.ones(words * 40, device=DEV)
    assert torch.equal(loss, got.loss) and torch.equal(lse, got.lse)
    assert torch.equal(dh, dgs.vocabulary_loss_grad(hidden, table, target, lse, dloss, again, add=True)) and torch.equal(dw, again)
    for call in (lambda: dgs.dgs_vocabulary_loss(h, w, target.data_ptr(), 4, loss.data_ptr(), lse.data_ptr(), work.data_ptr(), need[0], stream),
                 lambda: dgs.dgs_vocabulary_loss_grad(h, w, target.data_ptr(), lse.data_ptr(), dloss.data_ptr(), 2, matrix(dh), 0, 1, work.data_ptr(), need[1], stream)):
        with pytest.raises(dgs.DgsError) as e:
            call()
        assert e.value.code == dgs.DGS_EINVAL
    assert dgs.operator_status(DEV) == 0
