"""What the calls that move rows to the experts' lists and back refuse: no GPU needed.  Device pointers are made up; every refusal comes before they are used."""
import pytest
import torch

import paper_1910_10929_b200 as dgs
from paper_1910_10929_b200 import operators

P = 1 << 24
BAD = dgs.DGS_EINVAL


def matrix(rows=10, cols=64, stride=None, kind=dgs.DGS_TYPE_F32, data=P):
    return dgs.dgs_matrix(data, rows, cols if stride is None else stride, cols, kind)


def many(**kw):
    return matrix(**{"rows": 20, "data": 2 * P, **kw})


BAD_ALL = [dict(rows=19), dict(rows=21), dict(cols=63), dict(stride=63), dict(kind=1), dict(kind=3), dict(data=2 * P + 2), dict(data=0), dict(rows=1 << 31), dict(stride=1 << 45)]


@pytest.mark.parametrize("bad", BAD_ALL)
def test_matrices_that_do_not_fit(bad):
    L, o, p, w = dgs.lib(), 3 * P, 4 * P, 5 * P
    assert L.dgs_experts_gather(matrix(), o, p, 2, many(**bad), None) == BAD
    assert L.dgs_experts_combine(many(**bad), w, p, 2, matrix(), None) == BAD
    assert L.dgs_experts_combine_grad(matrix(), many(**bad), w, o, p, 2, many(data=6 * P), 7 * P, None) == BAD
    assert L.dgs_experts_combine_grad(matrix(), many(), w, o, p, 2, many(**{"data": 6 * P, **bad}), 7 * P, None) == BAD


def test_other_refusals():
    L, o, p, w, d = dgs.lib(), 3 * P, 4 * P, 5 * P, 7 * P
    for k in (0, 33, 1 << 31):
        assert L.dgs_experts_gather(matrix(), o, p, k, matrix(rows=10 * k % (1 << 31), data=2 * P), None) == BAD
        assert L.dgs_experts_combine(matrix(rows=10 * k % (1 << 31), data=2 * P), w, p, k, matrix(), None) == BAD
    gather = lambda x=matrix(), o=o, p=p, y=many(): L.dgs_experts_gather(x, o, p, 2, y, None)   # noqa: E731
    combine = lambda y=many(), w=w, p=p, out=matrix(): L.dgs_experts_combine(y, w, p, 2, out, None)   # noqa: E731
    grad = lambda g=matrix(), y=many(), w=w, o=o, p=p, dy=many(data=6 * P), d=d: L.dgs_experts_combine_grad(g, y, w, o, p, 2, dy, d, None)   # noqa: E731
    assert gather(o=None) == BAD and gather(p=None) == BAD and gather(o=o + 2) == BAD and gather(p=p + 1) == BAD and gather(x=None) == BAD and gather(y=None) == BAD
    assert combine(p=None) == BAD and combine(w=w + 2) == BAD and combine(p=p + 2) == BAD and combine(y=None) == BAD and combine(out=None) == BAD
    assert grad(g=None) == BAD and grad(y=None) == BAD and grad(w=None) == BAD and grad(o=None) == BAD and grad(p=None) == BAD and grad(dy=None) == BAD and grad(d=None) == BAD
    assert grad(w=w + 2) == BAD and grad(d=d + 2) == BAD
    # outputs over inputs or each other; an output whose rows are one row
    assert gather(y=many(data=P + 64)) == BAD and gather(y=many(data=o)) == BAD and gather(y=many(data=p)) == BAD and gather(y=many(stride=0)) == BAD
    assert combine(out=matrix(data=2 * P + 64)) == BAD and combine(out=matrix(data=w)) == BAD and combine(out=matrix(data=p)) == BAD
    assert grad(dy=many(data=2 * P)) == BAD and grad(dy=many(data=P)) == BAD and grad(dy=many(data=w)) == BAD and grad(d=w) == BAD and grad(d=6 * P + 16) == BAD and grad(d=o) == BAD
    # slots past 31 bits
    wide = matrix(rows=(1 << 31) - 1, stride=0)
    assert L.dgs_experts_gather(wide, o, p, 2, many(rows=(1 << 31) - 1), None) == BAD
    # nothing to do is no error, wherever the pointers point
    none = matrix(rows=0, data=0)
    assert gather(x=none, o=None, p=None, y=none) == combine(y=none, w=None, p=None, out=none) == dgs.DGS_OK
    assert grad(g=none, y=none, w=None, o=None, p=None, dy=none, d=None) == dgs.DGS_OK


def test_torch_calls_refuse_what_does_not_fit(monkeypatch):
    x, y, order, place, w = torch.zeros(4, 8), torch.zeros(8, 8), torch.zeros(8, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    calls = [lambda x=x, y=y, o=order, p=place, w=w: dgs.gather_experts(x, o, p), lambda x=x, y=y, o=order, p=place, w=w: dgs.gather_experts_grad(y, p),
             lambda x=x, y=y, o=order, p=place, w=w: dgs.combine_experts(y, w, p), lambda x=x, y=y, o=order, p=place, w=w: dgs.combine_experts_grad(x, y, w, o, p)]
    for call in calls:                                     # not on a GPU
        with pytest.raises(ValueError, match="CUDA"):
            call()
    monkeypatch.setattr(operators, "_on_gpu", lambda t, what: None)
    monkeypatch.setattr(operators, "_run", lambda *a: pytest.fail("enqueued"))
    for bad in (dict(p=place.long()), dict(p=place[:, :1]), dict(p=place[:3]), dict(p=torch.zeros(4, 33, dtype=torch.int32)), dict(p=torch.zeros(4, 0, dtype=torch.int32)),
                dict(p=torch.zeros(2, 4, dtype=torch.int32).T), dict(p=torch.zeros((), dtype=torch.int32)), dict(p=None)):
        for call in calls:
            if bad.get("p") is not None and bad["p"].shape == (4, 1) and call is calls[1]:
                continue                                   # eight rows, one slot each: another call
            with pytest.raises(ValueError):
                call(**bad)
    for call, bad in ((calls[0], dict(o=order[:7])), (calls[0], dict(o=order.long())), (calls[2], dict(w=w.double())), (calls[2], dict(w=w[:3])), (calls[1], dict(y=y[:7])),
                      (calls[3], dict(y=y[:6])), (calls[3], dict(y=y.half())), (calls[3], dict(y=y[:, :7])), (calls[3], dict(w=w.half())), (calls[3], dict(o=order[:1]))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ValueError):
        dgs.gather_experts(x, order, place, out=torch.zeros(8, 9))
    with pytest.raises(ValueError):
        dgs.combine_experts(y, w, place, out=torch.zeros(4, 8, dtype=torch.float16))
