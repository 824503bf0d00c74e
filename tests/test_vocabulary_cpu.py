"""What the loss over a vocabulary and its gradient refuse, and how they size things: no GPU needed.  Device pointers are made up; every refusal comes before
they are used."""
import ctypes as C

import pytest
import torch

import paper_1910_10929_b200 as dgs
from paper_1910_10929_b200 import operators

P = 1 << 36
NEED = 1 << 35
BAD = dgs.DGS_EINVAL


def matrix(rows=100, cols=64, stride=None, kind=dgs.DGS_TYPE_BF16, data=P):
    return dgs.dgs_matrix(data, rows, cols if stride is None else stride, cols, kind)


def words(**kw):
    return matrix(**{"rows": 5000, "data": 2 * P, **kw})


def loss(h=None, w=None, t=3 * P, flags=1, a=4 * P, b=5 * P, work=6 * P, size=NEED):
    return dgs.lib().dgs_vocabulary_loss(h or matrix(), w or words(), t, flags, a, b, work, size, None)


def grad(h=None, w=None, t=3 * P, lse=4 * P, g=5 * P, step=1, dh=None, dw=8 * P, flags=1, work=6 * P, size=NEED):
    return dgs.lib().dgs_vocabulary_loss_grad(h or matrix(), w or words(), t, lse, g, step, dh or matrix(data=7 * P), dw, flags, work, size, None)


@pytest.mark.parametrize("bad", [dict(cols=63), dict(stride=63), dict(kind=3), dict(data=P + 1), dict(data=0), dict(rows=1 << 31), dict(stride=1 << 45), dict(kind=0), dict(kind=2)])
def test_matrices_that_do_not_fit(bad):
    out = C.c_uint64(0)
    L, h, w = dgs.lib(), matrix(**bad), words(**{**bad, **({"data": 2 * P + 1} if bad.get("data") == P + 1 else {})})
    assert L.dgs_vocabulary_loss_bytes(h, words(), C.byref(out)) == BAD and L.dgs_vocabulary_loss_bytes(matrix(), w, C.byref(out)) == BAD
    assert L.dgs_vocabulary_loss_grad_bytes(h, words(), C.byref(out)) == BAD and L.dgs_vocabulary_loss_grad_bytes(matrix(), w, C.byref(out)) == BAD
    assert loss(h=h) == BAD and loss(w=w) == BAD and grad(h=h) == BAD and grad(w=w) == BAD
    assert grad(dh=matrix(**{"data": 7 * P, **{k: v for k, v in bad.items() if k != "data"}, **({"data": 7 * P + 1 if bad.get("data") else 0} if "data" in bad else {})})) == BAD


def test_other_refusals():
    L = dgs.lib()
    assert L.dgs_vocabulary_loss_bytes(matrix(), words(), None) == BAD and L.dgs_vocabulary_loss_bytes(None, words(), C.byref(C.c_uint64(0))) == BAD
    none = words(rows=0)
    assert loss(w=none) == BAD and grad(w=none) == BAD                      # a vocabulary without words
    assert loss(flags=2) == BAD and loss(flags=4) == BAD and grad(flags=4) == BAD and grad(step=2) == BAD
    for bad in (dict(t=None), dict(t=3 * P + 4), dict(t=3 * P + 2, flags=0), dict(a=None), dict(b=None), dict(a=4 * P + 2), dict(b=5 * P + 1), dict(work=None), dict(work=6 * P + 128)):
        assert loss(**bad) == BAD, bad
    for bad in (dict(t=None), dict(t=3 * P + 4), dict(lse=None), dict(g=None), dict(lse=4 * P + 2), dict(g=5 * P + 2), dict(dw=8 * P + 2), dict(work=None), dict(work=6 * P + 16),
                dict(dh=matrix(rows=99, data=7 * P)), dict(dh=matrix(stride=0, data=7 * P))):
        assert grad(**bad) == BAD, bad
    need = dgs.dgs_vocabulary_loss_bytes(matrix(), words()), dgs.dgs_vocabulary_loss_grad_bytes(matrix(), words())
    assert loss(size=need[0] - 1) == dgs.DGS_ENOMEM and grad(size=need[1] - 1) == dgs.DGS_ENOMEM
    # outputs over inputs or each other
    for at in (P, 2 * P + 640, 3 * P, 5 * P, 6 * P):
        assert loss(a=at) == BAD, at
    for at in (P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 7 * P):
        assert grad(dw=at) == BAD, at
    for at in (P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, 8 * P):
        assert grad(dh=matrix(data=at)) == BAD, at
    assert loss(work=P) == BAD and grad(work=4 * P) == BAD


def test_sizes():
    size = lambda h, w: (dgs.dgs_vocabulary_loss_bytes(h, w), dgs.dgs_vocabulary_loss_grad_bytes(h, w))   # noqa: E731
    assert size(matrix(rows=0, data=0), words()) == (0, 0)
    # GPT-2's head over 8192 rows: the loss takes 8 bytes a row and 64 words; the gradient far less than logits in f32
    h, w = matrix(rows=8192, cols=768), words(rows=50257, cols=768)
    a, b = size(h, w)
    assert 8192 * 8 * 786 <= a <= 8192 * 8 * 788 + 8192 * 4 and b < 500 << 20
    # copies where TMA copies cannot read
    odd = words(rows=50257, cols=768, data=2 * P + 2)
    assert size(h, odd)[0] == a + (50257 * 768 * 2 + 255) // 256 * 256
    assert size(matrix(rows=8192, cols=768, kind=0), words(rows=50257, cols=768, kind=0))[0] > a + (8192 + 50257) * 768 * 4
    for h, w in ((matrix(cols=(1 << 24) + 8), words(cols=(1 << 24) + 8)), (matrix(rows=(1 << 30) + 1, cols=8), words(cols=8)), (matrix(cols=8), words(rows=(1 << 30) + 1, cols=8)),
                 (matrix(cols=1 << 16), words(rows=1 << 23, cols=1 << 16)), (matrix(rows=1 << 28, cols=8), words(rows=1 << 28, cols=8))):
        with pytest.raises(dgs.DgsError) as e:
            dgs.dgs_vocabulary_loss_bytes(h, w)
        assert e.value.code == dgs.DGS_ELIMIT
    assert grad(h=matrix(rows=0, data=0), t=None, lse=None, g=None, dh=matrix(rows=0, data=0), dw=None, work=None, size=0) == dgs.DGS_OK
    assert loss(h=matrix(rows=0, data=0), t=None, a=None, b=None, work=None, size=0) == dgs.DGS_OK


def test_torch_calls_refuse_what_does_not_fit(monkeypatch):
    h, w, t, lse, g, dw = torch.zeros(4, 8), torch.zeros(10, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(4), torch.zeros(80)
    first = lambda h=h, w=w, t=t: dgs.vocabulary_loss(h, w, t)   # noqa: E731
    second = lambda h=h, w=w, t=t, lse=lse, g=g, dw=dw, **k: dgs.vocabulary_loss_grad(h, w, t, lse, g, dw, **k)   # noqa: E731
    for call in (first, second):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    monkeypatch.setattr(operators, "_on_gpu", lambda t, what: None)
    monkeypatch.setattr(operators, "_run", lambda *a: pytest.fail("enqueued"))
    for call in (first, second):
        for bad in (dict(w=w[:, :7]), dict(w=w.half()), dict(t=t[:3]), dict(t=t.float()), dict(t=t.to(torch.int16)), dict(t=None), dict(t=torch.zeros(8, dtype=torch.int64)[::2]), dict(h=h.double())):
            with pytest.raises(ValueError):
                call(**bad)
    for bad in (dict(lse=lse[:3]), dict(lse=lse.double()), dict(lse=None), dict(g=g[:3]), dict(g=g.half()), dict(g=1.0), dict(g=None), dict(dw=dw[:79]), dict(dw=dw.half()),
                dict(out=torch.zeros(4, 9)), dict(out=torch.zeros(3, 8)), dict(out=torch.zeros(4, 8, dtype=torch.float16))):
        with pytest.raises(ValueError):
            second(**bad)
