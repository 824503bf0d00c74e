"""What the operators of a worker's own computation refuse, and how they size things: no GPU needed.  Device pointers are made up; every refusal comes
before they are used."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_1910_10929_b200 as dgs
from _held import encode

P = 1 << 20          # an address, aligned to anything
NEED = 1 << 30


def matrix(rows=10, cols=64, stride=None, kind=dgs.DGS_TYPE_F32, data=P):
    return dgs.dgs_matrix(data, rows, cols if stride is None else stride, cols, kind)


def held(rows=10, cols=64, fmt=0, data=P << 4):
    return dgs.dgs_checkpoint(data, rows, cols, fmt)


def router(**kw):
    base = dict(k=2, score=0, groups=1, groups_kept=1, group_best=1, renormalise=1, scale=1.0)
    base.update(kw)
    return dgs.dgs_router(**base)


def test_sizes():
    assert dgs.dgs_checkpoint_bytes(0, 5) == 0
    for rows, cols in ((1, 1), (3, 32), (5, 33), (7, 128), (2, 129), (11, 2048)):
        buffer, _ = encode(np.zeros((rows, cols)), "int8")
        assert dgs.dgs_checkpoint_bytes(rows, cols) == len(buffer)
    assert dgs.dgs_checkpoint_bytes((1 << 31) - 1, 100) == ((1 << 31) - 1) * 132          # far past 32 bits
    for rows, cols in ((1, 0), (1, (1 << 30) + 1), (1 << 31, 1), ((1 << 31) - 1, 1 << 10)):
        with pytest.raises(dgs.DgsError) as e:
            dgs.dgs_checkpoint_bytes(rows, cols)
        assert e.value.code == dgs.DGS_EINVAL
    assert dgs.dgs_route_experts_bytes(router(), 0, 8) == 0
    assert dgs.dgs_route_experts_bytes(router(), 64, 8) == 0 and dgs.dgs_route_experts_bytes(router(), 65, 8) == 9 * 3 * 4
    assert dgs.lib().dgs_checkpoint_bytes(1, 1, None) == dgs.DGS_EINVAL


BAD_MATRICES = [dict(rows=9), dict(cols=63), dict(stride=63), dict(kind=3), dict(data=P + 2), dict(data=0), dict(rows=1 << 31),
                dict(stride=1 << 45)]


@pytest.mark.parametrize("bad", BAD_MATRICES)
def test_matrices_that_do_not_fit(bad):
    L, c, m = dgs.lib(), held(), matrix(**bad)
    assert L.dgs_checkpoint_save(c, m, 0, None, None) == dgs.DGS_EINVAL
    assert L.dgs_checkpoint_load(c, m, None) == dgs.DGS_EINVAL
    assert L.dgs_checkpoint_activation_grad(c, 1, m, matrix(data=P * 3), None) == dgs.DGS_EINVAL
    assert L.dgs_checkpoint_activation_grad(c, 1, matrix(data=P * 3), m, None) == dgs.DGS_EINVAL


def test_checkpoint_refusals():
    L, ok = dgs.lib(), matrix()
    for c in (held(fmt=2), held(data=0), held(data=P + 8), held(cols=0), None):
        assert L.dgs_checkpoint_save(c, ok, 0, None, None) == dgs.DGS_EINVAL
        assert L.dgs_checkpoint_load(c, ok, None) == dgs.DGS_EINVAL
        assert L.dgs_checkpoint_weight_grad(c, ok, None, P * 5, None, 0, None, 0, None) == dgs.DGS_EINVAL
    c = held()
    assert L.dgs_checkpoint_save(c, None, 0, None, None) == dgs.DGS_EINVAL
    for act in (-1, 5):
        assert L.dgs_checkpoint_save(c, ok, act, None, None) == dgs.DGS_EINVAL
        assert L.dgs_checkpoint_activation_grad(c, act, ok, ok, None) == dgs.DGS_EINVAL
    # overlaps: the checkpoint with a matrix, input with output a little apart, an output whose rows are one row
    assert L.dgs_checkpoint_save(c, matrix(data=(P << 4) + 64), 0, None, None) == dgs.DGS_EINVAL
    assert L.dgs_checkpoint_save(c, ok, 1, matrix(data=P + 4), None) == dgs.DGS_EINVAL
    assert L.dgs_checkpoint_save(c, ok, 1, matrix(data=P, stride=65), None) == dgs.DGS_EINVAL
    assert L.dgs_checkpoint_save(c, ok, 1, matrix(data=P * 3, kind=1), None) == dgs.DGS_EINVAL
    assert L.dgs_checkpoint_load(c, matrix(stride=0), None) == dgs.DGS_EINVAL
    assert L.dgs_checkpoint_activation_grad(c, 1, ok, matrix(data=P + 256), None) == dgs.DGS_EINVAL
    # nothing to do is no error, wherever the pointers point
    assert L.dgs_checkpoint_save(held(rows=0, data=0), matrix(rows=0, data=0), 0, None, None) == dgs.DGS_OK
    assert L.dgs_checkpoint_load(held(rows=0, data=0), matrix(rows=0, data=0), None) == dgs.DGS_OK


def test_weight_grad_refusals():
    L, c, dy = dgs.lib(), held(), matrix()
    call = lambda c=c, dy=dy, lists=None, dw=P * 5, db=None, flags=0, work=P << 12, size=NEED: L.dgs_checkpoint_weight_grad(   # noqa: E731
        c, dy, lists, dw, db, flags, work, size, None)
    assert call(dw=None) == dgs.DGS_EINVAL and call(dw=P * 5 + 2) == dgs.DGS_EINVAL and call(db=P * 6 + 1) == dgs.DGS_EINVAL
    assert call(flags=4) == dgs.DGS_EINVAL
    assert call(dy=matrix(rows=9)) == dgs.DGS_EINVAL
    assert call(dw=P) == dgs.DGS_EINVAL                        # over dy
    assert call(dw=P << 4) == dgs.DGS_EINVAL                   # over the checkpoint
    assert call(db=P * 5 + 64) == dgs.DGS_EINVAL               # over dw
    for lists in (dgs.dgs_row_lists(None, None, 2, 1), dgs.dgs_row_lists(P * 9, None, 0, 1), dgs.dgs_row_lists(P * 9, None, 2, 0),
                  dgs.dgs_row_lists(P * 9, P * 9 + 2, 2, 1), dgs.dgs_row_lists(P * 9, None, 1025, 1)):
        assert call(lists=lists) == dgs.DGS_EINVAL
    big, long = held(rows=100_000), matrix(rows=100_000)       # split: needs a workspace
    need = dgs.dgs_checkpoint_weight_grad_bytes(big, long)
    assert need > 0 and dgs.dgs_checkpoint_weight_grad_bytes(c, dy) == 0      # few rows: none
    assert call(big, long, dw=P << 8, work=P << 12, size=need - 1) == dgs.DGS_ENOMEM
    assert call(big, long, dw=P << 8, work=None, size=need) == dgs.DGS_EINVAL
    assert call(big, long, dw=P << 8, work=(P << 12) + 4, size=need) == dgs.DGS_EINVAL
    assert call(big, long, dw=P << 8, work=P << 8, size=need) == dgs.DGS_EINVAL
    out = C.c_uint64(0)
    huge = dgs.dgs_matrix(P, 10, 1 << 29, 1 << 29, 0)
    assert L.dgs_checkpoint_weight_grad_bytes(held(cols=1 << 29), huge, None, 0, C.byref(out)) == dgs.DGS_ELIMIT


@pytest.mark.parametrize("bad", [dict(k=0), dict(k=33), dict(k=65), dict(score=2), dict(groups=0), dict(groups=3), dict(groups=4, groups_kept=0),
                                 dict(groups=4, groups_kept=5), dict(group_best=0), dict(group_best=3), dict(renormalise=2),
                                 dict(scale=float("nan")), dict(scale=float("inf")), dict(groups=64, groups_kept=1, k=2)])
def test_routers_that_are_refused(bad):
    L, out = dgs.lib(), C.c_uint64(0)
    r, z = router(**bad), matrix()
    assert L.dgs_route_experts_bytes(r, 10, 64, C.byref(out)) == dgs.DGS_EINVAL
    assert L.dgs_route_experts(r, z, None, P * 3, P * 4, None, None, None, None, 0, None) == dgs.DGS_EINVAL
    assert L.dgs_route_experts_grad(r, z, P * 3, P * 4, matrix(data=P * 5), None) == dgs.DGS_EINVAL


def test_route_refusals():
    L, r, z = dgs.lib(), router(), matrix(rows=100)
    out = C.c_uint64(0)
    assert L.dgs_route_experts_bytes(r, 1 << 31, 64, C.byref(out)) == dgs.DGS_ELIMIT
    assert L.dgs_route_experts_bytes(r, 10, 1025, C.byref(out)) == dgs.DGS_EINVAL
    call = lambda z=z, bias=None, e=P * 3, w=P * 4, of=P * 5, o=P * 6, p=P * 7, ws=P * 8, n=NEED: L.dgs_route_experts(   # noqa: E731
        r, z, bias, e, w, of, o, p, ws, n, None)
    assert call(e=None) == dgs.DGS_EINVAL and call(w=None) == dgs.DGS_EINVAL and call(o=None) == dgs.DGS_EINVAL
    assert call(of=None) == dgs.DGS_EINVAL and call(p=None) == dgs.DGS_EINVAL and call(ws=None) == dgs.DGS_EINVAL
    assert call(n=65 * 3 * 4 - 1) == dgs.DGS_ENOMEM and call(ws=P * 8 + 4) == dgs.DGS_EINVAL
    assert call(e=P * 3 + 1) == dgs.DGS_EINVAL and call(bias=P * 9 + 2) == dgs.DGS_EINVAL
    assert call(w=P * 3) == dgs.DGS_EINVAL and call(e=P) == dgs.DGS_EINVAL and call(bias=P * 5) == dgs.DGS_EINVAL
    assert call(z=matrix(rows=100, cols=1025)) == dgs.DGS_EINVAL
    g = lambda z=z, e=P * 3, w=P * 4, dz=None: L.dgs_route_experts_grad(r, z, e, w, dz or matrix(rows=100, data=P * 5), None)   # noqa: E731
    assert g(e=None) == dgs.DGS_EINVAL and g(w=None) == dgs.DGS_EINVAL
    assert g(dz=matrix(rows=100, data=P * 5, cols=63)) == dgs.DGS_EINVAL and g(dz=matrix(rows=100, data=P * 5, kind=1)) == dgs.DGS_EINVAL
    assert g(dz=matrix(rows=100, data=P + 4)) == dgs.DGS_EINVAL and g(dz=matrix(rows=100, data=P * 3)) == dgs.DGS_EINVAL
    assert g(dz=matrix(rows=100, data=P * 5, stride=0)) == dgs.DGS_EINVAL


def test_torch_calls_refuse_what_is_not_on_a_gpu_or_not_known():
    x = torch.zeros(4, 8)
    for call in (lambda: dgs.route_experts(x, 2), lambda: dgs.route_experts_grad(x, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)),
                 lambda: dgs.Checkpoint(4, 8, data=torch.zeros(160, dtype=torch.uint8)), lambda: dgs.Checkpoint(4, 8, "int4"),
                 lambda: dgs.Checkpoint(-1, 8), lambda: dgs.Checkpoint(4, 0)):
        with pytest.raises(ValueError):
            call()
    assert dgs.lib().dgs_operator_status(None, None) == dgs.DGS_EINVAL


def test_the_numpy_format_is_its_definition():
    """The restatement that the GPU tests go by, on values worked out by hand."""
    x = np.zeros((1, 33), np.float32)
    x[0, :6] = [127.0, -63.5, 0.5, 1.5, -0.5, 2.49]      # e = 0: ties to even
    x[0, 32] = 127.5                                     # e = 1
    buffer, values = encode(x, "int8")
    assert values[0, :6].tolist() == [127, -64, 0, 2, 0, 2] and values[0, 32] == 128.0
    assert buffer[64:68].tolist() == [127, 128, 0, 0] and buffer[1] == 256 - 64
    buffer, values = encode(np.array([[448.0, 0.001, 17.0, 18.0, 19.0]]), "e4m3")
    assert values[0].tolist() == [448.0, 2.0 ** -9 * 1, 16.0, 18.0, 20.0] and buffer[0] == 0x7E
