"""The loss over a vocabulary and its gradient against plain 64-bit arithmetic, at the sizes, types, alignments, targets and magnitudes where they can go wrong.

Tolerances.  A sum of K products in the tensor cores passes through K / 16 additions that cut bits off (taken as 2^-22 of the sum of magnitudes each), is rounded
into a register every 512, and its parts are at most two numbers: cut(K).  What that does to a logit, the exponential of the hardware (2^-22), its argument
(2^-22 of it) and 22 bits of s are followed through the formulas, element by element.  An fp16 number is off by half a step, 2^-11; two of them by 2^-22, and the
product of two second parts, which is left out, is at most 2^-22 of the whole: 3 * 2^-22 for a product of f32 values, 2 * 2^-22 where s has its own share."""
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [(1, 1, 1), (1, 1, 2), (1, 64, 256), (2, 7, 5), (5, 16, 300), (64, 72, 128), (127, 65, 129), (128, 128, 256), (129, 130, 257), (256, 256, 512),
         (257, 31, 1000), (300, 768, 511), (513, 40, 2049), (700, 264, 777), (33, 1025, 640)]


def cut(k):
    return (min(k / 16, 64) + 4 + k / 512) * 2.0 ** -22


def strided(t, pad, offset):
    whole = torch.full((offset + t.shape[0] * (t.shape[1] + pad) + 1,), float("nan"), dtype=t.dtype, device=DEV)
    v = whole.as_strided(t.shape, (t.shape[1] + pad, 1), offset)
    v.copy_(t)
    return v, whole


def problem(rows, width, words, dtype, seed, ignored=0.2, kind=torch.int64, by=1.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    table = (torch.randn(words, width, generator=g, device=DEV) * (by / width ** 0.5)).to(dtype)
    target = torch.randint(0, words, (rows,), generator=g, device=DEV)
    sure = torch.rand(rows, 1, generator=g, device=DEV) * 8
    near = table[target].float()
    hidden = (torch.randn(rows, width, generator=g, device=DEV) + sure * near / near.norm(dim=1, keepdim=True).clamp(min=1e-6)).to(dtype)
    target = target.masked_fill(torch.rand(rows, generator=g, device=DEV) < ignored, -100).to(kind)
    return hidden, table, target, torch.rand(rows, generator=g, device=DEV) / rows


def logits(hidden, table):
    """z in 64 bits, and how far off the kernels' may be."""
    z, size = hidden.double() @ table.double().T, hidden.double().abs() @ table.double().abs().T
    return z, size * (cut(hidden.shape[1]) + (3 * 2.0 ** -22 if hidden.dtype == torch.float32 else 0.0))


def check_loss(hidden, table, target, got):
    z, dz = logits(hidden, table)
    lse = torch.logsumexp(z, 1)
    most = z.amax(1)
    # a part's sum of 128 exponentials, then the parts: each rounding 2^-24 of the sum, exponentials 2^-22 and 2^-22 of their argument (as far as they count)
    far = dz.amax(1) + (128 + 24 + table.shape[0] / 1024 + 8) * 2.0 ** -24 + 3 * 2.0 ** -22 + lse.abs() * 2.0 ** -23 + most.abs() * 2.0 ** -23
    assert got.loss.dtype == got.lse.dtype == torch.float32 and got.loss.shape == got.lse.shape == target.shape
    assert bool(((got.lse.double() - lse).abs() <= far).all())
    live = target >= 0
    want = torch.where(live, lse - z.gather(1, target.long().clamp(min=0)[:, None])[:, 0], 0.0)
    assert bool(((got.loss.double() - want).abs() <= far * 2 + want.abs() * 2.0 ** -23).all()) and bool((got.loss[~live] == 0).all())


def check_grad(hidden, table, target, lse, dloss, dhidden, dw, before=None):
    dtype, eps = hidden.dtype, torch.finfo(hidden.dtype).eps
    h, w, live = hidden.double(), table.double(), target >= 0
    h = torch.where(live[:, None], h, 0.0)                       # ignored rows take no part, whatever they hold
    g = torch.where(live, dloss.double().expand(h.shape[0]), 0.0)[:, None]
    z, dz = logits(h.to(dtype), table)
    x = z - torch.where(live, lse.double(), z.amax(1))[:, None]
    p = torch.exp(x)
    y = torch.zeros_like(p)
    y[live] = y[live].scatter_(1, target.long()[live][:, None], 1.0)
    s = g * (p - y)
    most = float(g.abs().max())
    parts = 2.0 ** -21 if dtype == torch.float32 else 2.0 ** -23
    ds = g.abs() * (p * (1.1 * dz + x.abs() * 2.0 ** -22 + 3 * 2.0 ** -22) + y * 2.0 ** -23) + s.abs() * 2.0 ** -21 + most * 2.0 ** -38
    tiny = torch.finfo(torch.float32).smallest_normal
    small = torch.finfo(dtype).smallest_normal * eps
    if dw is not None:
        want = s.T @ h
        near = ds.T @ h.abs() + (s.abs().T @ h.abs()) * (cut(2 * h.shape[0]) + parts) + want.abs() * 3 * 2.0 ** -24 + tiny
        if before is not None:
            want = want + before.double()
            near += want.abs() * 2.0 ** -24 + before.double().abs() * 2.0 ** -24
        assert bool(((dw.double() - want).abs() <= near).all())
    want = s @ w
    if dtype == torch.bfloat16:
        ds = ds + s.abs() * 2.0 ** -11 + most * 2.0 ** -38             # s is one fp16 number there, off by half a step of 2^-10
    near = ds @ w.abs() + (s.abs() @ w.abs()) * (cut(2 * w.shape[0]) + parts) + want.abs() * (eps / 2) * (1 + 2.0 ** -8) + small
    assert bool(((dhidden.double() - want).abs() <= near).all()) and not bool(dhidden[~live].any())


def grad(hidden, table, target, lse, dloss, before=None, pad=0, offset=0, want_dw=True):
    """vocabulary_loss_grad into guarded memory at an odd offset."""
    n = table.numel()
    flat = torch.full((3 + n,), float("nan"), device=DEV)
    dw = flat[1:1 + n] if want_dw else None
    if before is not None:
        dw.copy_(before.reshape(-1))
    out, whole = strided(torch.zeros_like(hidden), pad, offset)
    got = dgs.vocabulary_loss_grad(hidden, table, target, lse, dloss, dw, add=before is not None, out=out)
    assert got is out and dgs.operator_status(DEV) == 0
    assert int(torch.isnan(whole).sum()) == whole.numel() - out.numel() + int(torch.isnan(out).sum())
    assert bool(torch.isnan(flat[0])) and bool(torch.isnan(flat[1 + n:]).all())
    return out, dw.view(table.shape) if want_dw else None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,words", SIZES)
def test_loss(rows, width, words, dtype):
    for pad, offset, kind, ignored in ((0, 0, torch.int64, 0.2), (8, 8, torch.int32, 0.0), (1, 3, torch.int64, 1.0)):
        hidden, table, target, _ = problem(rows, width, words, dtype, rows + words + pad, ignored, kind)
        h, w = strided(hidden, pad, offset)[0], strided(table, pad, offset)[0]
        got = dgs.vocabulary_loss(h, w, target)
        assert dgs.operator_status(DEV) == 0
        check_loss(hidden, table, target, got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,words", SIZES)
def test_gradient(rows, width, words, dtype):
    for pad, offset, kind, ignored, each in ((0, 0, torch.int64, 0.2, True), (8, 8, torch.int32, 0.0, False), (1, 3, torch.int64, 0.5, True)):
        hidden, table, target, dloss = problem(rows, width, words, dtype, rows + words + pad, ignored, kind)
        lse = torch.logsumexp(hidden.double() @ table.double().T, 1).float()
        h, w = strided(hidden, pad, offset)[0], strided(table, pad, offset)[0]
        dloss = dloss if each else dloss[:1].clone()
        before = None if pad == 8 else torch.randn(words, width, device=DEV) / rows
        dh, dw = grad(h, w, target, lse, dloss, before, pad, offset)
        check_grad(hidden, table, target, lse, dloss, dh, dw, before)
        alone, _ = grad(h, w, target, lse, dloss, pad=pad, offset=offset, want_dw=False)
        assert torch.equal(alone, dh)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,words", [(20_000, 40, 300), (3, 96, 50_257), (1, 768, 50_257), (8192, 64, 20_000), (9000, 300, 5000), (70_000, 8, 700), (300, 2056, 4100)])
def test_long_sums_pieces_and_splits(rows, width, words, dtype):
    hidden, table, target, dloss = problem(rows, width, words, dtype, 5)
    got = dgs.vocabulary_loss(hidden, table, target)
    check_loss(hidden, table, target, got)
    dh, dw = grad(hidden, table, target, got.lse, dloss)
    check_grad(hidden, table, target, got.lse, dloss, dh, dw)
