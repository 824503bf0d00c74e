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
    before = torch.randn(words, width, device=DEV) / rows         # what an earlier part of the batch has left
    again, added = grad(hidden, table, target, got.lse, dloss, before)
    assert torch.equal(again, dh)
    check_grad(hidden, table, target, got.lse, dloss, again, added, before)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,width,words", [(40, 64, 300), (300, 64, 3000)])        # without tensor cores and with them
def test_ignored_rows_take_no_part_whatever_they_hold(rows, width, words, dtype):
    hidden, table, target, dloss = problem(rows, width, words, dtype, 9, ignored=0.3)
    clean = dgs.vocabulary_loss(hidden, table, target)
    dirty, live = hidden.clone(), target >= 0
    dirty[~live] = torch.tensor([float("nan"), float("inf"), float("-inf")], device=DEV).to(dtype)[torch.arange(int((~live).sum()), device=DEV) % 3][:, None]
    got = dgs.vocabulary_loss(dirty, table, target)
    assert torch.equal(got.loss, clean.loss) and torch.equal(got.lse[live], clean.lse[live])
    bad = dloss.masked_fill(~live, float("nan"))
    a, b = grad(hidden, table, target, clean.lse, dloss), grad(dirty, table, target, got.lse, bad)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and not bool(b[0][~live].any())
    # nothing but ignored rows
    none = torch.full_like(target, -1)
    assert not dgs.vocabulary_loss(dirty, table, none).loss.any()
    dh, dw = grad(dirty, table, none, got.lse, dloss)
    assert not dh.any() and not dw.any()
    before = torch.randn(words, width, device=DEV)
    assert torch.equal(grad(dirty, table, none, got.lse, dloss, before)[1], before)


@pytest.mark.parametrize("rows,width,words", [(40, 64, 300), (300, 64, 3000)])
def test_a_row_that_holds_a_nan_keeps_it_to_itself(rows, width, words):
    hidden, table, target, dloss = problem(rows, width, words, torch.bfloat16, 10, ignored=0.0)
    clean = dgs.vocabulary_loss(hidden, table, target)
    hidden[7, 3] = float("nan")
    got = dgs.vocabulary_loss(hidden, table, target)
    assert bool(torch.isnan(got.loss[7])) and bool(torch.isnan(got.lse[7]))
    others = torch.arange(rows, device=DEV) != 7
    assert torch.equal(got.loss[others], clean.loss[others]) and torch.equal(got.lse[others], clean.lse[others])
    dh, dw = grad(hidden, table, target, got.lse, dloss)
    assert bool(torch.isnan(dh[7]).all()) and not bool(torch.isnan(dh[others]).any()) and bool(torch.isnan(dw).all())


@pytest.mark.parametrize("rows,width,words", [(40, 64, 300), (300, 64, 3000)])
def test_targets_past_the_last_word_are_reported_and_ignored(rows, width, words):
    for kind in (torch.int64, torch.int32):
        hidden, table, target, dloss = problem(rows, width, words, torch.bfloat16, 11, ignored=0.1, kind=kind)
        ignored, bad = target.clone(), target.clone()
        ignored[5], ignored[rows - 1] = -1, -(1 << 31)
        bad[5], bad[rows - 1] = words, (1 << 31) - 1 if kind == torch.int32 else 1 << 40
        a, b = dgs.vocabulary_loss(hidden, table, ignored), dgs.vocabulary_loss(hidden, table, bad)
        assert dgs.operator_status(DEV) == dgs.DGS_EINVAL
        assert torch.equal(a.loss, b.loss) and torch.equal(a.lse, b.lse)
        dw = [torch.zeros(words * width, device=DEV) for _ in range(2)]
        dh = [dgs.vocabulary_loss_grad(hidden, table, t, a.lse, dloss, d) for t, d in zip((ignored, bad), dw)]
        assert dgs.operator_status(DEV) == dgs.DGS_EINVAL and dgs.operator_status(DEV) == 0
        assert torch.equal(dh[0], dh[1]) and torch.equal(dw[0], dw[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_magnitudes(dtype):
    """Columns and rows of very different size, and losses weighted by very small and very large numbers."""
    for rows in (50, 400):
        hidden, table, target, dloss = problem(rows, 96, 1500, dtype, 12, ignored=0.1, by=1.0)
        sizes = torch.exp2(torch.randint(-9, 10, (96,), generator=torch.Generator().manual_seed(1)).float()).to(DEV)
        hidden, table = (hidden.float() * sizes).to(dtype), (table.float() / sizes).to(dtype)
        for by in (1e-20, 1.0, 1e20) if dtype != torch.float16 else (1.0,):
            got = dgs.vocabulary_loss(hidden, table, target)
            check_loss(hidden, table, target, got)
            dh, dw = grad(hidden, table, target, got.lse, dloss * by)
            check_grad(hidden, table, target, got.lse, dloss * by, dh, dw)


def test_logits_that_are_far_apart():
    """One word certain, and all words but one impossible: exponentials that are 0, 1 and nothing between, in rows whose logits go to 1000 and -1000."""
    for rows in (16, 300):
        hidden = torch.zeros(rows, 32, device=DEV)
        hidden[:, 0] = torch.linspace(-30, 30, rows, device=DEV).round()
        table = torch.zeros(600, 32, device=DEV)
        table[:, 0] = torch.linspace(-32, 32, 600, device=DEV).round()
        target = torch.arange(rows, device=DEV) * 7 % 600
        for dtype in TYPES:
            h, w = hidden.to(dtype), table.to(dtype)          # whole numbers: exact in every type, as are the logits
            got = dgs.vocabulary_loss(h, w, target)
            z = h.double() @ w.double().T
            lse = torch.logsumexp(z, 1)
            assert bool(((got.lse.double() - lse).abs() <= lse.abs() * 2.0 ** -23 + 2.0 ** -18).all())
            want = lse - z.gather(1, target[:, None])[:, 0]
            assert bool(((got.loss.double() - want).abs() <= want.abs() * 2.0 ** -22 + 2.0 ** -18).all())
            dloss = torch.ones(rows, device=DEV)
            dh, dw = grad(h, w, target, got.lse, dloss)
            check_grad(h, w, target, got.lse, dloss, dh, dw)


def test_rows_that_are_one_row_and_a_loss_that_is_one_value():
    for rows in (30, 500):
        hidden, table, target, dloss = problem(rows, 72, 900, torch.bfloat16, 13)
        one, single = hidden[:1], dloss[:1].clone()
        a, b = dgs.vocabulary_loss(one.expand(rows, 72), table, target), dgs.vocabulary_loss(one.repeat(rows, 1), table, target)
        assert torch.equal(a.loss, b.loss) and torch.equal(a.lse, b.lse)
        dw = [torch.zeros(900 * 72, device=DEV) for _ in range(4)]
        dh = [dgs.vocabulary_loss_grad(h, table, target, a.lse, g, d) for h, g, d in zip((one.expand(rows, 72), one.repeat(rows, 1), one.repeat(rows, 1), one.repeat(rows, 1)),
                                                                                        (single, single, single.expand(rows), single.repeat(rows)), dw)]
        assert all(torch.equal(dh[0], x) for x in dh[1:]) and all(torch.equal(dw[0], x) for x in dw[1:])


def test_shapes_and_empty_batches():
    hidden, table, target, dloss = problem(60, 40, 700, torch.float16, 14)
    got = dgs.vocabulary_loss(hidden.view(3, 20, 40), table, target.view(3, 20))
    assert got.loss.shape == got.lse.shape == (3, 20)
    dh = dgs.vocabulary_loss_grad(hidden.view(3, 20, 40), table, target.view(3, 20), got.lse, dloss.view(3, 20))
    assert dh.shape == (3, 20, 40)
    alone = dgs.vocabulary_loss(hidden[4], table, target[4])                          # one row without a dimension for it
    assert alone.loss.shape == () and dgs.vocabulary_loss_grad(hidden[4], table, target[4], alone.lse, dloss[:1]).shape == (40,)
    empty = dgs.vocabulary_loss(hidden[:0], table, target[:0])
    assert empty.loss.shape == (0,)
    dw = torch.full((700 * 40,), 3.0, device=DEV)
    assert dgs.vocabulary_loss_grad(hidden[:0], table, target[:0], empty.lse, dloss[:1], dw, add=True).shape == (0, 40) and bool((dw == 3.0).all())
    dgs.vocabulary_loss_grad(hidden[:0], table, target[:0], empty.lse, dloss[:0], dw)
    assert not dw.any()


def test_gradient_against_differences():
    """The loss in 64 bits along directions: central differences of step e are off by e^2 / 6 of the third derivative, and the gradient by its own roundings."""
    for rows, words in ((33, 300), (300, 3000)):
        hidden, table, target, _ = problem(rows, 48, words, torch.float32, 15, ignored=0.2)
        weights = torch.rand(rows, device=DEV)
        lse = dgs.vocabulary_loss(hidden, table, target).lse
        dh, dw = grad(hidden, table, target, lse, weights)
        live, at = target >= 0, target.clamp(min=0)

        def value(h, w):
            z = h @ w.T
            return float(((torch.logsumexp(z, 1) - z.gather(1, at[:, None])[:, 0]) * weights.double() * live).sum())

        g = torch.Generator(device=DEV).manual_seed(1)
        for _ in range(3):
            a, b = torch.randn(hidden.shape, generator=g, device=DEV, dtype=torch.float64), torch.randn(table.shape, generator=g, device=DEV, dtype=torch.float64)
            e, h, w = 1e-5, hidden.double(), table.double()
            slope = (value(h + e * a, w + e * b) - value(h - e * a, w - e * b)) / (2 * e)
            mine = float((dh.double() * a).sum() + (dw.double() * b).sum())
            size = float((dh.double() * a).abs().sum() + (dw.double() * b).abs().sum())
            assert abs(slope - mine) <= 2e-5 * size


def test_the_same_bits_again_in_a_graph_and_on_another_stream():
    for rows, words in ((20, 400), (700, 9000)):
        hidden, table, target, dloss = problem(rows, 136, words, torch.bfloat16, 16)
        dw = torch.zeros(words * 136, device=DEV)

        def step():
            r = dgs.vocabulary_loss(hidden, table, target)
            return r.loss, r.lse, dgs.vocabulary_loss_grad(hidden, table, target, r.lse, dloss, dw)

        first = [t.clone() for t in step()] + [dw.clone()]
        side = torch.cuda.Stream(device=DEV)
        side.wait_stream(torch.cuda.current_stream(DEV))
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        out = []
        with torch.cuda.stream(side):
            for graph in graphs:                                # two of them, each with a workspace of its own
                with torch.cuda.graph(graph, stream=side):
                    out.append(step())
        torch.cuda.synchronize()
        for graph, o in zip(graphs, out):
            dw.fill_(5.0)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(first, [*o, dw]))
        hidden.mul_(0.5)                                        # other values in the same places
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        again = [t.clone() for t in step()]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, out[1]))
        with torch.cuda.stream(side):
            other = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, other)) and dgs.operator_status(DEV) == 0


def test_two_calls_at_once():
    """Calls on two streams, each with tensors of its own: what either gives alone."""
    sets = [problem(900, 200, 7000, torch.bfloat16, 17 + i) for i in range(2)]
    alone = []
    for h, w, t, g in sets:
        lse = dgs.vocabulary_loss(h, w, t).lse
        dw = torch.zeros(w.numel(), device=DEV)
        alone.append((lse, dgs.vocabulary_loss_grad(h, w, t, lse, g, dw), dw))
    torch.cuda.synchronize()
    streams, both = [torch.cuda.Stream(device=DEV) for _ in range(2)], [[], []]
    for _ in range(5):
        for i, (h, w, t, g) in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                lse = dgs.vocabulary_loss(h, w, t).lse
                dw = torch.zeros(w.numel(), device=DEV)
                both[i].append((lse, dgs.vocabulary_loss_grad(h, w, t, lse, g, dw), dw))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for r in both[i] for a, b in zip(r, alone[i]))
    assert dgs.operator_status(DEV) == 0


def test_calls_that_torch_would_record_warn():
    hidden, table, target, _ = problem(8, 16, 50, torch.float32, 18)
    for what, args in (("hidden", (hidden.clone().requires_grad_(True), table)), ("weight", (hidden, table.clone().requires_grad_(True)))):
        with pytest.warns(UserWarning, match=f"{what}.*vocabulary_loss"):
            dgs.vocabulary_loss(*args, target)
