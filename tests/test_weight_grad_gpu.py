"""Weight and bias gradients from checkpoints: sums that are exact in f32 must come out bit for bit, others within the roundings of their
accumulation, at the lengths, layouts, lists and alignments where tiles and splits can go wrong.  Up to 256 rows with little to do take a kernel
of their own; sizes lie on both sides."""
import numpy as np
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def whole_numbers(rows, inputs, outputs, dtype, seed, fmt):
    """A checkpoint and a gradient of small whole numbers: every sum over up to 2^16 rows is exact in f32, in any order."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randint(-7, 8, (rows, inputs), generator=g, device=DEV).float()
    dy = torch.randint(-8, 9, (rows, outputs), generator=g, device=DEV).to(dtype)
    c = dgs.Checkpoint(rows, inputs, fmt, device=DEV)
    c.save(x)
    assert torch.equal(c.load(), x)
    return c, x.double(), dy


def grads(c, dy, layout, add=None, **lists):
    e = lists["offsets"].numel() - 1 if "offsets" in lists else 1
    i, o = c.cols, dy.shape[1]
    flat = torch.full((3 + e * (i * o + o) + 5,), float("nan"), device=DEV)         # slices at odd offsets, guarded
    dw, db = flat[1:1 + e * i * o], flat[2 + e * i * o:2 + e * i * o + e * o]
    if add is not None:
        dw.copy_(add[0].reshape(-1))
        db.copy_(add[1].reshape(-1))
    c.weight_grad(dy, dw, db, layout=layout, add=add is not None, **lists)
    assert dgs.operator_status(DEV) == 0
    assert int(torch.isnan(flat).sum()) == flat.numel() - dw.numel() - db.numel()   # and nothing is written around them
    shape = (e, o, i) if layout == "out_in" else (e, i, o)
    return dw.view(shape).squeeze(0) if e == 1 else dw.view(shape), db.view(e, o).squeeze(0) if e == 1 else db.view(e, o)


def expected(x, dy, layout):
    d = dy.double()
    return (d.T @ x if layout == "out_in" else x.T @ d), d.sum(0)


@pytest.mark.parametrize("layout", ["out_in", "in_out"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("rows,inputs,outputs", [
    (1, 1, 1), (1, 128, 256), (15, 17, 9), (64, 128, 256), (65, 129, 257), (63, 127, 130), (200, 40, 1000), (128, 512, 8), (333, 64, 1),
    (4096, 1, 33), (1000, 300, 515), (513, 1, 1), (513, 128, 256), (575, 17, 9), (577, 129, 257), (640, 127, 130), (600, 40, 1000), (641, 512, 8),
    (512, 512, 513)])
def test_sums_of_whole_numbers_are_exact(rows, inputs, outputs, dtype, fmt, layout):
    c, x, dy = whole_numbers(rows, inputs, outputs, dtype, rows + inputs, fmt)
    dw, db = expected(x, dy, layout)
    got, gb = grads(c, dy, layout)
    assert torch.equal(got.double(), dw) and torch.equal(gb.double(), db)
    old = torch.randint(-99, 99, dw.shape, device=DEV).float(), torch.randint(-99, 99, db.shape, device=DEV).float()
    got, gb = grads(c, dy, layout, add=old)
    assert torch.equal(got.double(), dw + old[0]) and torch.equal(gb.double(), db + old[1])
    alone = torch.empty_like(got).reshape(-1)
    c.weight_grad(dy, alone, layout=layout)              # without a bias
    assert torch.equal(alone.view_as(dw).double(), dw)


@pytest.mark.parametrize("layout", ["out_in", "in_out"])
@pytest.mark.parametrize("rows", [64 * 40, 64 * 40 + 1, 20_000])
def test_rows_split_among_ctas(rows, layout):
    for dtype in TYPES:
        c, x, dy = whole_numbers(rows, 96, 80, dtype, rows, "int8")
        need = dgs.dgs_checkpoint_weight_grad_bytes(c._held, dgs.operators._matrix(dy, "dy"), None, 0)
        planes = {torch.float32: 6, torch.float16: 4, torch.bfloat16: 0}[dtype]
        assert need > (rows + 256) * (96 * 2 + 80 * planes)   # more than the operands as bfloat16 numbers: partial results
        dw, db = expected(x, dy, layout)
        got, gb = grads(c, dy, layout)
        assert torch.equal(got.double(), dw) and torch.equal(gb.double(), db)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset,pad", [(0, 0), (0, 8), (1, 0), (3, 5), (7, 1), (8, 0), (4, 4), (2, 6)])
@pytest.mark.parametrize("rows", [130, 600])
def test_gradients_that_begin_anywhere(rows, dtype, offset, pad):
    """Offsets and strides that put rows on every alignment, and a matrix at the very end of its memory."""
    inputs, outputs = 70, 300
    c, x, dy = whole_numbers(rows, inputs, outputs, dtype, offset * 10 + pad, "int8")
    stride = outputs + pad
    big = torch.full((offset + rows * stride - pad,), float("nan"), dtype=dtype, device=DEV)
    v = big.as_strided((rows, outputs), (stride, 1), offset)
    v.copy_(dy)
    for layout in ("out_in", "in_out"):
        got, gb = grads(c, v, layout)
        dw, db = expected(x, dy, layout)
        assert torch.equal(got.double(), dw) and torch.equal(gb.double(), db)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [100, 700])
def test_a_gradient_whose_rows_are_one_row(rows, dtype):
    c, x, dy = whole_numbers(rows, 33, 70, dtype, 3, "int8")
    one = dy[:1].expand(rows, 70)
    dw, db = expected(x, one, "out_in")
    got, gb = grads(c, one, "out_in")
    assert torch.equal(got.double(), dw) and torch.equal(gb.double(), db)


def make_lists(rows, experts, k, seed, empty=()):
    g = torch.Generator().manual_seed(seed)
    chosen = torch.stack([torch.randperm(experts, generator=g)[:k].sort().values for _ in range(rows)]) if rows else torch.zeros(0, k, dtype=torch.long)
    for e in empty:
        chosen[chosen == e] = (e + 1) % experts
    flat = chosen.reshape(-1)
    order = flat.argsort(stable=True)
    counts = torch.bincount(flat, minlength=experts)
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)])
    return offsets.to(torch.int32).to(DEV), order.to(torch.int32).to(DEV)


@pytest.mark.parametrize("layout", ["out_in", "in_out"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,experts,k,inputs,outputs", [(1, 4, 2, 40, 24), (50, 7, 1, 130, 260), (300, 5, 3, 64, 48), (5000, 2, 2, 33, 64), (257, 9, 2, 130, 72), (600, 3, 1, 32, 300)])
def test_experts(rows, experts, k, inputs, outputs, dtype, layout):
    c, x, _ = whole_numbers(rows, inputs, 1, dtype, rows, "e4m3")
    offsets, order = make_lists(rows, experts, k, rows, empty=(1,))
    dy = torch.randint(-8, 9, (rows * k, outputs), device=DEV).to(dtype)
    got, gb = grads(c, dy, layout, offsets=offsets, rows=order, rows_per=k)
    cut = offsets.tolist()
    for e in range(experts):
        part = slice(cut[e], cut[e + 1])
        dw, db = expected(x[order[part].long() // k], dy[part], layout)
        assert torch.equal(got[e].double(), dw) and torch.equal(gb[e].double(), db), e
    assert not bool(got[1].any())                        # no rows: zeros
    # without rows: row j of dy belongs to row j of the checkpoint
    c2, x2, dy2 = whole_numbers(rows * k, inputs, outputs, dtype, 1 + rows, "int8")
    got, gb = grads(c2, dy2, layout, offsets=offsets)
    for e in range(experts):
        part = slice(cut[e], cut[e + 1])
        dw, db = expected(x2[part], dy2[part], layout)
        assert torch.equal(got[e].double(), dw) and torch.equal(gb[e].double(), db), e


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cut", [(100, [3, 30, 30, 77]), (900, [3, 300, 300, 777]), (900, [1, 129, 129, 800])])
def test_rows_of_other_experts_and_behind_the_last_are_not_looked_at(rows, cut, dtype):
    """An expert's NaN stays its own: no tile lets a neighbour's row in, multiplied by zero or not."""
    inputs, outputs = 40, 72
    c, x, dy = whole_numbers(rows, inputs, outputs, dtype, 9, "int8")
    offsets = torch.tensor(cut, dtype=torch.int32, device=DEV)
    first, last, end = cut[0], cut[1], cut[3]
    dy[:first], dy[last:end], dy[end:] = float("nan"), float("inf"), float("nan")
    got, gb = grads_unchecked(c, dy, offsets)
    dw, db = expected(x[first:last], dy[first:last], "out_in")
    assert torch.equal(got[0].double(), dw) and torch.equal(gb[0].double(), db)
    assert not bool(got[1].any()) and not bool(gb[1].any())
    assert not bool(torch.isfinite(gb[2]).any())


def grads_unchecked(c, dy, offsets, rows=None, rows_per=1):
    e, i, o = offsets.numel() - 1, c.cols, dy.shape[1]
    dw, db = torch.zeros(e, o, i, device=DEV), torch.zeros(e, o, device=DEV)
    c.weight_grad(dy, dw, db, offsets=offsets, rows=rows, rows_per=rows_per)
    return dw, db


@pytest.mark.parametrize("n", [50, 700])
def test_lists_that_point_outside_are_skipped_and_reported(n):
    c, x, dy = whole_numbers(n, 32, 16, torch.float32, 2, "int8")
    rows = torch.arange(n, dtype=torch.int32, device=DEV)
    rows[7], rows[20] = n, -1                            # past the checkpoint's last row; 2^32 - 1
    offsets = torch.tensor([0, 10, n], dtype=torch.int32, device=DEV)
    got, gb = grads_unchecked(c, dy, offsets, rows)
    keep = torch.ones(n, dtype=torch.bool, device=DEV)
    keep[7] = keep[20] = False
    assert torch.equal(got[0].double(), dy[:10][keep[:10]].double().T @ x[:10][keep[:10]])
    assert torch.equal(got[1].double(), dy[10:][keep[10:]].double().T @ x[10:][keep[10:]])
    assert dgs.operator_status(DEV) == dgs.DGS_EINVAL and dgs.operator_status(DEV) == 0
    for bad in ([0, 10, n + 1], [20, 10, n], [n + 10, n + 20, n + 30], [-5, -3, -1]):
        grads_unchecked(c, dy, torch.tensor(bad, dtype=torch.int32, device=DEV))
        assert dgs.operator_status(DEV) == dgs.DGS_EINVAL
    grads_unchecked(c, dy, torch.tensor([4, 10, n - 6], dtype=torch.int32, device=DEV))      # some rows in no list: legal
    assert dgs.operator_status(DEV) == 0


def test_no_rows():
    c = dgs.Checkpoint(0, 40, device=DEV)
    for dtype in TYPES:
        dy = torch.zeros(0, 30, dtype=dtype, device=DEV)
        got, gb = grads(c, dy, "out_in")
        assert not bool(got.any()) and not bool(gb.any())
        old = torch.randn(30, 40, device=DEV), torch.randn(30, device=DEV)
        got, gb = grads(c, dy, "out_in", add=old)
        assert torch.equal(got, old[0]) and torch.equal(gb, old[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 600])
def test_every_bit_of_a_gradient_counts(rows, dtype):
    """One row that is not zero and codes of +-1, 2, 64: dw is the gradient itself times a power of two, for every finite gradient of the type."""
    g = torch.Generator(device=DEV).manual_seed(4)
    if dtype == torch.float32:
        bits = torch.randint(-2 ** 31, 2 ** 31, (1, 1 << 15), generator=g, device=DEV).to(torch.int32)
        dy = bits.view(torch.float32)
        dy = torch.where((dy.abs() > 2.0 ** -100) & (dy.abs() < 2.0 ** 120), dy, 1.0)
    else:
        dy = torch.arange(1 << 16, device=DEV).to(torch.int16).view(dtype)[None]
        dy = torch.where(torch.isfinite(dy) & (dy.abs().float() > 2.0 ** -100) & (dy.abs().float() < 2.0 ** 120), dy, 1.0)
    x = torch.zeros(rows, 4, device=DEV)
    x[-1] = torch.tensor([1.0, -1.0, 2.0, 64.0], device=DEV)
    c = dgs.Checkpoint(rows, 4, device=DEV)
    c.save(x)
    dy = torch.cat([torch.zeros(rows - 1, dy.shape[1], dtype=dtype, device=DEV), dy])
    got, gb = grads(c, dy, "out_in")
    assert torch.equal(got, dy[-1:].float().T * x[-1:]) and torch.equal(gb, dy[-1].float())


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("more", [0, 600])
def test_every_code_and_scale_is_decoded(more, fmt):
    """The products' decoding of all codes against what load says, through dw of one row and a gradient of one."""
    codes = torch.arange(256, dtype=torch.int16).to(torch.uint8)
    if fmt == "e4m3":
        codes[[127, 255]] = 0                            # not numbers: no save writes them
    else:
        codes[128] = 0                                   # -128: likewise, and with the largest scale past the largest float
    rows = []
    for byte in (1, 10, 60, 127, 200, 246, 248 if fmt == "int8" else 246):
        rows.append((codes, byte))
    rows += [(torch.zeros_like(codes), 127)] * more
    held = torch.cat([r[0] for r in rows] + [torch.full((8,), b, dtype=torch.uint8) for _, b in rows])
    c = dgs.Checkpoint(len(rows), 256, fmt, data=held.to(DEV))
    want = c.load()
    assert bool(torch.isfinite(want).all())
    for r in range(7):
        dy = torch.zeros(len(rows), 1, device=DEV)
        dy[r] = 1.0
        got, _ = grads(c, dy, "out_in")
        small = want[r].abs() < 2.0 ** -126              # subnormal values do not occur in what a save writes
        assert torch.equal(got[0][~small], want[r][~small])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["out_in", "in_out"])
def test_normal_values_within_the_roundings_of_their_sums(dtype, layout):
    rows, inputs, outputs = 3000, 200, 150
    g = torch.Generator(device=DEV).manual_seed(8)
    c = dgs.Checkpoint(rows, inputs, device=DEV)
    c.save(torch.randn(rows, inputs, generator=g, device=DEV))
    dy = (torch.randn(rows, outputs, generator=g, device=DEV) * 1e-3).to(dtype)
    x = c.load().double()
    dw, db = expected(x, dy, layout)
    size, bsize = expected(x.abs(), dy.abs(), layout)
    got, gb = grads(c, dy, layout)
    # products are exact; sixteen of them and the running sum are added at a time, each cut at no less than 2^-24 of the largest: 17 * 2^-24
    # of the sum of magnitudes for each of rows / 16 * parts additions at the very worst, a thousandth of that in the mean
    parts = {torch.float32: 3, torch.bfloat16: 1, torch.float16: 2}[dtype]
    worst = 17 * 2.0 ** -24 * (rows / 16 + 2) * parts
    assert bool(((got.double() - dw).abs() <= size * worst).all()) and bool(((gb.double() - db).abs() <= bsize * worst).all())
    # over all elements the roundings of 2^-23 of the sums so far add up like a walk: sqrt(3000 / 16 * 3) < 24 steps, and none leans one way further
    # than 3000 / 16 * 3 * 2^-24 = 3.4e-5
    assert float((got.double() - dw).norm() / dw.norm()) < 3.4e-5
    w = torch.randn_like(dw)                             # against differences: the loss is linear in the weights
    at, step = (min(3, dw.shape[0] - 1), 5), 0.5
    loss = lambda w: float((dy.double() * (x @ (w.T if layout == "out_in" else w))).sum())   # noqa: E731
    up, down = w.clone(), w.clone()
    up[at] += step
    down[at] -= step
    assert abs((loss(up) - loss(down)) / (2 * step) - float(got[at])) <= float(size[at]) * worst + 1e-9


def test_the_same_bits_every_time_and_on_a_replayed_graph():
    rows, inputs, outputs = 9000, 300, 200
    c = dgs.Checkpoint(rows, inputs, device=DEV)
    c.save(torch.randn(rows, inputs, device=DEV))
    dy = torch.randn(rows, outputs, device=DEV, dtype=torch.bfloat16)
    one, _ = grads(c, dy, "in_out")
    flat = torch.zeros(inputs * outputs, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.weight_grad(dy, flat, layout="in_out")
    for _ in range(3):
        flat.zero_()
        graph.replay()
        two, _ = grads(c, dy, "in_out")                  # an eager call between replays has a workspace of its own
        torch.cuda.synchronize()
        assert torch.equal(flat.view_as(one), one) and torch.equal(two, one)


def test_calls_that_overlap_on_two_streams():
    rows, inputs, outputs = 4096, 256, 256
    sets = []
    for s in range(2):
        c, x, dy = whole_numbers(rows, inputs, outputs, torch.bfloat16, 20 + s, "int8")
        sets.append((c, dy, expected(x, dy, "out_in")[0], torch.zeros(outputs * inputs, device=DEV), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(4):
        for c, dy, _, out, stream in sets:
            with torch.cuda.stream(stream):
                c.weight_grad(dy, out)
    torch.cuda.synchronize()
    for _, _, want, out, _ in sets:
        assert torch.equal(out.view_as(want).double(), want)
