"""Activations held in 8 bits: the bytes that a save writes, what a load reads, activations and their gradients, at the
lengths, strides and values where they can go wrong.  Bytes and held values are defined bit for bit; activations are compared with 64-bit ones."""
import numpy as np
import pytest
import torch

import paper_1910_10929_b200 as dgs
from _held import encode

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SHAPES = [(1, 1), (1, 31), (3, 32), (5, 33), (7, 127), (2, 129), (4, 160), (65, 256), (33, 1000), (517, 513), (0, 40)]


def strided(x, kind):
    """x as a matrix whose rows lie differently: odd offsets, gaps between rows."""
    rows, cols = x.shape
    if kind == "whole":
        return x.clone()
    pad, off = {"odd": (3, 1), "wide": (16, 8)}[kind]
    big = torch.full((rows * (cols + pad) + off + 64,), float("nan"), dtype=x.dtype, device=x.device)
    v = big[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(x)
    return v


def values(rows, cols, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-20, 12, (rows, 1), generator=g).float())
    if rows > 2:
        x[1] = 0.0
        x[2, ::2] = -0.0
    return x.to(dtype).to(DEV)


def same(a, b):
    """Equal values, NaN equal to NaN, zeros of either sign."""
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(0), b.nan_to_num(0))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_bytes_and_values(shape, dtype, fmt):
    x = values(*shape, dtype, sum(shape))
    want, held = encode(x.double().cpu().numpy(), fmt)
    for kind in ("whole", "odd", "wide"):
        c = dgs.Checkpoint(*shape, fmt, data=torch.full((len(want),), 0xAB, dtype=torch.uint8, device=DEV))
        assert c.save(strided(x, kind)) is None
        assert np.array_equal(c.data.cpu().numpy(), want), kind
        for to in TYPES:
            got = c.load(to)
            assert got.dtype == to and same(got, torch.from_numpy(held).to(DEV).to(to))
            out = strided(torch.zeros(shape, dtype=to, device=DEV), kind)
            c.load(out=out)
            assert same(out, got)
            if kind != "whole" and shape[0]:   # nothing is written between the rows or behind them
                base = out.as_strided((out.untyped_storage().nbytes() // out.element_size(),), (1,), 0)
                assert int(torch.isnan(base).sum()) == base.numel() - out.numel()
    assert dgs.operator_status(DEV) == 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_values_at_the_edges_of_the_format(fmt):
    top = {"int8": 127.0, "e4m3": 448.0}[fmt]
    rows = []
    for e in (-149, -140, -130, -127, -120, -20, 0, 20, 100, 119, 120, 121):
        for m in (top, np.nextafter(np.float32(top), np.float32(1e9)), np.nextafter(np.float32(top), np.float32(0)), top / 2, 1.0):
            with np.errstate(over="ignore", under="ignore"):
                big = np.float32(np.ldexp(np.float64(m), e))
            if np.isfinite(big):
                # halves of every code: ties; and neighbours of the ties
                codes = np.arange(31) * (0.5 if fmt == "int8" else 13.0)
                with np.errstate(over="ignore", under="ignore"):
                    rows.append(np.concatenate([[big], np.ldexp(codes, e).astype(np.float32)]))
    rows.append(np.full(32, np.float32(3.4028235e38)))
    rows.append(np.full(32, np.float32(1e-45)))
    x = np.array(rows, np.float32)
    x = np.concatenate([x, -x])
    x = x[np.isfinite(x).all(1)]
    want, held = encode(x, fmt)
    c = dgs.Checkpoint(*x.shape, fmt, device=DEV)
    c.save(torch.from_numpy(x).to(DEV))
    assert np.array_equal(c.data.cpu().numpy(), want)
    assert np.array_equal(c.load().cpu().numpy(), held.astype(np.float32))
    assert np.array_equal(c.load(torch.bfloat16).double().cpu().numpy(), held)      # every held value is a bfloat16 number


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("cols", [64, 70])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_block_with_an_infinity_or_nan_reads_as_nan_and_no_other(dtype, cols, fmt):
    x = torch.randn(4, cols, device=DEV).to(dtype)
    x[0, 3], x[1, 40], x[2, 31], x[2, 32] = float("inf"), float("nan"), -float("inf"), float("nan")
    want, held = encode(x.double().cpu().numpy(), fmt)
    c = dgs.Checkpoint(4, cols, fmt, device=DEV)
    c.save(x)
    assert np.array_equal(c.data.cpu().numpy(), want)
    assert same(c.load(), torch.from_numpy(held).float().to(DEV))


def act64(act, x):
    u = {"silu": x, "gelu_tanh": 2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3)}.get(act, x)
    if act == "relu":
        return torch.where(x > 0, x, 0.0), u
    if act == "gelu":
        return 0.5 * x * torch.special.erfc(-x / np.sqrt(2)), u
    return x * torch.sigmoid(u), u


def half_step(dtype, v):
    """Half a step of the type at v, subnormal steps included."""
    return v.abs() * torch.finfo(dtype).eps / 2 + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 1), (3, 33), (64, 512), (77, 1001)])
def test_activation_beside_the_save(shape, dtype, act):
    x = (torch.randn(shape, generator=torch.Generator().manual_seed(1)) * 4).to(dtype).to(DEV)
    x[0, 0] = -20.0
    c, plain = dgs.Checkpoint(*shape, device=DEV), dgs.Checkpoint(*shape, device=DEV)
    y = c.save(x, act)
    plain.save(x)
    assert torch.equal(c.data, plain.data)             # what is held is x, not act(x)
    want, u = act64(act, x.double())
    # roundings of 2^-24: expf, divide and products 12 at most (erfcf 16); the exponent's own three roundings make an error of
    # 3 |u| 2^-24 in e^-u, counted as 4; for erfc(a) the argument's two make 2 a^2 * 2 = 2 x^2, counted as 4
    rel = (16 + 4 * (x.double() ** 2 if act == "gelu" else u.abs())) * 2.0 ** -24
    bound = want.abs() * rel + half_step(dtype, want) + 2.0 ** -126
    assert bool(((y.double() - want).abs() <= bound).all())
    inplace = x.clone()
    c.save(inplace, act, out=inplace)
    assert torch.equal(inplace, y) and torch.equal(c.data, plain.data)
    wide = strided(x, "odd")
    assert torch.equal(c.save(wide, act), y)


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_activation_grad_against_the_formula_and_differences(dtype, act, fmt):
    shape = (67, 261)
    g = torch.Generator().manual_seed(5)
    x = (torch.randn(shape, generator=g) * 3).to(DEV)
    x[0, 0], x[1, 0], x[2, 0] = -25.0, 100.0, 1e30
    dy = torch.randn(shape, generator=g).to(dtype).to(DEV)
    c = dgs.Checkpoint(*shape, fmt, device=DEV)
    c.save(x)
    h = c.load().double()
    got = c.activation_grad(dy, act).double()
    hs = h.clone().requires_grad_(True)
    act64(act, hs)[0].sum().backward()
    slope = hs.grad.clone()
    slope[2] = torch.where(h[2].abs() > 100, (h[2] > 0).double(), slope[2])        # x^3 overflows nothing here; s(u) is 0 or 1
    u = act64(act, h)[1]
    # the slope is a sum of two terms of size at most 1 + |x u'|, each off by roundings as the activation is
    size = (2.2 if act == "relu" else 1.0) * torch.ones_like(h) + torch.clamp(h.abs(), max=30) * torch.exp(-0.5 * torch.clamp(h.abs(), max=30))
    rel = 40 * 2.0 ** -24
    if act == "gelu":
        rel = (16 + 4 * torch.clamp(h ** 2, max=400)) * 2.0 ** -24
    want = dy.double() * slope
    bound = dy.double().abs() * size * rel * (1 + torch.clamp(u.abs(), max=30) / 4) + half_step(dtype, want) * 1.01 + 2.0 ** -126
    assert bool(((got - want).abs() <= bound).all())
    step = 1e-5                                          # differences, away from relu's corner: off by step^2 * third derivative and cancellation
    diff = (act64(act, h + step)[0] - act64(act, h - step)[0]) / (2 * step)
    near = (h.abs() > 2 * step) & (h.abs() < 50)
    assert bool(((got - dy.double() * diff).abs() <= bound + dy.double().abs() * 1e-8)[near].all())
    inplace = dy.clone()
    c.activation_grad(inplace, act, out=inplace)
    assert torch.equal(inplace.double(), got)
    one = dy[:1].expand(shape)                           # a broadcast gradient: all rows are one row
    assert torch.equal(c.activation_grad(one, act, out=torch.empty(shape, dtype=dtype, device=DEV)),
                       c.activation_grad(one.contiguous(), act))


def test_more_than_one_stride_of_the_grid():
    """Rows and columns past what the grid covers at once: 148 * 6 CTAs of 256 units of 8."""
    for rows, cols in ((20_000, 257), (9, 600_000), (3, 1_900_001)):
        x = torch.randn(rows, cols, device=DEV, dtype=torch.bfloat16)
        c = dgs.Checkpoint(rows, cols, device=DEV)
        c.save(x)
        pick = torch.tensor([0, rows // 2, rows - 1], device=DEV)
        _, held = encode(x[pick].double().cpu().numpy(), "int8")
        assert torch.equal(c.load(torch.bfloat16)[pick].double().cpu(), torch.from_numpy(held))
        err = (c.load(torch.bfloat16).float() - x.float()).abs().amax()
        assert float(err) <= float(x.float().abs().amax()) / 127


def test_captured_and_replayed_on_another_stream():
    x = torch.randn(100, 300, device=DEV)
    dy = torch.randn(100, 300, device=DEV)
    c = dgs.Checkpoint(100, 300, device=DEV)
    y, h, dx = c.save(x, "silu"), c.load(), c.activation_grad(dy, "silu")
    side = torch.cuda.Stream()
    y2, h2, dx2 = torch.empty_like(y), torch.empty_like(h), torch.empty_like(dx)
    graph = torch.cuda.CUDAGraph()
    c2 = dgs.Checkpoint(100, 300, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        c2.save(x, "silu", out=y2)
        c2.load(out=h2)
        c2.activation_grad(dy, "silu", out=dx2)
    x.mul_(2)
    dy.mul_(3)
    graph.replay()
    torch.cuda.synchronize()
    y, h, dx = (c.save(x, "silu"), c.load(), c.activation_grad(dy, "silu"))
    assert torch.equal(y, y2) and torch.equal(h, h2) and torch.equal(dx, dx2)
