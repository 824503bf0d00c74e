"""Rows taken to the experts' lists and back, against plain 64-bit arithmetic, at the sizes, types, alignments and lists where they can go wrong."""
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def lists(tokens, k, experts, seed, masked=0.0):
    """(order, place) as a router leaves them, from plain indexing on the CPU."""
    g = torch.Generator().manual_seed(seed)
    chosen = torch.stack([torch.randperm(experts, generator=g)[:k] for _ in range(tokens)]) if tokens else torch.zeros(0, k, dtype=torch.long)
    chosen = chosen.masked_fill(torch.rand(tokens, k, generator=g) < masked, experts).sort(1).values
    flat = chosen.reshape(-1)
    order = flat.argsort(stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel())
    empty = flat == experts
    return order.masked_fill(empty[order], -1).to(torch.int32).to(DEV), place.masked_fill(empty, -1).to(torch.int32).view(tokens, k).to(DEV)


def values(rows, cols, dtype, seed, pad=0, offset=0):
    """Random numbers in a guarded view: rows `pad` elements apart, `offset` elements behind the start."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    whole = torch.full((offset + rows * (cols + pad) + 1,), float("nan"), dtype=dtype, device=DEV)
    v = whole.as_strided((rows, cols), (cols + pad, 1), offset)
    v.copy_(torch.randn(rows, cols, generator=g, device=DEV))
    return v, whole


def untouched(whole, view):
    return int(torch.isnan(whole).sum()) == whole.numel() - view.numel()


def taken(y, place):
    """[tokens, k, cols] in 64 bits, zeros in empty slots."""
    p = place.long()
    return torch.where(p[:, :, None] >= 0, y.double()[p.clamp(min=0)], 0.0)


SIZES = [(1, 1, 1), (1, 1, 768), (1, 2, 256), (2, 3, 7), (5, 2, 8), (33, 1, 255), (33, 4, 257), (100, 5, 512), (64, 8, 300), (17, 9, 129), (40, 32, 66),
         (300, 3, 1001), (9, 2, 8192), (5000, 2, 40), (3, 17, 2051)]


@pytest.mark.parametrize("masked", [0.0, 0.3])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,k,cols", SIZES)
def test_rows_go_to_their_places_and_back(tokens, k, cols, dtype, masked):
    order, place = lists(tokens, k, k + 3, tokens * 100 + k, masked)
    for pad, offset in ((0, 0), (8, 16), (1, 3)):
        x, _ = values(tokens, cols, dtype, 1, pad, offset)
        y, whole = values(tokens * k, cols, dtype, 2, pad, offset)
        y.fill_(7.0)
        assert dgs.gather_experts(x, order, place, out=y) is y
        want = torch.where(order[:, None] >= 0, x[order.long().clamp(min=0) // k], torch.zeros((), dtype=dtype, device=DEV))
        assert torch.equal(y, want) and untouched(whole, y)
        # the gradient: of random rows, those behind the last list holding NaN
        dy, _ = values(tokens * k, cols, dtype, 3, pad, offset)
        dy.masked_fill_(order[:, None] < 0, float("nan"))
        out, whole = values(tokens, cols, dtype, 4, pad, offset)
        assert dgs.gather_experts_grad(dy, place, out=out) is out
        rows = taken(dy, place)
        # k - 1 roundings of f32 sums that are at most the sum of magnitudes, one rounding to the type
        bound = rows.abs().sum(1) * k * 2.0 ** -24 + rows.sum(1).abs() * (torch.finfo(dtype).eps / 2) * (1 + 2.0 ** -10) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
        assert bool(((out.double() - rows.sum(1)).abs() <= bound).all()) and untouched(whole, out)
    assert dgs.operator_status(DEV) == 0


@pytest.mark.parametrize("masked", [0.0, 0.3])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,k,cols", SIZES)
def test_weighted_sums_and_their_gradient(tokens, k, cols, dtype, masked):
    order, place = lists(tokens, k, k + 3, tokens * 100 + k, masked)
    g = torch.Generator(device=DEV).manual_seed(9)
    weight = torch.rand(tokens, k, generator=g, device=DEV) * 2 - 0.5
    eps, tiny = torch.finfo(dtype).eps, torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    for pad, offset in ((0, 0), (8, 16), (1, 3)):
        y, _ = values(tokens * k, cols, dtype, 2, pad, offset)
        y.masked_fill_(order[:, None] < 0, float("nan"))
        out, whole = values(tokens, cols, dtype, 4, pad, offset)
        dgs.combine_experts(y, weight, place, out=out)
        rows = taken(y, place)
        terms = rows * weight.double()[:, :, None]
        bound = terms.abs().sum(1) * 2 * k * 2.0 ** -24 + terms.sum(1).abs() * (eps / 2) * (1 + 2.0 ** -10) + tiny
        assert bool(((out.double() - terms.sum(1)).abs() <= bound).all()) and untouched(whole, out)
        dout, _ = values(tokens, cols, dtype, 5, pad, offset)
        dy, whole = values(tokens * k, cols, dtype, 6, pad, offset)
        got, dweight = dgs.combine_experts_grad(dout, y, weight, order, place, out=dy)
        assert got is dy and untouched(whole, dy)
        slot = order.long().clamp(min=0)
        want = torch.where(order[:, None] >= 0, dout.double()[slot // k] * weight.double().view(-1)[slot][:, None], 0.0)
        # a product in f32, then the type
        assert bool(((dy.double() - want).abs() <= want.abs() * (eps / 2 + 2.0 ** -23) + tiny).all())
        products = rows * dout.double()[:, None, :]
        assert dweight.shape == place.shape and bool((dweight[place < 0] == 0).all())
        # f32 sums of `cols` products in some order: each of them passes through at most cols / 32 + 12 roundings
        assert bool(((dweight.double() - products.sum(2)).abs() <= products.abs().sum(2) * (cols / 32 + 12) * 2.0 ** -24).all())
    assert dgs.operator_status(DEV) == 0


@pytest.mark.parametrize("dtype", TYPES)
def test_all_slots_empty_and_no_tokens(dtype):
    none = torch.full((12,), -1, dtype=torch.int32, device=DEV)
    x, y = torch.ones(4, 40, dtype=dtype, device=DEV), torch.full((12, 40), float("nan"), dtype=dtype, device=DEV)
    place, weight = none.view(4, 3), torch.full((4, 3), float("nan"), device=DEV)      # weights of tokens without experts
    assert not dgs.gather_experts(x, none, place).any()
    assert not dgs.gather_experts_grad(y, place).any() and not dgs.combine_experts(y, weight, place).any()
    dy, dw = dgs.combine_experts_grad(x, y, weight, none, place)
    assert not dy.any() and not dw.any()
    assert dgs.gather_experts(x[:0], none[:0], place[:0]).shape == (0, 40) and dgs.gather_experts_grad(y[:0], place[:0]).shape == (0, 40)
    assert dgs.combine_experts(y[:0], weight[:0], place[:0]).shape == (0, 40)
    dy, dw = dgs.combine_experts_grad(x[:0], y[:0], weight[:0], none[:0], place[:0])
    assert dy.shape == (0, 40) and dw.shape == (0, 3)
    assert dgs.operator_status(DEV) == 0


def test_infinities_and_nan_stay_with_their_tokens():
    order, place = lists(50, 2, 4, 1)
    y, _ = values(100, 300, torch.bfloat16, 1)
    weight = torch.rand(50, 2, device=DEV)
    clean = dgs.combine_experts(y, weight, place)
    y[place[7, 1].long(), 13] = float("inf")
    y[place[8, 0].long(), 299] = float("nan")
    out = dgs.combine_experts(y, weight, place)
    assert float(out[7, 13]) == float("inf") and bool(torch.isnan(out[8, 299]))
    out[7, 13], out[8, 299] = clean[7, 13], clean[8, 299]
    assert torch.equal(out, clean)


def test_places_that_point_outside_are_left_out_and_reported():
    order, place = lists(40, 2, 4, 2)
    y, _ = values(80, 100, torch.float32, 1)
    weight = torch.rand(40, 2, device=DEV)
    bad = place.clone()
    bad[3, 1], bad[9, 0] = 80, 0x7FFFFFFF
    out = dgs.combine_experts(y, weight, bad)
    assert dgs.operator_status(DEV) == dgs.DGS_EINVAL and dgs.operator_status(DEV) == 0
    assert torch.equal(out[3], y[place[3, 0].long()] * weight[3, 0]) and torch.equal(out[9], y[place[9, 1].long()] * weight[9, 1])
    whole = dgs.gather_experts(y[:40], order, place)
    got = dgs.gather_experts(y[:40], order, bad, out=torch.full((80, 100), 5.0, device=DEV))
    assert dgs.operator_status(DEV) == dgs.DGS_EINVAL
    lost = torch.tensor([int(place[3, 1]), int(place[9, 0])], device=DEV)
    assert bool((got[lost] == 5.0).all())
    got[lost] = whole[lost]
    assert torch.equal(got, whole)
    _, dweight = dgs.combine_experts_grad(y[:40], y, weight, order, bad)
    assert dgs.operator_status(DEV) == dgs.DGS_EINVAL and float(dweight[3, 1]) == float(dweight[9, 0]) == 0.0


@pytest.mark.parametrize("dtype", TYPES)
def test_a_gradient_whose_rows_are_one_row(dtype):
    order, place = lists(70, 3, 5, 3, 0.1)
    one, _ = values(1, 264, dtype, 1)
    y, _ = values(210, 264, dtype, 2)
    weight = torch.rand(70, 3, device=DEV)
    a = dgs.combine_experts_grad(one.expand(70, 264), y, weight, order, place)
    b = dgs.combine_experts_grad(one.repeat(70, 1), y, weight, order, place)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(dgs.gather_experts(one.expand(70, 264), order, place), dgs.gather_experts(one.repeat(70, 1), order, place))


def test_the_lists_of_a_router():
    g = torch.Generator(device=DEV).manual_seed(4)
    z = torch.randn(333, 11, generator=g, device=DEV)
    z.masked_fill_(torch.rand(333, 11, generator=g, device=DEV) < 0.6, float("-inf"))
    z[5] = float("-inf")
    r = dgs.route_experts(z, 3)
    x = torch.randn(3, 111, 90, generator=g, device=DEV)
    y = dgs.gather_experts(x, r.order, r.place)
    out = dgs.combine_experts(y, r.weight, r.place).view_as(x)
    # weights of a token add up to 1, or to 0 where it has no experts: f32 roundings of three terms
    there = (r.expert >= 0).any(1).view(3, 111, 1)
    assert bool(((out - torch.where(there, x, 0.0)).abs() <= x.abs() * 8 * 2.0 ** -24).all()) and not out.view(333, 90)[5].any()
    back = dgs.gather_experts_grad(y, r.place).view_as(x)
    assert torch.equal(back, x * (r.expert >= 0).sum(1).view(3, 111, 1)) or bool(((back - x * (r.expert >= 0).sum(1).view(3, 111, 1)).abs() <= x.abs() * 3 * 2.0 ** -23).all())


def test_gradients_against_differences():
    """Weights and rows moved by a step: the sums are linear in both, so f64 differences of the formula are the gradient up to roundings."""
    order, place = lists(23, 3, 5, 6, 0.2)
    y, _ = values(69, 37, torch.float32, 1)
    y.masked_fill_(order[:, None] < 0, 0.0)
    dout, _ = values(23, 37, torch.float32, 2)
    weight = torch.rand(23, 3, device=DEV)
    value = lambda y, w: float((taken(y, place) * w.double()[:, :, None] * dout.double()[:, None]).sum())   # noqa: E731
    dy, dw = dgs.combine_experts_grad(dout, y, weight, order, place)
    for i, j in ((0, 0), (5, 2), (22, 1)):
        w = weight.double()
        up, down = w.clone(), w.clone()
        up[i, j] += 0.5
        down[i, j] -= 0.5
        slope = value(y, up) - value(y, down)
        assert abs(slope - float(dw[i, j])) <= 1e-5 * max(1.0, abs(slope))
    for i, j in ((0, 0), (40, 36), (68, 5)):
        up, down = y.double(), y.double()
        up[i, j] += 0.5
        down[i, j] -= 0.5
        assert abs(value(up, weight) - value(down, weight) - float(dy[i, j])) <= 1e-6


def test_captured_and_replayed_on_another_stream():
    order, place = lists(300, 2, 6, 7, 0.1)
    x, _ = values(300, 136, torch.bfloat16, 1)
    weight = torch.rand(300, 2, device=DEV)
    side = torch.cuda.Stream(device=DEV)
    side.wait_stream(torch.cuda.current_stream(DEV))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            y = dgs.gather_experts(x, order, place)
            out = dgs.combine_experts(y, weight, place)
            dy, dw = dgs.combine_experts_grad(x, y, weight, order, place)
            dx = dgs.gather_experts_grad(dy, place)
    torch.cuda.synchronize()
    for seed in (11, 12):
        x.copy_(torch.randn(300, 136, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        y2 = dgs.gather_experts(x, order, place)
        dy2, dw2 = dgs.combine_experts_grad(x, y2, weight, order, place)
        assert torch.equal(y, y2) and torch.equal(out, dgs.combine_experts(y2, weight, place)) and torch.equal(dy, dy2) and torch.equal(dw, dw2)
        assert torch.equal(dx, dgs.gather_experts_grad(dy2, place))


def test_calls_that_torch_would_record_warn():
    order, place = lists(8, 2, 4, 8)
    x = torch.randn(8, 16, device=DEV, requires_grad=True)
    w = torch.rand(8, 2, device=DEV, requires_grad=True)
    with pytest.warns(UserWarning, match="gather_experts"):
        y = dgs.gather_experts(x, order, place)
    with pytest.warns(UserWarning, match="combine_experts"):
        dgs.combine_experts(y, w, place)
