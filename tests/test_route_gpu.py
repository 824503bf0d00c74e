"""The router: its choice, with ties, masks and groups, against a selection in 64 bits token by token, its weights and
lists, and the gradient against the formula's and against differences."""
import math

import numpy as np
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def scores64(z, score):
    z = z.astype(np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if score == "sigmoid":
            return 1.0 / (1.0 + np.exp(-z))
        top = z.max(1, keepdims=True)
        s = np.exp(z - np.where(np.isfinite(top), top, 0.0))
        total = s.sum(1, keepdims=True)
        return s / np.where(total > 0, total, 1.0)


def choose(z, bias, k, score, groups=1, kept=1, best=1):
    """Token by token, by sorting."""
    T, E = z.shape
    s = scores64(z, score)
    out = np.full((T, k), -1, np.int64)
    size = E // groups
    for t in range(T):
        free = [e for e in range(E) if z[t, e] > -np.inf]
        key = {e: s[t, e] + float(bias[e]) if bias is not None else s[t, e] if groups > 1 and best == 2 else float(z[t, e]) for e in free}
        if groups > 1:
            total = {}
            for g in range(groups):
                members = sorted((key[e] for e in free if e // size == g), reverse=True)[:best]
                if members:
                    total[g] = sum(members)
            keep = sorted(total, key=lambda g: (-total[g], g))[:kept]
            free = [e for e in free if e // size in keep]
        chosen = sorted(sorted(free, key=lambda e: (-key[e], e))[:k])
        out[t, :len(chosen)] = chosen
    return out


def weights64(z, expert, score, renorm, scale):
    s = scores64(z, score)
    w = np.where(expert >= 0, np.take_along_axis(s, np.maximum(expert, 0), 1), 0.0)
    if renorm:
        total = w.sum(1, keepdims=True)
        w = w / np.where(total > 0, total, 1.0)
    return w * scale


def lists(expert, E):
    flat = expert.reshape(-1)
    there = np.flatnonzero(flat >= 0)
    order = there[np.argsort(flat[there], kind="stable")]
    place = np.full(flat.size, -1, np.int64)
    place[order] = np.arange(order.size)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[there], minlength=E))])
    return offsets, np.concatenate([order, np.full(flat.size - order.size, -1)]), place.reshape(expert.shape)


def check(z, k, score="softmax", bias=None, groups=1, kept=1, best=1, renorm=True, scale=1.0):
    dev = z.to(DEV)
    r = dgs.route_experts(dev, k, score=score, bias=None if bias is None else bias.to(DEV), groups=groups, groups_kept=kept, group_best=best,
                          renormalise=renorm, scale=scale)
    zn = z.double().numpy()
    expert = choose(zn, None if bias is None else bias.double().numpy(), k, score, groups, kept, best)
    assert np.array_equal(r.expert.cpu().numpy(), expert)
    want = weights64(zn, expert, score, renorm, scale)
    # roundings of 2^-24: the difference in the exponent (of size |z - ref|, which its exponential makes an error of z - ref roundings),
    # expf 2 ulp, the sum of at most 37 in sequence, two divisions, a product
    span = np.where(np.isfinite(zn), np.abs(zn), 0.0).max(initial=0.0)
    assert np.all(np.abs(r.weight.double().cpu().numpy() - want) <= want * (48 + 2 * span) * 2.0 ** -24 + 2.0 ** -126)
    offsets, order, place = lists(expert, z.shape[1])
    assert np.array_equal(r.offsets.cpu().numpy(), offsets)
    assert np.array_equal(r.order.cpu().numpy(), order)
    assert np.array_equal(r.place.cpu().numpy(), place)
    assert dgs.operator_status(DEV) == 0
    return r


def logits(T, E, dtype, seed, masked=0.0, levels=None):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(T, E, generator=g) * 2
    if levels:                                           # few distinct values: ties everywhere
        z = torch.randint(0, levels, (T, E), generator=g).float() - levels / 2
    if masked:
        z.masked_fill_(torch.rand(T, E, generator=g) < masked, -math.inf)
    return z.to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 2), (2, 33, 32), (63, 8, 8), (64, 60, 4), (65, 128, 1), (200, 257, 8), (130, 512, 6), (70, 1024, 32)])
def test_choice_weights_and_lists(T, E, k, dtype):
    for score in ("softmax", "sigmoid"):
        for renorm in (False, True):
            check(logits(T, E, dtype, T + E), k, score, renorm=renorm, scale=2.5 if renorm else 1.0)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("E,groups,kept,k", [(64, 8, 4, 6), (256, 8, 4, 8), (60, 5, 2, 7), (40, 40, 9, 9), (12, 3, 1, 4), (768, 48, 11, 20), (96, 2, 2, 5)])
def test_groups_and_bias(E, groups, kept, k, best, score):
    g = torch.Generator().manual_seed(E)
    bias = torch.randn(E, generator=g) * 0.1
    for b in (None, bias):
        check(logits(90, E, torch.float32, E + k), k, score, b, groups, kept, best)
        check(logits(90, E, torch.bfloat16, E + k + 1, masked=0.4), k, score, b, groups, kept, best, renorm=False)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("levels", [1, 2, 5])
def test_ties_go_to_the_lowest_index(levels, score):
    for E, groups, kept in ((48, 1, 1), (48, 4, 2), (130, 10, 3)):
        z = logits(100, E, torch.float32, levels + E, levels=levels, masked=0.1)
        for bias in (None, torch.zeros(E), torch.full((E,), 0.25)):
            for best in (1, 2):
                check(z, 7, score, bias, groups, kept, best)


def test_keys_that_32_bits_cannot_tell_apart():
    """Scores and biases that balance to within far less than an f32 rounding: decided in 64 bits, for experts and for groups."""
    E, T = 64, 300
    g = torch.Generator().manual_seed(0)
    z = torch.randn(T, E, generator=g)
    z = z[:1].expand(T, E).clone()
    for t in range(T):                                   # the same logits in another order, so that one bias vector cannot even them out
        z[t, 32:] = z[0, 32:][torch.randperm(32, generator=g)]
    s = torch.sigmoid(z[0].double())
    bias = (0.9 - s).float()                             # token 0: every key is 0.9 within a rounding of the bias
    check(z, 5, "sigmoid", bias)
    check(z, 5, "sigmoid", bias, groups=8, kept=3, best=2)
    check(z, 5, "softmax", (0.5 - torch.softmax(z[0].double(), 0)).float(), groups=8, kept=3, best=2)
    check(torch.full((4, E), 40.0), 3, "sigmoid", torch.linspace(0, 1e-9, E))       # scores that round to 1, keys that differ by 1e-11


def test_rows_with_few_or_no_experts_left():
    z = logits(70, 20, torch.float32, 3)
    z[5] = -math.inf
    z[6, 1:] = -math.inf
    z[7, :17] = -math.inf
    z[69] = -math.inf
    for score in ("softmax", "sigmoid"):
        for renorm in (False, True):
            r = check(z, 6, score, renorm=renorm)
            check(z, 6, score, torch.linspace(-1, 1, 20), groups=4, kept=2, best=2, renorm=renorm)
            assert r.expert[5].tolist() == [-1] * 6 and r.weight[5].tolist() == [0.0] * 6
    low = torch.full((3, 20), torch.finfo(torch.float32).min)                        # masks of the lowest value are logits like any other
    low[1, 4] = 0.0
    check(low, 3)
    check(low, 3, "sigmoid", renorm=False)


def test_weights_of_scores_that_underflow():
    """Experts chosen by their bias although their scores are next to nothing: their ratio is what counts."""
    z = torch.full((2, 8), -150.0)
    z[:, 0], z[0, 1] = 100.0, -149.0
    bias = torch.tensor([-5.0, 3.0, 3.0, 0, 0, 0, 0, 0])
    r = dgs.route_experts(z.to(DEV), 2, bias=bias.to(DEV))
    assert r.expert.tolist() == [[1, 2], [1, 2]]
    want = torch.softmax(z[:, 1:3].double(), 1)
    assert float((r.weight.cpu().double() - want).abs().max()) < 400 * 2.0 ** -24
    r = dgs.route_experts(z.to(DEV), 2, score="sigmoid", bias=bias.to(DEV))
    assert r.expert.tolist() == [[1, 2], [1, 2]]
    assert float((r.weight.cpu().double() - want).abs().max()) < 400 * 2.0 ** -24


def test_a_token_with_nan_or_infinity_has_no_experts():
    z = logits(66, 40, torch.float32, 1)
    z[0, 3], z[65, 39] = math.nan, math.inf
    r = dgs.route_experts(z.to(DEV), 3)
    for t in (0, 65):
        assert r.expert[t].tolist() == [-1] * 3 and bool(torch.isnan(r.weight[t]).all())
    assert int(r.offsets[-1]) == 64 * 3
    want = choose(z[1:65].double().numpy(), None, 3, "softmax")
    assert np.array_equal(r.expert[1:65].cpu().numpy(), want)
    dz = dgs.route_experts_grad(z.to(DEV), r.expert, torch.ones(66, 3, device=DEV))
    assert bool(torch.isnan(dz[0]).all()) and bool(torch.isnan(dz[65]).all()) and bool(torch.isfinite(dz[1:65]).all())


def test_strides_no_tokens_many_tokens():
    z = logits(100, 50, torch.float16, 8)
    big = torch.full((100, 57), float("nan"), dtype=torch.float16)
    big[:, 3:53] = z
    a, b = dgs.route_experts(big.to(DEV)[:, 3:53], 4), check(z, 4)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    r = dgs.route_experts(torch.zeros(0, 50, device=DEV), 4)
    assert r.expert.shape == (0, 4) and r.offsets.tolist() == [0] * 51 and r.order.numel() == 0
    one = z[:1].to(DEV).expand(100, 50)                   # all tokens are one row
    assert torch.equal(dgs.route_experts(one, 4).expert, dgs.route_experts(one.contiguous(), 4).expert)
    z = torch.randn(70_001, 16, device=DEV)               # more than 1024 tiles of 64 tokens
    r = dgs.route_experts(z, 2)
    want = z.topk(2, 1).indices.sort(1).values
    assert torch.equal(r.expert.long(), want)
    offsets, order, place = lists(want.cpu().numpy(), 16)
    assert np.array_equal(r.order.cpu().numpy(), order) and np.array_equal(r.offsets.cpu().numpy(), offsets)
    assert np.array_equal(r.place.cpu().numpy(), place)
    batch = dgs.route_experts(z[:70_000].view(7, 10_000, 16), 2)
    assert torch.equal(batch.expert, r.expert[:70_000])


def grad64(z, expert, dw, score, renorm, scale):
    """By torch's own differentiation of the weights in 64 bits."""
    z = z.double().clone().requires_grad_(True)
    at, there = expert.clamp(min=0).long(), expert >= 0
    if score == "sigmoid":
        s = torch.sigmoid(z)
    else:
        dead = ~(z > -math.inf).any(1, keepdim=True)
        s = torch.softmax(z.masked_fill(dead, 0.0), 1)
    w = torch.where(there, s.gather(1, at), 0.0)
    if renorm:
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
    (w * scale * dw.double()).sum().backward()
    return torch.where(z > -math.inf, z.grad, 0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (3, 64, 2), (50, 60, 7), (33, 300, 8), (9, 1000, 32)])
def test_gradient(T, E, k, renorm, score, dtype):
    z = logits(T, E, dtype, T * E, masked=0.1 if E > 1 else 0.0)
    if T > 2:
        z[1] = -math.inf
        z[2, 1:] = -math.inf
    dev = z.to(DEV)
    expert = dgs.route_experts(dev, k, score=score, renormalise=renorm).expert
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(2)).to(DEV)
    got = dgs.route_experts_grad(dev, expert, dw, score=score, renormalise=renorm, scale=1.5)
    want = grad64(dev, expert, dw, score, renorm, 1.5)
    # g and the sum of g p, each off by the roundings of p (48 + 2 * 8), of products and of a sum of 37: 128 roundings of the largest g, times p <= 1
    largest = (dw.abs().amax(1, keepdim=True) * 1.5).double()
    bound = largest * 2 * 128 * 2.0 ** -24 + want.abs() * torch.finfo(dtype).eps / 2 + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    assert bool(((got.double() - want).abs() <= bound).all())
    inplace = dev.clone()
    dgs.route_experts_grad(inplace, expert, dw, score=score, renormalise=renorm, scale=1.5, out=inplace)
    assert torch.equal(inplace, got)
    if dtype == torch.float32 and T > 2:                  # against differences of the weights in 64 bits, the choice held fixed
        zn, en, step = z.double().numpy(), expert.cpu().numpy().astype(np.int64), 1e-6
        loss = lambda v: float((weights64(v, en, score, renorm, 1.5) * dw.double().cpu().numpy()).sum())   # noqa: E731
        for t, e in ((0, 0), (0, int(expert[0, 0])), (T - 1, E - 1), (T - 1, int(expert[T - 1, -1]))):
            if zn[t, e] > -np.inf:
                up, down = zn.copy(), zn.copy()
                up[t, e] += step
                down[t, e] -= step
                assert abs((loss(up) - loss(down)) / (2 * step) - float(got[t, e])) <= float(bound[t, e]) + 1e-8 * (1 + T)


def test_gradient_of_a_callers_experts():
    """The same expert twice counts twice; an expert that does not exist is left out and reported."""
    z = torch.randn(4, 10, device=DEV)
    expert = torch.tensor([[3, 3], [0, 9], [-1, 2], [5, 10]], dtype=torch.int32, device=DEV)
    dw = torch.randn(4, 2, device=DEV)
    got = dgs.route_experts_grad(z, expert, dw, renormalise=False)
    assert dgs.operator_status(DEV) == dgs.DGS_EINVAL and dgs.operator_status(DEV) == 0
    s = torch.softmax(z.double(), 1)
    g = torch.zeros(4, 10, dtype=torch.float64, device=DEV)
    for t in range(4):
        for j in range(2):
            e = int(expert[t, j])
            if 0 <= e < 10:
                g[t, e] += float(dw[t, j])
    want = s * (g - (g * s).sum(1, keepdim=True))
    assert float((got.double() - want).abs().max()) < 1e-5


def test_captured_and_replayed():
    z = torch.randn(3000, 64, device=DEV)
    dw = torch.randn(3000, 4, device=DEV)
    dgs.route_experts(z, 4)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = dgs.route_experts(z, 4)
        dz = dgs.route_experts_grad(z, r.expert, dw)
    for _ in range(2):
        z.normal_()
        graph.replay()
        want = dgs.route_experts(z, 4)
        for x, y in zip(r, want):
            assert torch.equal(x, y)
        assert torch.equal(dz, dgs.route_experts_grad(z, want.expert, dw))
