"""Rows and vocabularies of more than 2^32 values: offsets past 32 bits, checked at rows and words from all over."""
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_rows_of_more_than_2_32_values():
    tokens, k, cols = (1 << 20) + 3, 2, 2056                       # 2 x 2056 x 2^20 = 4.3e9 values in 16 bits
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty(tokens, cols, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    order = torch.randperm(tokens * k, generator=g, device=DEV)
    place = torch.empty_like(order)
    place[order] = torch.arange(tokens * k, device=DEV)
    order, place = order.to(torch.int32), place.to(torch.int32).view(tokens, k)
    y = dgs.gather_experts(x, order, place)
    assert y.numel() > 1 << 32
    at = torch.cat([torch.arange(50, device=DEV), torch.randint(0, tokens * k, (500,), generator=g, device=DEV), tokens * k - 1 - torch.arange(50, device=DEV)])
    assert torch.equal(y[at], x[order[at].long() // k])
    weight = torch.rand(tokens, k, generator=g, device=DEV)
    t = torch.cat([torch.arange(50, device=DEV), torch.randint(0, tokens, (500,), generator=g, device=DEV), tokens - 1 - torch.arange(50, device=DEV)])
    out = dgs.combine_experts(y, weight, place)
    want = x[t].double() * weight[t].double().sum(1, keepdim=True)
    # bfloat16 keeps 8 bits, the first of them 1: half a step is at most 2^-8 of the value, beside four roundings in f32
    assert bool(((out[t].double() - want).abs() <= want.abs() * (2.0 ** -8 * (1 + 2.0 ** -8) + 4 * 2.0 ** -24)).all())
    del out
    dy, dweight = dgs.combine_experts_grad(x, y, weight, order, place)
    want = x[order[at].long() // k].double() * weight.view(-1)[order[at].long()].double()[:, None]
    assert bool(((dy[at].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -23)).all())
    square = (x[t].double() ** 2).sum(1, keepdim=True)
    assert bool(((dweight[t].double() - square).abs() <= square * (cols / 32 + 12) * 2.0 ** -24).all())
    assert dgs.operator_status(DEV) == 0


def test_a_vocabulary_of_more_than_2_32_values():
    rows, width, words = 130, 2056, (1 << 21) + 77                # 2056 x 2^21 = 4.3e9 values
    g = torch.Generator(device=DEV).manual_seed(2)
    table = torch.empty(words, width, dtype=torch.bfloat16, device=DEV)
    for part in table.split(1 << 18):
        part.copy_(torch.randn(part.shape, generator=g, device=DEV) * 0.04)
    assert table.numel() > 1 << 32
    target = torch.randint(0, words, (rows,), generator=g, device=DEV)
    target[:3] = torch.tensor([0, words - 1, -100], device=DEV)
    hidden = (torch.randn(rows, width, generator=g, device=DEV) + table[target.clamp(min=0)].float() * 4).to(torch.bfloat16)
    got = dgs.vocabulary_loss(hidden, table, target)
    z = torch.cat([hidden.double() @ part.double().T for part in table.split(1 << 16)], 1)
    lse = torch.logsumexp(z, 1)
    # logits: sums of 2056 products, 64 additions at a time (2^-22 of the magnitudes each); exponentials and sums 2^-19 in all
    far = 2.0 ** -15 + lse.abs() * 2.0 ** -22
    assert bool(((got.lse.double() - lse).abs() <= far).all())
    live = target >= 0
    want = torch.where(live, lse - z.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    assert bool(((got.loss.double() - want).abs() <= 2 * far).all())
    dloss = torch.rand(rows, generator=g, device=DEV)
    dw = torch.empty(words * width, device=DEV)
    dh = dgs.vocabulary_loss_grad(hidden, table, target, got.lse, dloss, dw)
    assert dgs.operator_status(DEV) == 0
    s = torch.exp(z - got.lse.double()[:, None])
    s[live] = s[live].scatter_add_(1, target[live][:, None], torch.full((int(live.sum()), 1), -1.0, dtype=torch.float64, device=DEV))
    s *= (dloss * live).double()[:, None]
    del z
    at = torch.cat([target[live], torch.arange(300, device=DEV), torch.randint(0, words, (2000,), generator=g, device=DEV), words - 1 - torch.arange(300, device=DEV)])
    h = torch.where(live[:, None], hidden.double(), 0.0)
    want, size = s[:, at].T @ h, s[:, at].abs().T @ h.abs()
    # s: its logit's error and 22 bits, and 2^-40 of the largest dloss; sums of 130 rows in two parts
    near = size * 2.0 ** -14 + 2.0 ** -38 * h.abs().sum(0)
    assert bool(((dw.view(words, width)[at].double() - want).abs() <= near).all())
    want, size = torch.zeros_like(h), torch.zeros_like(h)
    for i, part in enumerate(table.split(1 << 16)):
        mine = s[:, i << 16:(i << 16) + part.shape[0]]
        want += mine @ part.double()
        size += mine.abs() @ part.double().abs()
    near = size * (2.0 ** -11 + 2.0 ** -14) + want.abs() * 2.0 ** -8 + 2.0 ** -38 * 2.0 ** 21
    assert bool(((dh.double() - want).abs() <= near).all())
