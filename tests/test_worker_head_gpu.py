"""A worker's whole step with the operators in the order in which a model with experts uses them: embed, route, take the rows to the experts' lists, the experts' layer,
weigh and bring them back, the loss over the vocabulary, and back again into one flat gradient that the push takes.  The gradient is compared with 64-bit differentiation of the
same network, and the push with the oracle."""
import numpy as np
import pytest
import torch

import oracle
import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T, D, E, K = 300, 56, 5, 2


def cut(flat, words):
    """The flat vector's layers: three numbers, the router [E, D], the experts' layers [E, D, D] (out, in) and biases [E, D], the vocabulary [words, D] that embeds too."""
    at, parts = 3, {}
    for name, shape in (("router", (E, D)), ("w", (E, D, D)), ("b", (E, D)), ("table", (words, D))):
        n = int(np.prod(shape))
        parts[name] = flat[at:at + n].view(shape)
        at += n
    return parts, at


def forward64(p, ids, expert, target, weights):
    x = p["table"][ids]
    s = torch.softmax(x @ p["router"].T, 1)
    w = s.gather(1, expert)
    w = w / w.sum(1, keepdim=True)
    out = x
    for e in range(E):
        t, j = torch.nonzero(expert == e, as_tuple=True)
        h = x[t] @ p["w"][e].T + p["b"][e]
        out = out.index_add(0, t, w[t, j, None] * h * torch.sigmoid(h))
    z = out @ p["table"].T
    live = target >= 0
    nll = torch.logsumexp(z, 1) - z.gather(1, target.clamp(min=0)[:, None])[:, 0]
    return (nll * weights * live).sum()


@pytest.mark.parametrize("words", [211, 5000])                      # the head without tensor cores and with them
def test_from_tokens_to_packets(words):
    gen = torch.Generator(device=DEV).manual_seed(words)
    size = cut(torch.empty(1 << 22), words)[1]
    theta = torch.randn(size, generator=gen, device=DEV) * 0.25
    p, _ = cut(theta, words)
    p["table"].copy_((p["table"] * 64).round().clamp(-100, 100) / 64)   # embedded rows that 8 bits hold exactly
    ids = torch.randint(0, words, (T,), generator=gen, device=DEV)
    target = torch.randint(0, words, (T,), generator=gen, device=DEV).masked_fill(torch.rand(T, generator=gen, device=DEV) < 0.1, -100)
    dloss = 1.0 / (target >= 0).sum().float().view(1)

    grad = torch.zeros(size, device=DEV)
    g, _ = cut(grad, words)
    x = p["table"][ids]
    held_x = dgs.Checkpoint(T, D, device=DEV)
    held_x.save(x)
    z = x @ p["router"].T
    r = dgs.route_experts(z, K)
    spans = [slice(*r.offsets[e:e + 2].tolist()) for e in range(E)]
    rows = dgs.gather_experts(x, r.order, r.place)
    h = torch.cat([rows[s] @ p["w"][e].T + p["b"][e] for e, s in enumerate(spans)])
    a = h * torch.sigmoid(h)
    out = x + dgs.combine_experts(a, r.weight, r.place)
    loss = dgs.vocabulary_loss(out, p["table"], target)
    # backward
    dout = dgs.vocabulary_loss_grad(out, p["table"], target, loss.lse, dloss, g["table"].view(-1))
    da, dweight = dgs.combine_experts_grad(dout, a, r.weight, r.order, r.place)
    s = torch.sigmoid(h)
    dh = da * s * (1 + h * (1 - s))
    held_x.weight_grad(dh, g["w"].view(-1), g["b"].view(-1), offsets=r.offsets, rows=r.order, rows_per=K)
    drows = torch.cat([dh[q] @ p["w"][e] for e, q in enumerate(spans)])
    dz = dgs.route_experts_grad(z, r.expert, dweight)
    held_x.weight_grad(dz, g["router"].view(-1))
    dx = dout + dgs.gather_experts_grad(drows, r.place) + dz @ p["router"]
    g["table"].index_add_(0, ids, dx)
    assert dgs.operator_status(DEV) == 0

    exact = theta.double().requires_grad_(True)
    e, _ = cut(exact, words)
    total = forward64(e, ids, r.expert.long(), target, float(dloss))
    total.backward()
    mean = float((loss.loss.double() * float(dloss)).sum())
    assert abs(mean - total.item()) <= 1e-5 * abs(total.item())
    want, _ = cut(exact.grad, words)
    # f32 throughout: sums of at most 600 terms after one another in four layers, 600 * 2^-24 of their size each at the worst
    for name in want:
        assert float((g[name].double() - want[name]).norm() / want[name].norm()) <= 4 * 600 * 2.0 ** -24, name

    offset, length = [0, 3], [3, E * D]
    for n in (E * D * D, E * D, words * D):
        offset.append(offset[-1] + length[-1])
        length.append(n)
    k = [max(1, n // 20) for n in length]
    ctx = dgs.Context(size, 2, 0.1, 0.9, offset, length, k, k, theta)
    orc = oracle.Oracle(size, 2, 0.1, 0.9, offset, length, k, k, theta.cpu().numpy())
    push, pull = ctx.event(0, grad)
    (oi, ov), (qi, qv) = orc.event(0, grad.cpu().numpy())
    pi, pv = (t.cpu().numpy() for t in ctx.packet(push))
    gi, gv = (t.cpu().numpy() for t in ctx.packet(pull))
    assert np.array_equal(pi.view(np.uint32), oi) and np.array_equal(pv.view(np.uint32), ov.view(np.uint32))
    assert np.array_equal(gi.view(np.uint32), qi) and np.array_equal(gv.view(np.uint32), qv.view(np.uint32))
    assert ctx.status() == 0
    ctx.close()
