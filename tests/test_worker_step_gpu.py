"""The operators of a worker's own computation together, as a worker of a model with experts uses them between two pushes: route, hold the
inputs in 8 bits, apply an activation, form every layer's gradient in its slice of the flat vector, push.  The gradient is compared with the one that
64-bit differentiation of the same network gives, and what the push makes of it with the oracle, bit for bit."""
import numpy as np
import pytest
import torch

import oracle
import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T, D, F, E, K = 300, 48, 72, 5, 2     # tokens, width, hidden width, experts, experts a token


class Layers:
    """A flat vector cut into layers: router [E, D], first [E, D, F] (in, out), its bias [E, F], second [E, D, F] (out, in), bias [E, D], scale [3]."""

    def __init__(self, flat):
        self.flat, at = flat, 3                           # an odd offset before everything else
        self.seg = [(0, 3)]
        for name, shape in (("router", (E, D)), ("w1", (E, D, F)), ("b1", (E, F)), ("w2", (E, D, F)), ("b2", (E, D))):
            n = int(np.prod(shape))
            setattr(self, name, flat[at:at + n].view(shape))
            self.seg.append((at, n))
            at += n
        assert at == flat.numel()

    @staticmethod
    def size():
        return 3 + E * D + 2 * E * D * F + E * F + E * D


def forward64(p, x, held, expert, loss_to):
    """The loss in 64 bits with the choice of experts held fixed; held: what the checkpoints hold, as constants added on."""
    z = x @ p.router.T
    s = torch.softmax(z, 1)
    w = torch.where(expert >= 0, s.gather(1, expert.clamp(min=0)), 0.0)
    w = w / w.sum(1, keepdim=True)
    y = torch.zeros(T, D, dtype=torch.float64, device=DEV)
    for e in range(E):
        t, j = torch.nonzero(expert == e, as_tuple=True)
        h = x[t] @ p.w1[e] + p.b1[e]
        a = 0.5 * h * (1 + torch.erf(h * 0.5 ** 0.5))
        y = y.index_add(0, t, w[t, j, None] * (a @ p.w2[e].T + p.b2[e]))
    return (y * loss_to).sum()


def worker_gradient(p, x, loss_to, grad):
    """The gradient of sum(y * loss_to), by the operators; matrix products by torch, as a worker's model would have them."""
    g = Layers(grad)
    z = x @ p.router.T
    r = dgs.route_experts(z, K)
    rows = r.order // K
    cut = r.offsets.tolist()
    spans = [slice(cut[e], cut[e + 1]) for e in range(E)]
    held_x = dgs.Checkpoint(T, D, device=DEV)
    held_x.save(x)                                        # one row a token, however many experts take it
    h = torch.cat([x[rows[s].long()] @ p.w1[e] + p.b1[e] for e, s in enumerate(spans)])
    held_h = dgs.Checkpoint(T * K, F, device=DEV)
    a = held_h.save(h, "gelu")
    held_a = dgs.Checkpoint(T * K, F, device=DEV)
    held_a.save(a)
    out = torch.cat([a[s] @ p.w2[e].T + p.b2[e] for e, s in enumerate(spans)])
    w = r.weight.reshape(-1)[r.order.long()]
    # backward
    dy = loss_to[rows.long()]
    dout = dy * w[:, None]
    dweight = (dy * out).sum(1)[r.place.reshape(-1).long()].view(T, K)
    held_a.weight_grad(dout, g.w2.reshape(-1), g.b2.reshape(-1), offsets=r.offsets)
    da = torch.cat([dout[s] @ p.w2[e] for e, s in enumerate(spans)])
    dh = held_h.activation_grad(da, "gelu")
    held_x.weight_grad(dh, g.w1.reshape(-1), g.b1.reshape(-1), layout="in_out", offsets=r.offsets, rows=r.order, rows_per=K)
    dz = dgs.route_experts_grad(z, r.expert, dweight)
    held_x.weight_grad(dz, g.router.reshape(-1))
    return r, (held_x, held_h, held_a)


def test_a_worker_with_experts_from_tokens_to_packets():
    gen = torch.Generator(device=DEV).manual_seed(7)
    n = Layers.size()
    theta = torch.randn(n, generator=gen, device=DEV) * 0.2
    p = Layers(theta)
    # inputs and weights that 8 bits hold exactly: the only rounding that differs from 64 bits in a large way is then that of h and a
    x = torch.randint(-60, 61, (T, D), generator=gen, device=DEV).float() / 64
    loss_to = torch.randn(T, D, generator=gen, device=DEV)
    grad = torch.zeros(n, device=DEV)
    r, (held_x, held_h, held_a) = worker_gradient(p, x, loss_to, grad)
    assert dgs.operator_status(DEV) == 0
    exact = theta.double().requires_grad_(True)
    forward64(Layers(exact), x.double(), None, r.expert.long(), loss_to.double()).backward()
    got, want = Layers(grad.double()), Layers(exact.grad)
    assert torch.equal(held_x.load(), x)
    # b2 and the router see no 8-bit value but x: f32 roundings only, of sums of at most 600 terms: 600 * 2^-24 of their size at the worst
    for name, bound in (("b2", 600 * 2.0 ** -24), ("router", 4 * 600 * 2.0 ** -24)):
        a, b = getattr(got, name), getattr(want, name)
        assert float((a - b).norm() / b.norm()) < bound, name
    # the others see h or a held to 1/127 of a block's largest value: in the mean over a block's values (largest 2.5 of their size) an error of
    # 2.5 / 127 / sqrt(3) = 1.1e-2 at the worst exponent, and gelu' changes by at most 1.13 of what h does, on a slope of 0.6 in the mean
    for name, bound in (("w2", 0.012), ("w1", 0.022), ("b1", 0.022)):
        a, b = getattr(got, name), getattr(want, name)
        assert float((a - b).norm() / b.norm()) < bound, name
    # and they are the products of what is held, to f32 roundings
    spans = [slice(*r.offsets[e:e + 2].tolist()) for e in range(E)]
    dout = loss_to[(r.order // K).long()] * r.weight.reshape(-1)[r.order.long()][:, None]
    for e, s in enumerate(spans):
        w2 = dout[s].double().T @ held_a.load()[s].double()
        assert float((got.w2[e] - w2).norm()) <= 600 * 2.0 ** -24 * float(w2.norm()) + 1e-30
    # the push of that gradient, against the oracle
    seg = Layers(theta).seg
    off, length = [s[0] for s in seg], [s[1] for s in seg]
    k = [max(1, v // 20) for v in length]
    ctx = dgs.Context(n, 2, 0.1, 0.9, off, length, k, k, theta)
    orc = oracle.Oracle(n, 2, 0.1, 0.9, off, length, k, k, theta.cpu().numpy())
    for worker in (0, 1, 0):
        push, pull = ctx.event(worker, grad)
        (oi, ov), (qi, qv) = orc.event(worker, grad.cpu().numpy())
        pi, pv = (v.cpu().numpy() for v in ctx.packet(push))
        gi, gv = (v.cpu().numpy() for v in ctx.packet(pull))
        assert np.array_equal(pi.view(np.uint32), oi) and np.array_equal(pv.view(np.uint32), ov.view(np.uint32))
        assert np.array_equal(gi.view(np.uint32), qi) and np.array_equal(gv.view(np.uint32), qv.view(np.uint32))
    assert ctx.status() == 0
    ctx.close()


def test_gradients_of_two_micro_batches_add_up_in_the_flat_vector():
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randint(-50, 51, (200, D), generator=gen, device=DEV).float()
    dy = torch.randint(-3, 4, (200, F), generator=gen, device=DEV).to(torch.bfloat16)
    flat = torch.zeros(1 + D * F + F, device=DEV)
    for half in (slice(0, 100), slice(100, 200)):
        c = dgs.Checkpoint(100, D, device=DEV)
        c.save(x[half])
        c.weight_grad(dy[half], flat[1:1 + D * F], flat[1 + D * F:], layout="in_out", add=True)
    assert torch.equal(flat[1:1 + D * F].view(D, F).double(), x.double().T @ dy.double())
    assert torch.equal(flat[1 + D * F:].double(), dy.double().sum(0)) and float(flat[0]) == 0.0
