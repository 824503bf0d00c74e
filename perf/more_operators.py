"""What the performance of a worker's operators around its layers is measured on: rows taken to the experts' lists and back, and the
loss over a vocabulary with its gradient.

A case is one pass through one of these operators:

  gather        dgs.gather_experts: the tokens' rows in the order of the experts' lists.
  gather_grad   dgs.gather_experts_grad: the rows' gradients added up for each token.
  combine       dgs.combine_experts: each token's rows, weighted and added up.
  combine_grad  dgs.combine_experts_grad: the gradient of the rows, in the lists' order, and of the weights.
  loss          dgs.vocabulary_loss: softmax cross entropy of hidden states against the rows of a vocabulary.
  loss_grad     dgs.vocabulary_loss_grad: its gradient, to the hidden states and to the vocabulary's slice of a flat
                gradient vector (at an odd offset, as slices behind layers of odd length lie).

Where `own` is false each is computed in its plain form from the same inputs.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "fp16": 2}


def _rows(kind, tokens, cols, k, dtype, experts=16, masked=0.0, **name):
    return dict(kind=kind, tokens=tokens, cols=cols, k=k, dtype=dtype, experts=experts, masked=masked, **name)


def _loss(kind, tokens, width, words, dtype, ignored=0.0, each=False, add=False, **name):
    return dict(kind=kind, tokens=tokens, width=width, words=words, dtype=dtype, ignored=ignored, each=each, add=add, **name)


def listed():
    return [
        # one token of a worker that evaluates while it trains: nothing but latency
        _rows("gather", 1, 768, 2, "bf16", name="gather 1x768 top2"),
        # 16 sequences of 1024 at GPT-2's width, two of 16 experts each, some of them off
        _rows("gather", 16384, 768, 2, "bf16", masked=0.05, name="gather 16384x768 top2 masked"),
        # a small odd batch in f32
        _rows("gather_grad", 777, 1000, 2, "f32", name="gather grad 777x1000 top2 f32"),
        # the same 16 sequences with many small experts
        _rows("gather_grad", 16384, 768, 8, "bf16", experts=64, name="gather grad 16384x768 top8"),
        # rows that begin anywhere, tokens with fewer experts than k
        _rows("combine", 4097, 1001, 3, "fp16", masked=0.1, name="combine 4097x1001 top3 masked"),
        # the largest: 32 sequences of 1024, rows of 2048, eight experts a token
        _rows("combine", 32768, 2048, 8, "bf16", experts=64, name="combine 32768x2048 top8"),
        # one image batch's worth of odd rows in f32
        _rows("combine_grad", 1000, 513, 2, "f32", masked=0.1, name="combine grad 1000x513 top2 f32"),
        _rows("combine_grad", 16384, 768, 8, "bf16", experts=64, name="combine grad 16384x768 top8"),
        # one token's loss against GPT-2's vocabulary: the vocabulary is read once
        _loss("loss", 1, 768, 50257, "fp16", name="loss 1x768x50257 fp16"),
        # 8 sequences of 1024 with GPT-2's head, padding ignored
        _loss("loss", 8192, 768, 50257, "bf16", ignored=0.05, name="loss 8192x768x50257"),
        # ResNet-18's fc (512 -> 1000) on an odd batch in f32, every sample with a weight of its own
        _loss("loss_grad", 37, 512, 1000, "f32", each=True, name="loss grad 37x512x1000 f32"),
        # the same 8 sequences' gradient, added to what the embedding has left (tied weights)
        _loss("loss_grad", 8192, 768, 50257, "bf16", ignored=0.05, add=True, name="loss grad 8192x768x50257"),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    kind = rng.choice(["gather", "gather_grad", "combine", "combine_grad", "loss", "loss_grad"])
    dtype = rng.choice(["f32", "bf16", "bf16", "fp16"])
    if kind in ("loss", "loss_grad"):
        width, words = _log(rng, 16, 2048), _log(rng, 100, 131072)
        most = min(8192 * 50257 // words, 8192 * 768 * 50257 // (width * words)) // (6 if dtype == "f32" else 1)
        return _loss(kind, _log(rng, 1, max(1, min(16384, most))), width, words, dtype, rng.choice([0.0, 0.05, 0.5]), rng.random() < 0.3,
                     kind == "loss_grad" and rng.random() < 0.5)
    cols = _log(rng, 1, 8192)
    if rng.random() < 0.5:
        cols = 8 * -(-cols // 8)                     # widths of models; the others begin anywhere
    experts = _log(rng, 2, 256)
    k = rng.randint(1, min(8, experts))
    tokens = _log(rng, 1, min(65536, 32768 * 2048 * 4 // (k * max(cols, 64))))
    return _rows(kind, tokens, cols, k, dtype, experts, rng.choice([0.0, 0.0, 0.1]))


# ---- inputs -----------------------------------------------------------------------------------

def _lists(c, gen):
    """What a router leaves for these tokens: experts ascending in a token, lists in the tokens' order, -1 in empty places."""
    t, e, k = c["tokens"], c["experts"], c["k"]
    z = torch.randn(t, e, generator=gen, device=DEV) + torch.randn(e, generator=gen, device=DEV) * 0.7
    chosen = z.argsort(dim=1, descending=True)[:, :k]
    if c["masked"]:
        chosen = chosen.masked_fill(torch.rand(t, k, generator=gen, device=DEV) < c["masked"], e)
        chosen = chosen.masked_fill(torch.rand(t, 1, generator=gen, device=DEV) < c["masked"] / 10, e)
    chosen = chosen.sort(1).values
    empty = chosen.reshape(-1) == e
    order = chosen.reshape(-1).argsort(stable=True)
    place = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device=DEV))
    weight = torch.rand(t, k, generator=gen, device=DEV) + 0.05
    weight = weight / weight.sum(1, keepdim=True)
    c["order"] = order.masked_fill(empty[order], -1).to(torch.int32)
    c["place"] = place.masked_fill(empty, -1).to(torch.int32).view(t, k)
    c["weight"] = weight.masked_fill(empty.view(t, k), 0.0)


def _normal(rows, cols, gen, dtype, by=1.0):
    return (torch.randn(rows, cols, generator=gen, device=DEV) * by).to(TYPE[dtype])


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    c = dict(case)
    if c["kind"] not in ("loss", "loss_grad"):
        _lists(c, gen)
        t, k, cols, dtype = c["tokens"], c["k"], c["cols"], c["dtype"]
        if c["kind"] == "gather":
            c["x"] = _normal(t, cols, gen, dtype)
        else:
            c["y"] = _normal(t * k, cols, gen, dtype, 1e-3 if c["kind"] == "gather_grad" else 1.0)
            c["y"].masked_fill_(c["order"][:, None] < 0, math.nan)               # nobody writes rows behind the last list
        if c["kind"] == "combine_grad":
            c["dout"] = _normal(t, cols, gen, dtype, 1e-3)
        return c
    n, d, v = c["tokens"], c["width"], c["words"]
    table = torch.randn(v, d, generator=gen, device=DEV) * (1.5 / math.sqrt(d))
    target = torch.randint(0, v, (n,), generator=gen, device=DEV)
    sure = torch.rand(n, 1, generator=gen, device=DEV) * 10                      # from words nobody expects to words that are certain
    hidden = torch.randn(n, d, generator=gen, device=DEV) + sure * table[target] / table[target].norm(dim=1, keepdim=True)
    if c["ignored"]:
        target = target.masked_fill(torch.rand(n, generator=gen, device=DEV) < c["ignored"], -100)
    c["hidden"], c["table"], c["target"] = hidden.to(TYPE[c["dtype"]]), table.to(TYPE[c["dtype"]]), target
    if c["kind"] == "loss_grad":
        z = c["hidden"].float() @ c["table"].float().T
        top = z.amax(1)
        c["lse"] = (z.sub_(top[:, None]).exp_().sum(1, dtype=torch.float64).log() + top).float()
        if c["each"]:
            c["dloss"] = torch.rand(n, generator=gen, device=DEV) / n
        else:
            c["dloss"] = 1.0 / (target >= 0).sum().clamp(min=1).float().view(1)  # the mean over what is not ignored
        c["gradient"] = torch.zeros(1 + v * d, device=DEV)
        if c["add"]:
            c["gradient"].normal_(generator=gen).mul_(1e-4)
        c["before"] = c["gradient"].clone() if c["add"] else None
    return c


# ---- the plain forms --------------------------------------------------------------------------

def _plain_gather(c):
    order = c["order"].long()
    y = c["x"][order.clamp(min=0) // c["k"]].masked_fill(order[:, None] < 0, 0.0)
    return {"y": y}


def _taken(c):
    """The rows of the tokens' slots [tokens, k, cols], zeros for empty ones."""
    at = c["place"].long()
    return c["y"][at.clamp(min=0)].float().masked_fill_(at[:, :, None] < 0, 0.0)


def _plain_sum(c, weighted):
    rows = _taken(c)
    return (rows.mul_(c["weight"][:, :, None]) if weighted else rows).sum(1).to(c["y"].dtype)


def _plain_combine_grad(c):
    order, k = c["order"].long(), c["k"]
    slot = order.clamp(min=0)
    dout = c["dout"].float()
    dy = (dout[slot // k] * c["weight"].reshape(-1)[slot][:, None]).masked_fill(order[:, None] < 0, 0.0)
    return {"dy": dy.to(c["y"].dtype), "dweight": _taken(c).mul_(dout[:, None, :]).sum(2)}


def _plain_loss(c):
    z = c["hidden"].float() @ c["table"].float().T
    top = z.amax(1, keepdim=True)
    lse = torch.log(torch.exp(z - top).sum(1)) + top[:, 0]
    at = c["target"].clamp(min=0)
    return {"loss": (lse - z.gather(1, at[:, None])[:, 0]).masked_fill(c["target"] < 0, 0.0), "lse": lse}


def _plain_loss_grad(c):
    hidden, table, target = c["hidden"].float(), c["table"].float(), c["target"]
    s = (hidden @ table.T).sub_(c["lse"][:, None]).exp_()
    s.scatter_add_(1, target.clamp(min=0)[:, None], torch.full((c["tokens"], 1), -1.0, device=DEV))
    s.mul_(c["dloss"].expand(c["tokens"])[:, None]).masked_fill_(target[:, None] < 0, 0.0)
    dw = s.T @ hidden
    if c["add"]:
        dw = dw + c["before"][1:].view_as(dw)
    return {"dhidden": (s @ table).to(c["hidden"].dtype), "dw": dw}


# ---- one pass ---------------------------------------------------------------------------------

def run(c):
    kind = c["kind"]
    if not own:
        if kind in ("gather_grad", "combine"):
            return {"out": _plain_sum(c, kind == "combine")}
        return {"gather": _plain_gather, "combine_grad": _plain_combine_grad, "loss": _plain_loss, "loss_grad": _plain_loss_grad}[kind](c)
    import paper_1910_10929_b200 as dgs
    if kind == "gather":
        return {"y": dgs.gather_experts(c["x"], c["order"], c["place"])}
    if kind == "gather_grad":
        return {"out": dgs.gather_experts_grad(c["y"], c["place"])}
    if kind == "combine":
        return {"out": dgs.combine_experts(c["y"], c["weight"], c["place"])}
    if kind == "combine_grad":
        dy, dweight = dgs.combine_experts_grad(c["dout"], c["y"], c["weight"], c["order"], c["place"])
        return {"dy": dy, "dweight": dweight}
    if kind == "loss":
        r = dgs.vocabulary_loss(c["hidden"], c["table"], c["target"])
        return {"loss": r.loss, "lse": r.lse}
    if c["add"]:
        c["gradient"].copy_(c["before"])                      # a pass can be made again on the same state
    dw = c["gradient"][1:]
    dhidden = dgs.vocabulary_loss_grad(c["hidden"], c["table"], c["target"], c["lse"], c["dloss"], dw, add=c["add"])
    return {"dhidden": dhidden, "dw": dw.view(c["words"], c["width"])}


def work(case):
    c, size = case, SIZE[case["dtype"]]
    if c["kind"] in ("loss", "loss_grad"):
        n, d, v = c["tokens"], c["width"], c["words"]
        if c["kind"] == "loss":
            return {"bytes": (n + v) * d * size + 16 * n, "flops": 2 * n * v * d}
        return {"bytes": (2 * n + v) * d * size + 4 * v * d * (2 if c["add"] else 1) + 12 * n + 4 * (n if c["each"] else 1), "flops": 6 * n * v * d}
    t, k, row = c["tokens"], c["k"], c["cols"] * size
    slots, n = t * k, t * k * c["cols"]
    if c["kind"] == "gather":
        return {"bytes": t * row + slots * (row + 4), "flops": 0}
    if c["kind"] == "combine_grad":
        return {"bytes": t * row + slots * (2 * row + 16), "flops": 3 * n}
    return {"bytes": t * row + slots * (row + (8 if c["kind"] == "combine" else 4)), "flops": (2 if c["kind"] == "combine" else 1) * n}


# ---- the definitions in 64 bits -----------------------------------------------------------------

def exact(case, seed):
    c = prepare(case, seed)
    kind = c["kind"]
    if kind == "gather":
        x = c["x"].double()
        slots = torch.cat([x.repeat_interleave(c["k"], 0), torch.zeros(1, c["cols"], dtype=torch.float64, device=DEV)])
        return {"y": slots[c["order"].long()]}                 # -1: the row of zeros behind the last
    if kind not in ("loss", "loss_grad"):
        t, k, cols = c["tokens"], c["k"], c["cols"]
        there = c["order"] >= 0
        slot = c["order"][there].long()
        token = torch.div(slot, k, rounding_mode="floor")
        y, w = c["y"][there].double(), c["weight"].double().view(-1)[slot]
        if kind in ("gather_grad", "combine"):
            return {"out": torch.zeros(t, cols, dtype=torch.float64, device=DEV).index_add_(0, token, y * w[:, None] if kind == "combine" else y)}
        dout = c["dout"].double()[token]
        dy = torch.zeros(t * k, cols, dtype=torch.float64, device=DEV)
        dy[there] = dout * w[:, None]
        dweight = torch.zeros(t * k, dtype=torch.float64, device=DEV)
        dweight[slot] = torch.einsum("rc,rc->r", dout, y)
        return {"dy": dy, "dweight": dweight.view(t, k)}
    hidden, table, target = c["hidden"].double(), c["table"].double(), c["target"]
    rows = torch.arange(c["tokens"], device=DEV)[target >= 0]
    if kind == "loss":
        loss, lse = [torch.zeros(c["tokens"], dtype=torch.float64, device=DEV) for _ in range(2)]
        for part in torch.arange(c["tokens"], device=DEV).split(2048):
            lse[part] = torch.logsumexp(hidden[part] @ table.T, 1)
        loss[rows] = lse[rows] - torch.einsum("rc,rc->r", hidden[rows], table[target[rows]])
        return {"loss": loss, "lse": lse}
    dhidden, dw = torch.zeros_like(hidden), torch.zeros_like(table)
    g = torch.broadcast_to(c["dloss"].double(), (c["tokens"],))
    for part in rows.split(2048):
        h, word = hidden[part], target[part]
        p = torch.exp(h @ table.T - c["lse"][part, None].double()) * g[part, None]
        dhidden[part] = p @ table - g[part, None] * table[word]
        dw += p.T @ h
        dw.index_add_(0, word, -g[part, None] * h)
    if c["add"]:
        dw += c["before"][1:].view_as(dw).double()
    return {"dhidden": dhidden, "dw": dw}
