"""What the performance of a worker's own operators is measured on: what it computes between two pushes.

A case is one pass through one of these operators:

  route       dgs.route_experts: every token's experts, their weights, and the experts' lists of slots.
  route_grad  dgs.route_experts_grad: the gradient of the weights taken back to the logits.
  save        Checkpoint.save and .load: an activation is applied and its input held in 8 bits, then read back.
  act_grad    Checkpoint.activation_grad: the activation's gradient from its input as the checkpoint holds it.
  weight      Checkpoint.weight_grad: a layer's weight and bias gradient from the checkpoint of its input, written
              to the layer's slice of a flat gradient vector (at an odd offset, as layers behind biases of
              odd length lie), for one layer or for all experts of one.

Where `own` is false each is computed in its plain form from the same inputs.

A checkpoint of [rows, cols] is one byte buffer: codes [rows][cols up to a multiple of 32], then scale bytes
[rows][4 for each 128 columns begun], one byte e + 127 for each block of 32 columns; a value is code * 2^e, the code an
int8 or an e4m3 number, and 2^e the smallest power of two for which the block's largest magnitude is at most
127 * 2^e (int8) or 448 * 2^e (e4m3).
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "fp16": 2}
LARGEST = {"int8": 127.0, "e4m3": 448.0}


def _route(tokens, experts, k, dtype, score, renorm, bias=False, groups=1, kept=1, best=1, scale=1.0, masked=0.0, grad=False, **name):
    return dict(kind="route_grad" if grad else "route", tokens=tokens, experts=experts, k=k, dtype=dtype, score=score, renorm=renorm,
                bias=bias, groups=groups, kept=kept, best=best, scale=scale, masked=masked, **name)


def _save(rows, cols, dtype, fmt, act, **name):
    return dict(kind="save", rows=rows, cols=cols, dtype=dtype, fmt=fmt, act=act, **name)


def _act_grad(rows, cols, dtype, fmt, act, **name):
    return dict(kind="act_grad", rows=rows, cols=cols, dtype=dtype, fmt=fmt, act=act, **name)


def _weight(rows, inputs, outputs, dtype, fmt, layout, experts=0, k=1, add=False, **name):
    return dict(kind="weight", rows=rows, inputs=inputs, outputs=outputs, dtype=dtype, fmt=fmt, layout=layout, experts=experts, k=k,
                add=add, **name)


def listed():
    return [
        # one token of a worker that evaluates while it trains: nothing but latency
        _route(1, 64, 2, "bf16", "softmax", True, name="route 1x64 top2"),
        # one sequence batch of the GPT-2 sizes (8 x 1024), a small number of experts, some masked (experts that are off)
        _route(8192, 60, 4, "bf16", "softmax", False, masked=0.05, name="route 8192x60 top4 masked"),
        # many small experts, balance bias, groups: the largest routers in use
        _route(65536, 256, 8, "f32", "sigmoid", True, bias=True, groups=8, kept=4, best=2, scale=2.5, name="route 65536x256 top8 groups"),
        _route(65536, 256, 8, "f32", "sigmoid", True, bias=True, groups=8, kept=4, best=2, scale=2.5, grad=True,
               name="route grad 65536x256 top8"),
        # one image batch of a ResNet's last block: small and odd
        _save(1000, 513, "fp16", "e4m3", "relu", name="save 1000x513 relu"),
        # the hidden layer of a feed-forward block over 32 sequences of 1024
        _save(32768, 2048, "bf16", "int8", "gelu_tanh", name="save 32768x2048 gelu"),
        _act_grad(777, 1000, "f32", "int8", "silu", name="act grad 777x1000 silu"),
        _act_grad(32768, 2048, "bf16", "int8", "gelu_tanh", name="act grad 32768x2048 gelu"),
        # ResNet-18's fc (512 -> 1000) on an odd batch, gradients in f32
        _weight(37, 512, 1000, "f32", "int8", "out_in", name="weight 37x512x1000 f32"),
        # GPT-2's c_attn (768 -> 2304) over 8 sequences, added to what an earlier part of the batch left
        _weight(8192, 768, 2304, "bf16", "int8", "in_out", add=True, name="weight 8192x768x2304"),
        # 16 experts, two for each of 16384 tokens, of unequal length
        _weight(16384, 768, 2048, "bf16", "e4m3", "out_in", experts=16, k=2, name="weight 16 experts 768x2048"),
        # GPT-2's head: rows of 50257 elements begin anywhere
        _weight(8192, 768, 50257, "bf16", "int8", "out_in", name="weight 8192x768x50257"),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    kind = rng.choice(["route", "route_grad", "save", "act_grad", "weight", "experts"])
    dtype, fmt = rng.choice(["f32", "bf16", "fp16"]), rng.choice(["int8", "e4m3"])
    act = rng.choice(["relu", "gelu", "gelu_tanh", "silu"])
    if kind in ("route", "route_grad"):
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * _log(rng, 8, 512 // groups)
        kept = rng.randint(1, groups)
        k = rng.randint(1, min(16, experts // groups * kept))
        bias = rng.random() < 0.5
        return _route(_log(rng, 1, 65536 * 256 // max(experts, 256)), experts, k, dtype, rng.choice(["softmax", "sigmoid"]), k > 1 and rng.random() < 0.7, bias,
                      groups, kept, rng.choice([1, 2]) if groups > 1 else 1, rng.choice([1.0, 2.5]), rng.choice([0.0, 0.0, 0.1]),
                      kind == "route_grad")
    if kind in ("save", "act_grad"):
        cols = _log(rng, 1, 8192)
        rows = _log(rng, 1, 32768 * 2048 // max(cols, 2048))
        return (_save if kind == "save" else _act_grad)(rows, cols, dtype, fmt, act)
    inputs, outputs, layout, add = _log(rng, 16, 4096), _log(rng, 16, 8192), rng.choice(["out_in", "in_out"]), rng.random() < 0.3
    if kind == "experts":
        experts = rng.randint(2, 32)
        inputs, outputs = min(inputs, 2048), min(outputs, 2048)
        k = rng.randint(1, min(4, experts))
        return _weight(_log(rng, 1, 16384 * 2 // k), inputs, outputs, dtype, fmt, layout, experts, k, add)
    return _weight(_log(rng, 1, min(32768, 8192 * 768 * 8192 // (inputs * outputs))), inputs, outputs, dtype, fmt, layout, 0, 1, add)


# ---- the checkpoint's format ------------------------------------------------------------------

def _encode(x, fmt):
    """(codes uint8 [rows, cols up to 32], scale bytes [rows, 4 per 128 columns])"""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    v = torch.zeros(rows, blocks * 32, dtype=torch.float32, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, blocks, 32)
    m, ex = torch.frexp(v.abs().amax(2))                     # amax = m * 2^ex, 0.5 <= m < 1
    top = LARGEST[fmt]
    tm, te = math.frexp(top)
    e = ex.to(torch.int32) - te + (m > tm).to(torch.int32)
    e = torch.where(m == 0, -127, e).clamp(-126 if fmt == "int8" else -117, 121 if fmt == "int8" else 119)
    w = torch.ldexp(v, -e[:, :, None]).clamp(-top, top)
    codes = torch.round(w).to(torch.int8).view(torch.uint8) if fmt == "int8" else w.to(torch.float8_e4m3fn).view(torch.uint8)
    scales = torch.zeros(rows, 4 * -(-cols // 128), dtype=torch.uint8, device=x.device)
    scales[:, :blocks] = (e + 127).to(torch.uint8)
    return codes.view(rows, blocks * 32), scales


def _decode(codes, scales, cols, fmt):
    rows, width = codes.shape
    q = codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).to(torch.float32).view(rows, width // 32, 32)
    e = scales[:, :width // 32].to(torch.int32) - 127
    return torch.ldexp(q, e[:, :, None]).view(rows, width)[:, :cols]


def _pack(x, fmt):
    codes, scales = _encode(x, fmt)
    return torch.cat([codes.reshape(-1), scales.reshape(-1)])


def _unpack(data, rows, cols, fmt):
    width = 32 * -(-cols // 32)
    return _decode(data[:rows * width].view(rows, width), data[rows * width:].view(rows, -1), cols, fmt)


# ---- inputs -----------------------------------------------------------------------------------

def _activations(rows, cols, gen):
    """Roughly normal, with a few channels that are far larger than the others, as hidden states have."""
    x = torch.randn(rows, cols, generator=gen, device=DEV)
    big = torch.rand(cols, generator=gen, device=DEV) < 0.01
    return x.mul_(torch.where(big, 12.0, 1.0))


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    c = dict(case)
    if c["kind"] in ("route", "route_grad"):
        t, e = c["tokens"], c["experts"]
        z = torch.randn(t, e, generator=gen, device=DEV) * 1.5 + torch.randn(e, generator=gen, device=DEV) * 0.7
        if c["masked"]:
            z.masked_fill_(torch.rand(t, e, generator=gen, device=DEV) < c["masked"], -math.inf)
            z.masked_fill_(torch.rand(t, 1, generator=gen, device=DEV) < c["masked"] / 10, -math.inf)
        c["logits"] = z.to(TYPE[c["dtype"]])
        c["balance"] = torch.randn(e, generator=gen, device=DEV) * 0.05 if c["bias"] else None
        if c["kind"] == "route_grad":
            c["expert"] = _choose(c["logits"], c["balance"], c)
            c["dweight"] = torch.randn(t, c["k"], generator=gen, device=DEV)
    elif c["kind"] == "save":
        c["x"] = _activations(c["rows"], c["cols"], gen).to(TYPE[c["dtype"]])
    elif c["kind"] == "act_grad":
        c["data"] = _pack(_activations(c["rows"], c["cols"], gen), c["fmt"])
        c["dy"] = (torch.randn(c["rows"], c["cols"], generator=gen, device=DEV) * 1e-3).to(TYPE[c["dtype"]])
    else:
        n, e = c["rows"], max(1, c["experts"])
        c["data"] = _pack(_activations(n, c["inputs"], gen), c["fmt"])
        c["dy"] = (torch.randn(n * c["k"], c["outputs"], generator=gen, device=DEV) * 1e-3).to(TYPE[c["dtype"]])
        w = e * c["inputs"] * c["outputs"]
        c["gradient"] = torch.zeros(1 + w + e * c["outputs"], device=DEV)        # an odd offset, then weights and biases
        if c["add"]:
            c["gradient"].normal_(generator=gen).mul_(1e-3)
        c["before"] = c["gradient"].clone() if c["add"] else None
        if c["experts"]:
            z = torch.randn(n, e, generator=gen, device=DEV) + torch.randn(e, generator=gen, device=DEV) * 0.7
            chosen = z.argsort(dim=1, descending=True)[:, :c["k"]].sort(1).values.reshape(-1)
            c["order"] = chosen.argsort(stable=True).to(torch.int32)
            counts = torch.bincount(chosen, minlength=e)
            c["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
            c["most"] = int(counts.max())                                         # a program that pads the experts' rows knows it
    return c


# ---- the plain forms --------------------------------------------------------------------------

def _choose(z, bias, c):
    """The chosen experts of every token, ascending, -1 behind the last.  In 64 bits: keys may be next to one another."""
    t, e = z.shape
    z = z.double()
    free = z > -math.inf
    s = torch.sigmoid(z) if c["score"] == "sigmoid" else torch.softmax(z.masked_fill(~free.any(1, keepdim=True), 0.0), 1)
    key = s + bias.double() if bias is not None else z if c["best"] == 1 else s
    key = key.masked_fill(~free, -math.inf)
    if c["groups"] > 1:
        parts = key.view(t, c["groups"], -1)
        top = parts.sort(dim=2, descending=True).values[:, :, :c["best"]]
        total = top.masked_fill(top == -math.inf, 0.0).sum(2).masked_fill(top[:, :, 0] == -math.inf, -math.inf)
        kept = total.sort(dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        stays = torch.zeros(t, c["groups"], dtype=torch.bool, device=z.device).scatter_(1, kept, True)
        key = parts.masked_fill(~stays[:, :, None], -math.inf).view(t, e)
    best = key.sort(dim=1, descending=True, stable=True)
    chosen = best.indices[:, :c["k"]].masked_fill(best.values[:, :c["k"]] == -math.inf, e).sort(1).values
    return chosen.masked_fill(chosen == e, -1).to(torch.int32)


def _plain_route(c):
    z, e, k = c["logits"], c["experts"], c["k"]
    expert = _choose(z, c["balance"], c)
    there = expert >= 0
    z = z.float()
    at = expert.clamp(min=0).long()
    if c["score"] == "sigmoid":
        w = torch.sigmoid(z).gather(1, at).masked_fill(~there, 0.0)
    else:
        w = torch.softmax(z, 1).gather(1, at).masked_fill(~there, 0.0)
    if c["renorm"]:
        total = w.sum(1, keepdim=True)
        w = w / total.masked_fill(total == 0, 1.0)
    bins = expert.reshape(-1).masked_fill(~there.reshape(-1), e).long()
    order = bins.argsort(stable=True)
    place = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device=z.device))
    empty = ~there.reshape(-1)
    counts = torch.bincount(bins, minlength=e + 1)[:e]
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return {"expert": expert, "weight": w * c["scale"], "offsets": offsets.to(torch.int32),
            "order": order.masked_fill(empty[order], -1).to(torch.int32), "place": place.masked_fill(empty, -1).to(torch.int32)}


def _plain_route_grad(c):
    z, at = c["logits"].float(), c["expert"].clamp(min=0).long()
    there = c["expert"] >= 0
    g = (c["dweight"] * c["scale"]).masked_fill(~there, 0.0)
    if c["score"] == "sigmoid":
        s = torch.sigmoid(z)
        slope = s * (1 - s)
    else:
        s = torch.softmax(z, 1).masked_fill(~(z > -math.inf).any(1, keepdim=True), 0.0)
        slope = None
    w = s.gather(1, at).masked_fill(~there, 0.0)
    if c["renorm"]:
        total = w.sum(1, keepdim=True)
        total = total.masked_fill(total == 0, 1.0)
        g = (g - (g * w).sum(1, keepdim=True) / total) / total
    ds = torch.zeros_like(z).scatter_add_(1, at, g.masked_fill(~there, 0.0))
    dz = ds * slope if slope is not None else s * (ds - (ds * s).sum(1, keepdim=True))
    return {"dlogits": dz.to(c["logits"].dtype)}


def _act(act, x):
    if act == "relu":
        return x.clamp(min=0)
    if act == "silu":
        return x * torch.sigmoid(x)
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))


def _act_slope(act, x):
    if act == "relu":
        return (x > 0).to(x.dtype)
    if act == "silu":
        s = torch.sigmoid(x)
        return s * (1 + x * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    a = math.sqrt(2 / math.pi)
    t = torch.tanh(a * (x + 0.044715 * x * x * x))
    return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * a * (1 + 3 * 0.044715 * x * x)


def _plain_save(c):
    x = c["x"].float()
    codes, scales = _encode(x, c["fmt"])
    return {"y": _act(c["act"], x).to(c["x"].dtype), "held": _decode(codes, scales, c["cols"], c["fmt"]).to(c["x"].dtype)}


def _plain_act_grad(c):
    x = _unpack(c["data"], c["rows"], c["cols"], c["fmt"])
    return {"dx": (c["dy"].float() * _act_slope(c["act"], x)).to(c["dy"].dtype)}


def _plain_weight(c):
    x, dy, e = _unpack(c["data"], c["rows"], c["inputs"], c["fmt"]), c["dy"].float(), c["experts"]
    if e:                                                     # the experts' rows side by side, filled up with zeros
        row = torch.arange(c["most"], device=DEV)
        first, last = c["offsets"][:-1, None].long(), c["offsets"][1:, None].long()
        there = (first + row < last)[:, :, None]
        at = (first + row).clamp(max=dy.shape[0] - 1)
        x = x[c["order"].long()[at] // c["k"]]
        dy = dy[at] * there
        db = dy.sum(1)
    else:
        x, dy = x[None], dy[None]
        db = dy.sum(1)
    dw = torch.bmm(dy.transpose(1, 2), x) if c["layout"] == "out_in" else torch.bmm(x.transpose(1, 2), dy)
    if c["add"]:
        old = c["before"]
        dw = dw + old[1:1 + dw.numel()].view_as(dw)
        db = db + old[1 + dw.numel():].view_as(db)
    return {"dw": dw, "db": db}


# ---- one pass ---------------------------------------------------------------------------------

def run(c):
    if not own:
        return {"route": _plain_route, "route_grad": _plain_route_grad, "save": _plain_save, "act_grad": _plain_act_grad,
                "weight": _plain_weight}[c["kind"]](c)
    import paper_1910_10929_b200 as dgs
    if c["kind"] == "route":
        r = dgs.route_experts(c["logits"], c["k"], score=c["score"], bias=c["balance"], groups=c["groups"], groups_kept=c["kept"],
                              group_best=c["best"], renormalise=c["renorm"], scale=c["scale"])
        return {"expert": r.expert, "weight": r.weight, "offsets": r.offsets, "order": r.order, "place": r.place.view(-1)}
    if c["kind"] == "route_grad":
        return {"dlogits": dgs.route_experts_grad(c["logits"], c["expert"], c["dweight"], score=c["score"], renormalise=c["renorm"],
                                                  scale=c["scale"])}
    if c["kind"] == "save":
        held = dgs.Checkpoint(c["rows"], c["cols"], c["fmt"], device=c["x"].device)
        y = held.save(c["x"], activation=c["act"])
        return {"y": y, "held": held.load(c["x"].dtype)}
    if c["kind"] == "act_grad":
        held = dgs.Checkpoint(c["rows"], c["cols"], c["fmt"], data=c["data"])
        return {"dx": held.activation_grad(c["dy"], c["act"])}
    held = dgs.Checkpoint(c["rows"], c["inputs"], c["fmt"], data=c["data"])
    e = max(1, c["experts"])
    split = 1 + e * c["inputs"] * c["outputs"]
    dw, db = c["gradient"][1:split], c["gradient"][split:]
    if c["add"]:
        c["gradient"].copy_(c["before"])                      # a pass can be made again on the same state
    lists = dict(offsets=c["offsets"], rows=c["order"], rows_per=c["k"]) if c["experts"] else {}
    held.weight_grad(c["dy"], dw, db, layout=c["layout"], add=c["add"], **lists)
    shape = (e, c["outputs"], c["inputs"]) if c["layout"] == "out_in" else (e, c["inputs"], c["outputs"])
    return {"dw": dw.view(shape), "db": db.view(e, c["outputs"])}


def work(case):
    c = case
    if c["kind"] in ("route", "route_grad"):
        t, e, k, size = c["tokens"], c["experts"], c["k"], SIZE[c["dtype"]]
        if c["kind"] == "route":
            return {"bytes": t * e * size + 16 * t * k + 4 * (e + 1) + (4 * e if c["bias"] else 0), "flops": 10 * t * e}
        return {"bytes": 2 * t * e * size + 8 * t * k, "flops": 10 * t * e}
    if c["kind"] in ("save", "act_grad"):
        n, size = c["rows"] * c["cols"], SIZE[c["dtype"]]
        held = c["rows"] * (32 * -(-c["cols"] // 32) + 4 * -(-c["cols"] // 128))
        if c["kind"] == "save":
            return {"bytes": 3 * n * size + 2 * held, "flops": 25 * n}
        return {"bytes": 2 * n * size + held, "flops": 25 * n}
    n, i, o, e = c["rows"], c["inputs"], c["outputs"], max(1, c["experts"])
    held = n * (32 * -(-i // 32) + 4 * -(-i // 128))
    lists = 4 * n * c["k"] + 4 * (e + 1) if c["experts"] else 0
    result = 4 * e * o * (i + 1) * (2 if c["add"] else 1)
    return {"bytes": held + n * c["k"] * o * SIZE[c["dtype"]] + lists + result, "flops": 2 * n * c["k"] * i * o}


# ---- the definitions in 64 bits -----------------------------------------------------------------

def _exact_held(x, fmt):
    """What a checkpoint of x holds: the exponents by logarithm and comparison, the codes by a grid of steps."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -cols % 32)).view(rows, -1, 32)
    top = LARGEST[fmt]
    largest = v.abs().amax(2, keepdim=True)
    e = torch.ceil(torch.log2(largest.clamp(min=1e-300) / top))
    e = torch.where(largest > top * torch.exp2(e), e + 1, e)
    e = torch.where(largest <= top * torch.exp2(e - 1), e - 1, e)
    e = e.clamp(-126 if fmt == "int8" else -117, 121 if fmt == "int8" else 119)
    w = v / torch.exp2(e)
    if fmt == "int8":
        step = torch.ones_like(w)
    else:
        low = torch.floor(torch.log2(w.abs().clamp(min=2.0 ** -6)))
        step = torch.exp2(low - 3)
    w = (torch.round(w / step) * step).clamp(-top, top)
    return (w * torch.exp2(e)).reshape(rows, -1)[:, :cols]


def _exact_bytes(data, rows, cols, fmt):
    """The values of a checkpoint's bytes, from the bits."""
    width = 32 * -(-cols // 32)
    b = data[:rows * width].view(rows, width).to(torch.int64)
    e = data[rows * width:].view(rows, -1).to(torch.int64)[:, :width // 32].repeat_interleave(32, 1) - 127
    if fmt == "int8":
        q = (b - 256 * (b >= 128)).double()
    else:
        x, m = (b >> 3) & 15, b & 7
        q = torch.where(x == 0, m * 2.0 ** -9, (8 + m).double() * torch.exp2((x - 10).double())) * torch.where(b >= 128, -1.0, 1.0)
    return (q * torch.exp2(e.double()))[:, :cols]


def _exact_first(key, count):
    """The `count` largest keys of every row, the first of equal ones, without those at -inf: where they are."""
    border = key.topk(count, 1).values[:, -1:]
    above, level = key > border, key == border
    return (above | (level & (level.cumsum(1) <= count - above.sum(1, keepdim=True)))) & (key > -math.inf)


def _exact_choose(z, s, c):
    t, e = z.shape
    key = z if c["balance"] is None and c["best"] == 1 else s if c["balance"] is None else s + c["balance"].double()
    key = torch.where(z > -math.inf, key, -math.inf)
    if c["groups"] > 1:
        top = key.view(t, c["groups"], -1).topk(min(c["best"], e // c["groups"]), 2).values
        total = torch.where(top[:, :, 0] > -math.inf, torch.where(top > -math.inf, top, 0.0).sum(2), -math.inf)
        key = torch.where(_exact_first(total, c["kept"]).repeat_interleave(e // c["groups"], 1), key, -math.inf)
    at = torch.where(_exact_first(key, c["k"]), torch.arange(e, device=DEV), e)
    return at.topk(c["k"], 1, largest=False).values.sort(1).values


def _exact_act(act, x):
    if act == "relu":
        return torch.where(x > 0, x, 0.0)
    if act == "gelu":
        return x * 0.5 * torch.erfc(-x / math.sqrt(2))
    return x / (1 + torch.exp(-x if act == "silu" else -2 * math.sqrt(2 / math.pi) * x * (1 + 0.044715 * x * x)))


def _exact_act_slope(act, x):
    if act == "relu":
        return torch.where(x > 0, 1.0, 0.0)
    if act == "gelu":
        return 0.5 * torch.erfc(-x / math.sqrt(2)) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    inner = x if act == "silu" else 2 * math.sqrt(2 / math.pi) * x * (1 + 0.044715 * x * x)
    slope = 1.0 if act == "silu" else 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * x * x)
    return 1 / (1 + torch.exp(-inner)) + x * slope / (1 + torch.exp(-inner)) / (1 + torch.exp(inner))


def exact(case, seed):
    c = prepare(case, seed)
    if c["kind"] in ("route", "route_grad"):
        z = c["logits"].double()
        if c["score"] == "sigmoid":
            s = 1 / (1 + torch.exp(-z))
        else:
            s = torch.exp(z - z.clamp(min=-1e300).amax(1, keepdim=True))
            s = s / s.sum(1, keepdim=True).clamp(min=1e-300)
        expert = _exact_choose(z, s, c) if c["kind"] == "route" else c["expert"]
        chosen = torch.zeros(z.shape[0], z.shape[1] + 1, dtype=torch.bool, device=DEV)
        chosen.scatter_(1, expert.long() % (z.shape[1] + 1), True)
        chosen = chosen[:, :-1]
        part = s * chosen
        total = part.sum(1, keepdim=True).clamp(min=1e-300) if c["renorm"] else torch.ones_like(s[:, :1])
        p = part / total
        if c["kind"] == "route":
            w = torch.cat([p, torch.zeros_like(p[:, :1])], 1).gather(1, expert.long() % (z.shape[1] + 1)) * c["scale"]
            return {"expert": None, "weight": w, "offsets": None, "order": None, "place": None}
        g = torch.zeros(z.shape[0], z.shape[1] + 1, dtype=torch.float64, device=DEV)
        g = g.scatter(1, expert.long() % (z.shape[1] + 1), c["dweight"].double() * c["scale"])[:, :-1]
        pull = (g * p).sum(1, keepdim=True)
        if c["score"] == "sigmoid":
            dz = (g - pull if c["renorm"] else g) * p * (1 - s)
        else:
            dz = p * (g - pull) if c["renorm"] else s * (g * chosen - pull)
        return {"dlogits": dz}
    if c["kind"] == "save":
        return {"y": _exact_act(c["act"], c["x"].double()), "held": _exact_held(c["x"], c["fmt"])}
    if c["kind"] == "act_grad":
        return {"dx": c["dy"].double() * _exact_act_slope(c["act"], _exact_bytes(c["data"], c["rows"], c["cols"], c["fmt"]))}
    x, dy, e = _exact_bytes(c["data"], c["rows"], c["inputs"], c["fmt"]), c["dy"], c["experts"]
    dws, dbs = [], []
    cut = c["offsets"].tolist() if e else [0, c["rows"]]
    for first, last in zip(cut[:-1], cut[1:]):
        d = dy[first:last].double()
        xe = x[c["order"][first:last].long() // c["k"]] if e else x
        dws.append(d.T @ xe if c["layout"] == "out_in" else xe.T @ d)
        dbs.append(d.sum(0))
    dw, db = torch.stack(dws), torch.stack(dbs)
    if c["add"]:
        old = c["before"].double()
        dw += old[1:1 + dw.numel()].view_as(dw)
        db += old[1 + dw.numel():].view_as(db)
    return {"dw": dw, "db": db}
