"""Torch-backed calls of a worker's own operators (include/dgs.h, "what a worker computes before its push"):
activations held in 8 bits and the gradients formed from them, the router of a model with experts, rows taken to its lists and back, and the loss over a vocabulary.

Outputs and workspaces are torch tensors of the inputs' device, and work is enqueued on that device's current
stream, whichever device is current for the caller; as with torch's own operators, a tensor used on another stream
than the one it was made on has to be ordered and recorded by the caller.  Nothing waits for the GPU.  They are not
part of torch's differentiation: a backward pass calls them by name.  Where torch would record a call's result (an activation, a router's
weights), the call warns that it is cut off.  Arguments that do not fit raise ValueError
before any work is enqueued, what the library refuses raises DgsError.
"""
from __future__ import annotations

import functools
import warnings
from typing import NamedTuple, Optional

import torch

import paper_1910_10929_b200 as dgs

_TYPE = {torch.float32: dgs.DGS_TYPE_F32, torch.bfloat16: dgs.DGS_TYPE_BF16, torch.float16: dgs.DGS_TYPE_FP16}
_FORMAT = {"int8": dgs.DGS_FORMAT_INT8, "e4m3": dgs.DGS_FORMAT_E4M3}
_ACT = {None: dgs.DGS_ACT_NONE, "relu": dgs.DGS_ACT_RELU, "gelu": dgs.DGS_ACT_GELU, "gelu_tanh": dgs.DGS_ACT_GELU_TANH,
        "silu": dgs.DGS_ACT_SILU}
_SCORE = {"softmax": dgs.DGS_SCORE_SOFTMAX, "sigmoid": dgs.DGS_SCORE_SIGMOID}
_LAYOUT = {"out_in": 0, "in_out": dgs.DGS_WEIGHT_IN_OUT}


def _pick(table, key, what):
    try:
        return table[key]
    except (KeyError, TypeError):
        raise ValueError(f"{what} is one of {sorted(map(str, table))}: got {key!r}") from None


# What torch.cuda's own calls end in.  A torch without CUDA has neither: the package is imported all the same, and every call here refuses its tensors.
_device_now, _stream_now = getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _on_gpu(t, what):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA tensor: this library has no CPU path")


def _matrix(t: torch.Tensor, what: str) -> "dgs.dgs_matrix":
    """The last dimension as columns, all others as rows that lie evenly spaced."""
    _on_gpu(t, what)
    kind = _TYPE.get(t.dtype)
    if kind is None:
        raise ValueError(f"{what} must be float32, bfloat16 or float16: got {t.dtype}")
    shape = t.shape
    if len(shape) == 2:
        rows, cols = shape
        stride, step = t.stride()
    else:
        if not shape:
            raise ValueError(f"{what} needs a last dimension")
        cols = shape[-1]
        rows, stride, step = t.numel() // cols if cols else 0, cols, t.stride(-1)
        if rows > 1 and not t.is_contiguous():
            stride, run = None, 1                        # the rows so far: `run` of them, `stride` apart
            for n, s in zip(reversed(shape[:-1]), reversed(t.stride()[:-1])):
                if n == 1:
                    continue
                if stride is None:
                    stride = s
                elif s != stride * run:
                    raise ValueError(f"{what}: the rows of all but the last dimension must lie evenly spaced (shape {tuple(shape)}, strides {t.stride()})")
                run *= n
    if cols >= 1 << 32:                                  # it would wrap around in the library's 32 bits
        raise ValueError(f"{what} has {cols} columns: 2^32 - 1 at most")
    if step != 1 and cols > 1 and rows:
        raise ValueError(f"{what}: neighbours in the last dimension must be neighbours in memory (stride {step})")
    return dgs.dgs_matrix(t.data_ptr(), rows, stride if rows > 1 else cols, cols, kind)


def _plain(t: Optional[torch.Tensor], what: str, dtype: torch.dtype, numel: int, device) -> int:
    """The address of a contiguous tensor of that type and length (0 for None)."""
    if t is None:
        return 0
    _on_gpu(t, what)
    if t.dtype != dtype or t.numel() != numel or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of {numel} elements on {device}: got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _same_device(device, *tensors) -> None:
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"tensors of one call must be on one device: {device} and {t.device}")


def _cut_off(t: torch.Tensor, what: str, call: str) -> None:
    if t.requires_grad and torch.is_grad_enabled():
        warnings.warn(f"{what} requires a gradient, but what {call} returns is cut off from torch's differentiation: the backward pass calls "
                      "the gradient by name. Detach the argument, or call under torch.no_grad().", stacklevel=3)


def _enqueue(device, call, *args) -> None:
    """call(*args, stream) with the device current and its current stream."""
    index = device.index
    if index == _device_now():
        call(*args, _stream_now(index))
    else:
        with torch.cuda.device(device):
            call(*args, _stream_now(index))


def _run(device, name, *args) -> None:
    """_enqueue for an entry point by its name, without the binding's function in between (0.5 us of a small call's 10)."""
    index = device.index
    if index == _device_now():
        rc = getattr(dgs.lib(), name)(*args, _stream_now(index))
    else:
        with torch.cuda.device(device):
            rc = getattr(dgs.lib(), name)(*args, _stream_now(index))
    if rc:
        raise dgs.DgsError(rc, name)


def operator_status(device=None) -> int:
    """Waits for the device's current stream; the lowest status (0, DGS_EINVAL, DGS_ETIMEOUT) that kernels of these
    operators have left on the device since the last call."""
    with torch.cuda.device(device):
        return dgs.dgs_operator_status(_stream_now(_device_now()))


class Checkpoint:
    """A [rows, cols] activation held in 8 bits: int8 or e4m3 codes and a power-of-two scale for each 32 values of a row."""

    def __init__(self, rows: int, cols: int, format: str = "int8", device=None, data: Optional[torch.Tensor] = None):
        self.rows, self.cols, self.format = int(rows), int(cols), format
        code = _pick(_FORMAT, format, "format")
        if self.rows < 0 or not 1 <= self.cols < 1 << 32:
            raise ValueError(f"a checkpoint has rows >= 0 and cols >= 1 below 2^32: got {rows} x {cols}")
        size = self.rows * (-(-self.cols // 32) * 32 + -(-self.cols // 128) * 4)
        if self.rows >= 1 << 31 or self.cols > 1 << 30 or self.rows * self.cols > 1 << 40:
            size = dgs.dgs_checkpoint_bytes(self.rows, self.cols)   # raises what the library says
        if data is None:
            data = torch.empty(size, dtype=torch.uint8, device="cuda" if device is None else device)
        elif device is not None and torch.device(device) not in (data.device, torch.device(data.device.type)):
            raise ValueError(f"data is on {data.device}, not on {device}")
        _on_gpu(data, "data")
        self.device = data.device
        self._held = dgs.dgs_checkpoint(_plain(data, "data", torch.uint8, size, data.device), self.rows, self.cols, code)
        self.data = data

    def _fit(self, t: torch.Tensor, what: str) -> "dgs.dgs_matrix":
        m = _matrix(t, what)
        if m.cols != self.cols or m.rows != self.rows:
            raise ValueError(f"{what} must be {self.rows} x {self.cols}: got {tuple(t.shape)}")
        _same_device(self.device, t)
        return m

    def save(self, x: torch.Tensor, activation: Optional[str] = None, out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """Holds x.  With an activation (relu, gelu, gelu_tanh, silu) also returns act(x), written to `out` if given (which may be x)."""
        act = _pick(_ACT, activation, "activation")
        mx = self._fit(x, "x")
        if activation is None and out is not None:
            raise ValueError("out needs an activation")
        if activation is not None:
            _cut_off(x, "x", "Checkpoint.save")
        if activation is not None and out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        my = None
        if out is not None:
            my = self._fit(out, "out")
        _enqueue(self.device, dgs.dgs_checkpoint_save, self._held, mx, act, my)
        return out

    def load(self, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The values held (exact in float32 and bfloat16)."""
        if out is None:
            out = torch.empty(self.rows, self.cols, dtype=dtype, device=self.device)
        m = self._fit(out, "out")
        _enqueue(self.device, dgs.dgs_checkpoint_load, self._held, m)
        return out

    def activation_grad(self, dy: torch.Tensor, activation: str, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """dy * act'(held), of dy's type; `out` may be dy."""
        act = _pick(_ACT, activation, "activation")
        my = self._fit(dy, "dy")
        if out is None:
            out = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
        mx = self._fit(out, "out")
        _enqueue(self.device, dgs.dgs_checkpoint_activation_grad, self._held, act, my, mx)
        return out

    def weight_grad(self, dy: torch.Tensor, dw: torch.Tensor, db: Optional[torch.Tensor] = None, *, layout: str = "out_in",
                    add: bool = False, offsets: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None,
                    rows_per: int = 1) -> None:
        """The gradient of a layer whose input this is: dw[o, i] = sum_r dy[r, o] held[r, i] and db[o] = sum_r dy[r, o], written to
        (with `add`, added to) contiguous float32 tensors of that many elements, such as a layer's slice of the flat gradient.  layout: "out_in" or
        "in_out", how dw lies.  offsets (int32 [experts + 1]) and rows (int32, one for each row of dy) are lists as route_experts
        makes them: one gradient per expert, over the rows offsets[e] .. offsets[e + 1] of dy and rows[j] // rows_per of the checkpoint."""
        flags = _pick(_LAYOUT, layout, "layout") | (dgs.DGS_WEIGHT_ADD if add else 0)
        m = _matrix(dy, "dy")
        _same_device(self.device, dy)
        experts, lists = 1, None
        if offsets is not None:
            experts = offsets.numel() - 1
            if experts < 1 or not 1 <= rows_per < 1 << 32:
                raise ValueError("offsets holds experts + 1 numbers, and rows_per is at least 1 and below 2^32")
            lists = dgs.dgs_row_lists(_plain(offsets, "offsets", torch.int32, experts + 1, self.device),
                                      _plain(rows, "rows", torch.int32, m.rows, self.device), experts, rows_per)
        elif rows is not None or rows_per != 1:
            raise ValueError("rows and rows_per need offsets")
        elif m.rows != self.rows:
            raise ValueError(f"dy must have {self.rows} rows: got {m.rows}")
        pw = _plain(dw, "dw", torch.float32, experts * self.cols * m.cols, self.device)
        pb = _plain(db, "db", torch.float32, experts * m.cols, self.device)
        need = dgs.dgs_checkpoint_weight_grad_bytes(self._held, m, lists, flags)
        work = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
        _enqueue(self.device, dgs.dgs_checkpoint_weight_grad, self._held, m, lists, pw, pb, flags, work.data_ptr() if need else 0, need)


class Route(NamedTuple):
    """What route_experts returns; all but weight int32, -1 (DGS_NO_EXPERT) in empty places."""
    expert: torch.Tensor    # [tokens, k], ascending in a row
    weight: torch.Tensor    # [tokens, k] float32
    offsets: torch.Tensor   # [experts + 1]: expert e's slots are order[offsets[e]:offsets[e + 1]]
    order: torch.Tensor     # [tokens * k]: slots t * k + j
    place: torch.Tensor     # [tokens, k]: where in order a slot stands


@functools.lru_cache(maxsize=64)
def _router_of(k: int, score: str, groups: int, groups_kept: int, group_best: int, renormalise: bool, scale: float) -> "dgs.dgs_router":
    for v, what in ((k, "k"), (groups, "groups"), (groups_kept, "groups_kept"), (group_best, "group_best")):
        if not 0 < v < 1 << 31:
            raise ValueError(f"{what} is a positive whole number: got {v!r}")
    return dgs.dgs_router(k, _pick(_SCORE, score, "score"), groups, groups_kept, group_best, renormalise, scale)


def _whole(v, what) -> int:
    n = int(v)
    if n != v:
        raise ValueError(f"{what} is a positive whole number: got {v!r}")
    return n


def _router(k, score, groups, groups_kept, group_best, renormalise, scale) -> "dgs.dgs_router":
    # Looked up by plain numbers: a tensor given for one may hold another value by the next call.  (Made anew each time: 1 us; + 0.0: -0 and 0 are one key.)
    if not (type(k) is type(groups) is type(groups_kept) is type(group_best) is int and type(score) is str and type(renormalise) is bool and type(scale) is float):
        k, groups, groups_kept, group_best = _whole(k, "k"), _whole(groups, "groups"), _whole(groups_kept, "groups_kept"), _whole(group_best, "group_best")
        _pick(_SCORE, score, "score")
        renormalise, scale = bool(renormalise), float(scale)
    return _router_of(k, score, groups, groups_kept, group_best, renormalise, scale + 0.0)


def route_experts(logits: torch.Tensor, k: int, *, score: str = "softmax", bias: Optional[torch.Tensor] = None, groups: int = 1,
                  groups_kept: int = 1, group_best: int = 1, renormalise: bool = True, scale: float = 1.0) -> Route:
    """Chooses k experts for every token (dgs_route_experts): by softmax or sigmoid of the logits plus `bias`, in the `groups_kept` best of
    `groups` groups, ties to the lowest index; with the experts' lists of slots."""
    m = _matrix(logits, "logits")
    _cut_off(logits, "logits", "route_experts")
    router = _router(k, score, groups, groups_kept, group_best, renormalise, scale)
    tokens, experts, device = m.rows, m.cols, logits.device
    pb = _plain(bias, "bias", torch.float32, experts, device)
    need = dgs.dgs_route_experts_bytes(router, tokens, experts)
    slots = tokens * router.k
    whole = torch.empty(3 * slots + experts + 1, dtype=torch.int32, device=device)
    expert, order, place, offsets = whole.split([slots, slots, slots, experts + 1])
    weight = torch.empty(tokens, router.k, dtype=torch.float32, device=device)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    at = whole.data_ptr()
    _enqueue(device, dgs.dgs_route_experts, router, m, pb, at, weight.data_ptr(), at + 12 * slots, at + 4 * slots, at + 8 * slots,
             work.data_ptr() if need else 0, need)
    return Route(expert.view(tokens, router.k), weight, offsets, order, place.view(tokens, router.k))


def route_experts_grad(logits: torch.Tensor, expert: torch.Tensor, dweight: torch.Tensor, *, score: str = "softmax", renormalise: bool = True,
                       scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of route_experts' weights taken back to the logits, of the logits' type; `out` may be the logits."""
    m = _matrix(logits, "logits")
    if expert.dim() < 1 or expert.shape[-1] < 1:
        raise ValueError("expert is [tokens, k]")
    k = expert.shape[-1]
    router = _router(k, score, 1, 1, 1, renormalise, scale)
    pe = _plain(expert, "expert", torch.int32, m.rows * k, logits.device)
    pw = _plain(dweight, "dweight", torch.float32, m.rows * k, logits.device)
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    mo = _matrix(out, "out")
    _same_device(logits.device, out)
    _enqueue(logits.device, dgs.dgs_route_experts_grad, router, m, pe, pw, mo)
    return out


def _slots(place: torch.Tensor) -> int:
    """k of a [tokens, k] place."""
    k = place.shape[-1] if isinstance(place, torch.Tensor) and place.dim() else 0
    if not 1 <= k <= 32:                                # DGS_ROUTE_MAX_K
        raise ValueError(f"place is [tokens, k], k from 1 to {dgs.DGS_ROUTE_MAX_K}")
    return k


def _fit(m: "dgs.dgs_matrix", what: str, rows: int, cols: int, kind: int) -> None:
    if m.rows != rows or m.cols != cols or m.type != kind:
        raise ValueError(f"{what} must be {rows} x {cols} and of the other matrices' type: got {m.rows} x {m.cols}")


def _rows_like(out: Optional[torch.Tensor], m: "dgs.dgs_matrix", rows: int, like: torch.Tensor):
    """(out, its matrix): `rows` rows of m's columns and type, a new tensor if there is none."""
    cols, kind = m.cols, m.type
    if out is None:
        out = like.new_empty(rows, cols)                # 1 us less than torch.empty
        return out, dgs.dgs_matrix(out.data_ptr(), rows, cols, cols, kind)
    mo = _matrix(out, "out")
    _fit(mo, "out", rows, cols, kind)
    _same_device(like.device, out)
    return out, mo


def gather_experts(x: torch.Tensor, order: torch.Tensor, place: torch.Tensor, *, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The tokens' rows in the order of the experts' lists (order and place of a Route): row i is that of token order[i] // k, and
    zero where order[i] is -1.  Returns [tokens * k, cols]."""
    m = _matrix(x, "x")
    _cut_off(x, "x", "gather_experts")
    k, device = _slots(place), x.device
    slots = m.rows * k
    po = _plain(order, "order", torch.int32, slots, device)
    pp = _plain(place, "place", torch.int32, slots, device)
    out, mo = _rows_like(out, m, slots, x)
    _run(device, "dgs_experts_gather", m, po, pp, k, mo)
    return out


def _combine(y, weight, place, out, what):
    m = _matrix(y, what)
    k, rows, device = _slots(place), m.rows, y.device
    if rows % k:
        raise ValueError(f"{what} has a row for each of the tokens' {k} slots: got {rows} rows")
    pw = _plain(weight, "weight", torch.float32, rows, device)
    pp = _plain(place, "place", torch.int32, rows, device)
    out, mo = _rows_like(out, m, rows // k, y)
    _run(device, "dgs_experts_combine", m, pw, pp, k, mo)
    return out


def gather_experts_grad(dy: torch.Tensor, place: torch.Tensor, *, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of gather_experts: the gradients of a token's rows added up.  Returns [tokens, cols]."""
    return _combine(dy, None, place, out, "dy")


def combine_experts(y: torch.Tensor, weight: torch.Tensor, place: torch.Tensor, *, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Each token's rows of y [tokens * k, cols] (in the order of the experts' lists), weighted (float32 [tokens, k]) and added up in float32.
    Empty slots take no part.  Returns [tokens, cols]."""
    _on_gpu(weight, "weight")
    if isinstance(y, torch.Tensor):
        _cut_off(y, "y", "combine_experts")
    _cut_off(weight, "weight", "combine_experts")
    return _combine(y, weight, place, out, "y")


def combine_experts_grad(dout: torch.Tensor, y: torch.Tensor, weight: torch.Tensor, order: torch.Tensor, place: torch.Tensor, *,
                         out: Optional[torch.Tensor] = None):
    """The gradient of combine_experts: (dy [tokens * k, cols] in the order of the experts' lists, zero behind the last one, and
    dweight float32 [tokens, k])."""
    m = _matrix(dout, "dout")
    my = _matrix(y, "y")
    k, device = _slots(place), dout.device
    slots = m.rows * k
    _fit(my, "y", slots, m.cols, m.type)
    _same_device(device, y)
    _on_gpu(weight, "weight")
    pw = _plain(weight, "weight", torch.float32, slots, device)
    po = _plain(order, "order", torch.int32, slots, device)
    pp = _plain(place, "place", torch.int32, slots, device)
    out, mo = _rows_like(out, m, slots, dout)
    dweight = weight.new_empty(place.shape)
    _run(device, "dgs_experts_combine_grad", m, my, pw, po, pp, k, mo, dweight.data_ptr())
    return out, dweight


class VocabularyLoss(NamedTuple):
    """What vocabulary_loss returns, float32 of the targets' shape."""
    loss: torch.Tensor   # 0 in ignored rows
    lse: torch.Tensor    # log of the sum of exponentials of a row's logits: what the gradient takes


def _head(hidden, weight, target):
    """(hidden's and weight's matrix, the targets' address, flags) of a head's call."""
    mh, mw = _matrix(hidden, "hidden"), _matrix(weight, "weight")
    if mw.cols != mh.cols or mw.type != mh.type:
        raise ValueError(f"weight has a row of {mh.cols} values for each word, of hidden's type: got {mw.rows} x {mw.cols} in {weight.dtype}")
    if not isinstance(target, torch.Tensor) or target.dtype not in (torch.int64, torch.int32):
        raise ValueError("target must be an int64 or int32 tensor")
    pt = _plain(target, "target", target.dtype, mh.rows, hidden.device)
    _same_device(hidden.device, weight)
    return mh, mw, pt, dgs.DGS_TARGET_I64 if target.dtype == torch.int64 else 0


@functools.lru_cache(maxsize=256)
def _head_bytes(grad: bool, rows: int, stride: int, at: int, words: int, word_stride: int, word_at: int, cols: int, kind: int) -> int:
    """The workspace of a head's call; at, word_at: the addresses' last 8 bits (their alignment counts)."""
    ask = dgs.dgs_vocabulary_loss_grad_bytes if grad else dgs.dgs_vocabulary_loss_bytes
    return ask(dgs.dgs_matrix(at + 256, rows, stride, cols, kind), dgs.dgs_matrix(word_at + 256, words, word_stride, cols, kind))


def _workspace(grad: bool, mh: "dgs.dgs_matrix", mw: "dgs.dgs_matrix") -> int:
    return _head_bytes(grad, mh.rows, mh.stride, (mh.data or 0) & 255, mw.rows, mw.stride, (mw.data or 0) & 255, mh.cols, mh.type)


def vocabulary_loss(hidden: torch.Tensor, weight: torch.Tensor, target: torch.Tensor) -> VocabularyLoss:
    """Softmax cross entropy of hidden states [..., width] against a vocabulary [words, width] of their type, a loss for each row, without keeping the
    logits.  target: int64 or int32, a word for each row; below 0: the row is ignored (loss 0)."""
    mh, mw, pt, flags = _head(hidden, weight, target)
    _cut_off(hidden, "hidden", "vocabulary_loss")
    _cut_off(weight, "weight", "vocabulary_loss")
    device = hidden.device
    need = _workspace(False, mh, mw)
    loss, lse = torch.empty(2, *target.shape, dtype=torch.float32, device=device).unbind()
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _run(device, "dgs_vocabulary_loss", mh, mw, pt, flags, loss.data_ptr(), lse.data_ptr(), work.data_ptr() if need else 0, need)
    return VocabularyLoss(loss, lse)


def vocabulary_loss_grad(hidden: torch.Tensor, weight: torch.Tensor, target: torch.Tensor, lse: torch.Tensor, dloss: torch.Tensor,
                         dw: Optional[torch.Tensor] = None, *, add: bool = False, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of vocabulary_loss: returns that of the hidden states, of their type, and writes (with `add`, adds) the vocabulary's to dw, a
    contiguous float32 tensor of words * width elements such as the layer's slice of the flat gradient.  dloss: float32, one for each row or one for all (an expanded one too)."""
    mh, mw, pt, flags = _head(hidden, weight, target)
    device = hidden.device
    if add:
        flags |= dgs.DGS_LOSS_ADD
    if not isinstance(lse, torch.Tensor) or not isinstance(dloss, torch.Tensor):
        raise ValueError("lse and dloss are tensors")
    rows, one = mh.rows, dloss.numel() == 1
    if not one and dloss.numel() == rows and rows and not any(dloss.stride()):       # one value, seen from every row
        dloss, one = dloss[(0,) * dloss.dim()], True
    pl = _plain(lse, "lse", torch.float32, rows, device)
    pg = _plain(dloss, "dloss", torch.float32, 1 if one else rows, device)
    pw = _plain(dw, "dw", torch.float32, mw.rows * mw.cols, device)
    if out is None:
        out = hidden.new_empty(hidden.shape)
        mo = dgs.dgs_matrix(out.data_ptr(), rows, mh.cols, mh.cols, mh.type)
    else:
        mo = _matrix(out, "out")
        _fit(mo, "out", rows, mh.cols, mh.type)
        _same_device(device, out)
    need = _workspace(True, mh, mw)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _run(device, "dgs_vocabulary_loss_grad", mh, mw, pt, pl, pg, 0 if one else 1, mo, pw, flags, work.data_ptr() if need else 0, need)
    return out
