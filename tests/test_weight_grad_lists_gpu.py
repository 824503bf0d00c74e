"""Weight gradients of experts at the lengths that the products' kernel treats apart: last steps that share a copy's rows with the next expert, at
every place in a run of steps, and tiles without rows between others.  Sums of whole numbers are exact in f32 in any order, so results must come out bit for bit."""
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def check(lengths, inputs, outputs, dtype, layout, behind=0, seed=0, scattered=False):
    """dw and db of experts with these numbers of rows, `behind` rows of dy in no list, the checkpoint's rows in order or in any."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    rows, experts = sum(lengths) + behind, len(lengths)
    x = torch.randint(-7, 8, (rows, inputs), generator=g, device=DEV).float()
    dy = torch.randint(-8, 9, (rows, outputs), generator=g, device=DEV).to(dtype)
    c = dgs.Checkpoint(rows, inputs, "e4m3", device=DEV)
    c.save(x)
    order = torch.randperm(rows, generator=g, device=DEV).to(torch.int32) if scattered else None
    offsets = torch.tensor([0] + lengths).cumsum(0).to(torch.int32).to(DEV)
    shape = (experts, outputs, inputs) if layout == "out_in" else (experts, inputs, outputs)
    dw, db = torch.full(shape, float("nan"), device=DEV), torch.full((experts, outputs), float("nan"), device=DEV)
    c.weight_grad(dy, dw, db, layout=layout, offsets=offsets, rows=order)
    assert dgs.operator_status(DEV) == 0
    at = 0
    for e, n in enumerate(lengths):
        d = dy[at:at + n].double()
        h = (x[order[at:at + n].long()] if scattered else x[at:at + n]).double()
        want = d.T @ h if layout == "out_in" else h.T @ d
        assert torch.equal(dw[e].double(), want) and torch.equal(db[e].double(), d.sum(0)), e
        at += n


@pytest.mark.parametrize("layout", ["out_in", "in_out"])
@pytest.mark.parametrize("dtype", TYPES)
def test_last_steps_at_every_place_in_a_run(dtype, layout):
    """Experts of 5 to 45 steps of 64 rows, the last one never whole: it is any of the four or eight steps between two sums, and comes up to eight
    steps after the sums before.  All bias sums are one CTA's, which keeps its stages longest; more tiles than pairs of CTAs."""
    check([64 * (5 + e) + 1 + e for e in range(40)], 64, 300, dtype, layout, behind=70)


# f32 2048 x 2048 takes two runs of rows a tile and 512 tiles for 74 pairs: those of 1 and 5 rows leave the second run empty between others
@pytest.mark.parametrize("lengths,inputs,outputs,dtype,layout", [
    ([30000, 1, 5, 16000], 2048, 2048, torch.float32, "out_in"), ([100, 100, 100, 30000], 2048, 768, torch.float32, "in_out"),
    ([30000, 1, 5, 16000], 2048, 2048, torch.bfloat16, "out_in"), ([100, 100, 100, 30000], 2048, 768, torch.float16, "in_out")])
def test_runs_without_rows_between_others(lengths, inputs, outputs, dtype, layout):
    check(lengths, inputs, outputs, dtype, layout, behind=3)


@pytest.mark.parametrize("layout", ["out_in", "in_out"])
@pytest.mark.parametrize("dtype", TYPES)
def test_sixteen_experts_of_unequal_length_on_more_tiles_than_pairs(dtype, layout):
    lengths = [0, 700, 3, 0, 1500, 64, 128, 1, 0, 2050, 129, 63, 640, 0, 31, 999]
    check(lengths, 768, 700, dtype, layout, behind=5, scattered=True)


@pytest.mark.parametrize("layout", ["out_in", "in_out"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,inputs,outputs,named", [([20, 0, 30], 70, 40, True), ([20, 0, 30], 70, 40, False), ([700, 90, 1, 300], 40, 72, True),
                                                          ([700, 90, 1, 300], 40, 72, False), ([20000, 130], 96, 300, True)])
def test_rows_that_name_no_row_of_the_checkpoint_take_no_part(lengths, inputs, outputs, named, dtype, layout):
    """Neither in dw nor in db, whatever they hold: NaN, infinities and large numbers of dy stay out.  named: by rows; otherwise dy has more rows than the
    checkpoint.  In whole steps and in last ones, in one run of rows and in several."""
    g = torch.Generator(device=DEV).manual_seed(len(lengths))
    n, experts, k = sum(lengths), len(lengths), 3
    held = n if named else n - 17
    x = torch.randint(-7, 8, (held, inputs), generator=g, device=DEV).float()
    dy = torch.randint(-8, 9, (n + 4, outputs), generator=g, device=DEV).to(dtype)
    c = dgs.Checkpoint(held, inputs, device=DEV)
    c.save(x)
    rows, there = None, torch.arange(n, device=DEV) < held
    at = torch.arange(n, device=DEV)
    if named:
        at = torch.randint(0, held, (n,), generator=g, device=DEV)
        rows = torch.cat([at * k + 1, torch.tensor([-1, held * k, 0, -5], device=DEV)]).to(torch.int32)   # behind the last list: not looked at
        out = torch.rand(n, generator=g, device=DEV) < 0.05
        out[[0, lengths[0] - 1, n - 1]] = True
        there = ~out
        bad = torch.tensor([held * k, -1, -(1 << 31)], device=DEV).to(torch.int32)
        rows[:n] = torch.where(out, bad[at % 3], rows[:n])
    dy[:n][~there] = torch.tensor([float("nan"), float("inf"), -float("inf"), 60000.0], device=DEV).to(dtype)[torch.arange(int((~there).sum()), device=DEV) % 4][:, None]
    dy[n:] = float("nan")
    offsets = torch.tensor([0] + lengths).cumsum(0).to(torch.int32).to(DEV)
    shape = (experts, outputs, inputs) if layout == "out_in" else (experts, inputs, outputs)
    dw, db = torch.full(shape, float("nan"), device=DEV), torch.full((experts, outputs), float("nan"), device=DEV)
    c.weight_grad(dy, dw, db, layout=layout, offsets=offsets, rows=rows, rows_per=k if named else 1)
    assert dgs.operator_status(DEV) == dgs.DGS_EINVAL and dgs.operator_status(DEV) == 0
    cut = offsets.tolist()
    for e in range(experts):
        part = torch.arange(cut[e], cut[e + 1], device=DEV)
        part = part[there[part]]
        d, h = dy[part].double(), x[at[part]].double()
        assert torch.equal(dw[e].double(), d.T @ h if layout == "out_in" else h.T @ d) and torch.equal(db[e].double(), d.sum(0)), e


@pytest.mark.parametrize("dtype", TYPES)
def test_one_row_that_names_no_row_wherever_it_stands(dtype):
    n, inputs, outputs = 9000, 40, 24
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randint(-7, 8, (n, inputs), generator=g, device=DEV).float()
    clean = torch.randint(-8, 9, (n, outputs), generator=g, device=DEV).to(dtype)
    c = dgs.Checkpoint(n, inputs, device=DEV)
    c.save(x)
    offsets = torch.tensor([2, 5000, 8997], dtype=torch.int32, device=DEV)
    for at in (2, 4095, 4096, 4999, 5000, 8191, 8192, 8996, 1, 8997):
        rows = torch.arange(n, dtype=torch.int32, device=DEV)
        dy = clean.clone()
        rows[at], dy[at] = n, float("nan")
        dw, db = torch.zeros(2, outputs, inputs, device=DEV), torch.zeros(2, outputs, device=DEV)
        c.weight_grad(dy, dw, db, offsets=offsets, rows=rows)
        assert dgs.operator_status(DEV) == (dgs.DGS_EINVAL if 2 <= at < 8997 else 0), at    # in no list: not looked at
        for e, (a, b) in enumerate(((2, 5000), (5000, 8997))):
            keep = torch.arange(a, b, device=DEV)
            keep = keep[keep != at]
            d = clean[keep].double()
            assert torch.equal(dw[e].double(), d.T @ x[keep].double()) and torch.equal(db[e].double(), d.sum(0)), (at, e)
