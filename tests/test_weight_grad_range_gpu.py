"""Weight gradients at the ends of their types and sizes: gradients next to nothing, long sums, few rows of large layers, replayed graphs."""
import pytest
import torch

import paper_1910_10929_b200 as dgs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("rows", [1, 600])               # few rows, and by the tensor cores
def test_f32_gradients_next_to_nothing(rows):
    """Three bfloat16 numbers add up to a float of at least 2^-110; below, what lies under bfloat16's last bit, 2^-133, may be missing, and no more."""
    g = torch.Generator(device=DEV).manual_seed(0)
    e = torch.randint(-149, -99, (1 << 14,), generator=g, device=DEV)
    d = (torch.ldexp(torch.rand(1 << 14, generator=g, device=DEV, dtype=torch.float64) + 1, e)).float()
    d[::2] *= -1
    h = torch.tensor([1.0, -1.0, 2.0, 64.0], device=DEV)
    x, dy = torch.zeros(rows, 4, device=DEV), torch.zeros(rows, 1 << 14, device=DEV)
    x[-1], dy[-1] = h, d
    c = dgs.Checkpoint(rows, 4, device=DEV)
    c.save(x)
    dw, db = torch.full((1 << 14, 4), float("nan"), device=DEV), torch.full((1 << 14,), float("nan"), device=DEV)
    c.weight_grad(dy, dw, db)
    cut = torch.where(d.abs() < 2.0 ** -110, 2.0 ** -133, 0.0).double()
    # a product with h, a power of two, is a float wherever d is
    assert bool(((dw.double() - d.double()[:, None] * h.double()).abs() <= cut[:, None] * h.abs().double()).all())
    assert bool(((db.double() - d.double()).abs() <= cut).all())
    assert dgs.operator_status(DEV) == 0


@pytest.mark.parametrize("layout", ["out_in", "in_out"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_long_sums_keep_their_digits(dtype, layout):
    """About as many tiles as pairs of CTAs, so that rows are not split: every sum is over all 16384 rows in one CTA."""
    rows, inputs, outputs = 16384, 2048, 2304
    g = torch.Generator(device=DEV).manual_seed(1)
    c = dgs.Checkpoint(rows, inputs, device=DEV)
    c.save(torch.randn(rows, inputs, generator=g, device=DEV))
    dy = (torch.randn(rows, outputs, generator=g, device=DEV) * 1e-3).to(dtype)
    shape = (outputs, inputs) if layout == "out_in" else (inputs, outputs)
    dw, db = torch.full(shape, float("nan"), device=DEV), torch.full((outputs,), float("nan"), device=DEV)
    planes = {torch.float32: 6, torch.float16: 4, torch.bfloat16: 0}[dtype]
    need = dgs.dgs_checkpoint_weight_grad_bytes(c._held, dgs.operators._matrix(dy, "dy"), None, 0)
    assert need < (rows + 256) * (inputs * 2 + outputs * planes) + 32 * 4 * outputs      # the operands as bfloat16 numbers: no partial results
    c.weight_grad(dy, dw, db, layout=layout)
    h, d = c.load().double(), dy.double()
    want = d.T @ h if layout == "out_in" else h.T @ d
    # Accumulators are taken to f32 sums with rounding every 512 rows (256 of f32 gradients, of three parts): 32 additions (48) of sixteen rows each. An addition
    # cuts off less than 2^-23 of the sum so far, half of that in the mean, and always towards zero; the sums so far are no larger than the last one in the
    # mean.  The few f32 roundings beside are of no weight.  All rows in one accumulator: 1024 additions, 5e-6 and more.
    additions = 48 if dtype == torch.float32 else 32 * (2 if dtype == torch.float16 else 1)
    assert float((dw.double() - want).norm() / want.norm()) < additions * 2.0 ** -24
    # the bias: 64 threads' f32 sums of 4096 rows each, roundings of half a step that add up like a walk (64 steps), with parts likewise
    want = d.sum(0)
    assert float((db.double() - want).norm() / want.norm()) < 64 * 2 * 2.0 ** -24


# past the products for which few rows take a kernel of their own
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,inputs,outputs,experts", [(0, 8192, 16500, 0), (0, 4100, 33000, 2), (1, 8200, 16400, 0), (1, 16400, 8200, 2), (37, 2049, 2050, 0),
                                                         (37, 2050, 2049, 5), (200, 1030, 700, 0), (200, 700, 1030, 3), (256, 800, 801, 1)])
def test_few_rows_of_large_layers(rows, inputs, outputs, experts, dtype, add):
    assert inputs * outputs * max(rows, 1) > 1 << 27
    g = torch.Generator(device=DEV).manual_seed(rows)
    x = torch.randint(-7, 8, (rows, inputs), generator=g, device=DEV).float()
    dy = torch.randint(-8, 9, (rows, outputs), generator=g, device=DEV).to(dtype)
    c = dgs.Checkpoint(rows, inputs, "e4m3", device=DEV)
    c.save(x)
    n = max(1, experts)
    cut = sorted(torch.randint(0, rows + 1, (n - 1,), generator=torch.Generator().manual_seed(rows)).tolist())
    cut = [0] + cut + [rows]
    lists = dict(offsets=torch.tensor(cut, dtype=torch.int32, device=DEV)) if experts else {}
    flat = torch.full((1 + n * outputs * (inputs + 1),), 5.0 if add else float("nan"), device=DEV)
    dw, db = flat[1:1 + n * outputs * inputs], flat[1 + n * outputs * inputs:]
    c.weight_grad(dy, dw, db, add=add, **lists)
    assert dgs.operator_status(DEV) == 0
    for e in range(n):
        d = dy[cut[e]:cut[e + 1]].float()                # whole numbers: f32 sums are exact
        want = d.T @ x[cut[e]:cut[e + 1]] if d.shape[0] else torch.zeros(outputs, inputs, device=DEV)
        assert torch.equal(dw.view(n, outputs, inputs)[e], want + 5.0 if add else want)
        assert torch.equal(db.view(n, outputs)[e], d.sum(0) + 5.0 if add else d.sum(0))


@pytest.mark.parametrize("dtype,outputs", [(torch.float32, 96), (torch.float16, 96), (torch.bfloat16, 96), (torch.bfloat16, 97)])
@pytest.mark.parametrize("listed", [False, True])
def test_captured_with_other_lists_and_gradients_at_each_replay(listed, dtype, outputs):
    rows, inputs, experts, k = 3000, 130, 6, 2
    g = torch.Generator(device=DEV).manual_seed(2)
    c = dgs.Checkpoint(rows, inputs, device=DEV)
    c.save(torch.randint(-7, 8, (rows, inputs), generator=g, device=DEV).float())
    n = rows * k if listed else rows
    dy = torch.zeros(n, outputs, dtype=dtype, device=DEV)
    lists = {}
    if listed:
        lists = dict(offsets=torch.zeros(experts + 1, dtype=torch.int32, device=DEV), rows=torch.zeros(n, dtype=torch.int32, device=DEV), rows_per=k)

    def change(seed):
        dy.copy_(torch.randint(-8, 9, dy.shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))
        if listed:
            r = dgs.route_experts(torch.randn(rows, experts, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV), k)
            lists["offsets"].copy_(r.offsets)
            lists["rows"].copy_(r.order)

    def flat():
        return torch.full((max(1, experts if listed else 1) * outputs * (inputs + 1),), float("nan"), device=DEV)

    def call(f):
        at = f.numel() // (inputs + 1) * inputs
        c.weight_grad(dy, f[:at], f[at:], layout="in_out", **lists)

    change(0)
    got, want = flat(), flat()
    call(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]           # two graphs of the same call: workspaces of their own
    for graph in graphs:
        with torch.cuda.graph(graph, stream=side):
            call(got)
    for seed in (1, 2, 3):
        change(seed)
        got.fill_(float("nan"))
        graphs[seed % 2].replay()
        call(want)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and bool(torch.isfinite(got).all())
    assert dgs.operator_status(DEV) == 0


@pytest.mark.parametrize("inputs,outputs", [(40, 24), (4100, 33000)])    # by the kernel for few rows, and by the other
def test_lists_that_point_outside_a_gradient_without_rows_are_reported(inputs, outputs):
    c = dgs.Checkpoint(7, inputs, device=DEV)
    c.save(torch.ones(7, inputs, device=DEV))
    dy = torch.zeros(0, outputs, device=DEV)
    dw, db = torch.full((2 * outputs * inputs,), float("nan"), device=DEV), torch.full((2 * outputs,), float("nan"), device=DEV)
    for offsets, status in (([0, 0, 0], 0), ([0, 0, 5], dgs.DGS_EINVAL), ([3, 3, 3], dgs.DGS_EINVAL)):
        dw.fill_(float("nan"))
        c.weight_grad(dy, dw, db, offsets=torch.tensor(offsets, dtype=torch.int32, device=DEV))
        assert dgs.operator_status(DEV) == status
        assert not bool(dw.any()) and not bool(db.any())
