"""What the torch-backed calls of a worker's own operators make of their arguments: no GPU needed."""
import os
import subprocess
import sys

import pytest
import torch

from paper_1910_10929_b200 import operators


def test_a_router_is_made_from_the_values_that_arguments_have_now():
    scale, k, renormalise = torch.tensor(1.5), torch.tensor(2), torch.tensor(True)
    make = lambda: operators._router(k, "softmax", 1, 1, 1, renormalise, scale)   # noqa: E731
    r = make()
    assert (r.k, r.renormalise, r.scale) == (2, 1, 1.5)
    scale.fill_(0.25)
    k.fill_(3)
    renormalise.fill_(False)
    r = make()
    assert (r.k, r.renormalise, r.scale) == (3, 0, 0.25)
    for bad in (0, -1, 1.5, 1 << 31):
        with pytest.raises(ValueError):
            operators._router(bad, "softmax", 1, 1, 1, True, 1.0)
    with pytest.raises(ValueError):
        operators._router(2, "relu", 1, 1, 1, True, 1.0)


def test_views_of_more_dimensions_whose_rows_lie_evenly_spaced(monkeypatch):
    monkeypatch.setattr(operators, "_on_gpu", lambda t, what: None)
    whole = torch.arange(2 * 3 * 5 * 24, dtype=torch.float32).view(2, 3, 5, 24)
    even = [whole, whole[..., 3:11], whole[:, :, :, :1], whole[:, :, 2:3, :8], whole[1:, 1:2, ::2, :8], whole[1:, :, :, 4:], whole[:1, :1, :1, 5:9],
            whole[0, 0, 0], whole[0, 0, 0, :1].expand(4, 3, 1), whole[0, 0, :1, :7].expand(6, 2, 5, 7), whole[:0, :, 1:], whole[:1, 2:, :, :5].transpose(0, 1),
            whole.view(6, 5, 24)[:, :, 8:16]]
    for v in even:
        m = operators._matrix(v, "v")
        assert m.rows * m.cols == v.numel() and m.cols == v.shape[-1]
        if v.numel():
            at = v.storage_offset() + torch.arange(m.rows)[:, None] * m.stride + torch.arange(m.cols)
            assert torch.equal(whole.reshape(-1)[at], v.reshape(-1, v.shape[-1])) and m.data == v.data_ptr()
    for v in (whole[:, :, :3, :8], whole[:, :2], whole[:, 1:2, ::2, :8], whole[:, 2:, :, :5].transpose(0, 1), whole.transpose(0, 1), whole.transpose(2, 3), whole[..., ::2], whole[:, :1].expand(2, 4, 5, 24),
              whole[0, 0, :, :7].expand(6, 5, 7)):
        with pytest.raises(ValueError):
            operators._matrix(v, "v")


def test_sizes_past_32_bits_are_refused_and_not_wrapped_around(monkeypatch):
    monkeypatch.setattr(operators, "_on_gpu", lambda t, what: None)
    for shape in (((1 << 32) + 8,), (2, (1 << 32) + 8), (1 << 32,)):
        with pytest.raises(ValueError, match="columns"):
            operators._matrix(torch.empty(shape, dtype=torch.bfloat16, device="meta"), "x")
    m = operators._matrix(torch.empty((1 << 32) - 1, dtype=torch.bfloat16, device="meta"), "x")
    assert (m.rows, m.cols) == (1, (1 << 32) - 1)
    with pytest.raises(ValueError):
        operators.Checkpoint(1, (1 << 32) + 8, data=torch.empty(36, dtype=torch.uint8))
    c = operators.Checkpoint(4, 8, data=torch.empty(4 * 36, dtype=torch.uint8))
    for rows_per in (0, 1 << 32, (1 << 32) + 1):
        with pytest.raises(ValueError, match="rows_per"):
            c.weight_grad(torch.zeros(4, 8), torch.zeros(64), offsets=torch.zeros(2, dtype=torch.int32), rows=torch.zeros(4, dtype=torch.int32), rows_per=rows_per)


def test_the_package_is_imported_where_torch_has_no_cuda():
    code = ("import torch\n"
            "for name in ('_cuda_getDevice', '_cuda_getCurrentRawStream'):\n"
            "    if hasattr(torch._C, name): delattr(torch._C, name)\n"
            "import paper_1910_10929_b200 as dgs\n"
            "try: dgs.route_experts(torch.zeros(4, 8), 2)\n"
            "except ValueError as e: assert 'CUDA' in str(e)\n"
            "else: raise SystemExit(2)\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", code], check=True, cwd=root)
