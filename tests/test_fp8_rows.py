"""Tensors of any shape as a matrix of rows (CPU)."""
import pytest
import torch


@pytest.mark.parametrize("shape", [(5,), (1,), (4, 5), (4, 1), (2, 3, 5), (2, 3, 1), (0, 3, 5), (2, 0, 5), (2, 3, 0), (0, 0, 0), (7, 0), (0,)])
def test_rows(shape):
    from paper_2604_22312_amd.fp8 import _rows_of
    rows = 1
    for n in shape[:-1]:
        rows *= n
    x = torch.arange(max(rows * shape[-1], 1)).float()[:rows * shape[-1]].view(shape)
    m = _rows_of(x)
    assert m.shape == (rows, shape[-1]) and torch.equal(m.reshape(shape), x)
    assert shape[-1] <= 1 or m.stride(1) == 1
    e = x[..., :1].expand(shape) if shape[-1] else x   # (a sum's gradient)
    assert torch.equal(_rows_of(e).reshape(shape), e)
