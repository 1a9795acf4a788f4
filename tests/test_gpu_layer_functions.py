"""The layer functions with the kernels behind them: rows that no sequence has, faulty sequences, recomputed passes, what is written
again before the gradients are taken.  What they do is exact: zeros, flags, errors, the same bits."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from paper_2504_03702_amd import binding as ps
from paper_2504_03702_amd import layers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def drawn(*shapes, dtype=torch.float32, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return [torch.randn(s, generator=g, device=DEV).to(dtype).requires_grad_() for s in shapes]


def offsets(*at):
    return torch.tensor(at, dtype=torch.int32, device=DEV)


def leave_nan(*shapes, dtype):
    """Freed memory of these sizes that the next tensors of them get."""
    t = [torch.full(s, float("nan"), dtype=dtype, device=DEV) for s in shapes for _ in range(4)]
    del t


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_no_sequence_are_zeros(dtype):
    q, k, v = drawn((10, 2, 16), (10, 2, 16), (10, 2, 16), dtype=dtype)
    (w,) = drawn((32, 8), dtype=dtype, seed=1)
    leave_nan(q.shape, (2, 10), dtype=dtype)
    out = layers.attention(q, k, v, layers.Sequences(offsets(2, 6), offsets(0, 4), 4, 4))
    assert torch.all(out[:2] == 0) and torch.all(out[6:] == 0) and torch.all(out[2:6] != 0)
    (out.reshape(10, 32) @ w)[2:6].sum().backward()
    assert all(torch.isfinite(t.grad).all() for t in (q, k, v, w))
