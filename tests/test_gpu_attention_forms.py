"""ps_attention_forward / ps_attention_backward where the kernels go other ways than at the sizes of test_gpu_attention.py, whose
bounds these are: scores stay under 30 in powers of two here too."""
import numpy as np
import pytest
import torch

from paper_2504_03702_amd import binding as ps
from tests.test_gpu_attention import Problem, SLOPES

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cap", [20.0, 50.0, 256.0, 257.0, 1e3, 1e6, 1e20, 2.0 ** 100, 3e38])
def test_caps_of_any_size(dtype, cap):
    """A score near zero of a large cap keeps its places: tanh is as good there as the quotient."""
    for size in (64, 96, 128):
        Problem(dtype, [100, 1, 70], [100, 1, 70], size=size, causal=True, cap=cap, big=3.0).check()
    Problem(dtype, [1, 2], [900, 40], size=64, causal=True, cap=cap, slopes=SLOPES, big=3.0).check(backward=False)


@pytest.mark.parametrize("q_lens,k_lens,rows", [([3, 0, 2], [4, 1, 4], 5), ([0, 1], [2, 0], 0)])
def test_calls_without_rows_tell_faulty_sequences(q_lens, k_lens, rows):
    """A bound, or a tensor, of no rows: sequences that have some are faulty, and the others get their gradients."""
    p = Problem(torch.float32, q_lens, k_lens)
    p.max_q = 0
    p.q, p.dout = p.q[:rows], p.dout[:rows]
    bad = q_lens.index(max(q_lens))
    out, lse = p.forward()
    assert torch.all(out == 7.0) and ps.ps_status_read(p.status) == (ps.PS_ST_BAD_LENGTH, bad)
    p.status.zero_()
    dq, dk, dv = p.backward(out, lse)
    assert ps.ps_status_read(p.status) == (ps.PS_ST_BAD_LENGTH, bad) and torch.all(dq == 7.0)
    left = torch.tensor(np.repeat(np.array(q_lens) > 0, k_lens))
    for t in (dk, dv):
        assert torch.all(t[left] == 7.0) and torch.all(t[~left] == 0)


def test_the_largest_place():
    """2^30 rows from place 2^30 on: the last one stands at 2^31 - 1, and sees the keys like the others."""
    n = 1 << 30
    q, out = torch.zeros(n, 1, 8, dtype=torch.bfloat16, device=DEV), torch.zeros(n, 1, 8, dtype=torch.bfloat16, device=DEV)
    k = torch.ones(3, 1, 8, dtype=torch.bfloat16, device=DEV)
    nb = ps.ps_attention_workspace_bytes(1, n, 3, n, 3, 1, 1, 8, torch.bfloat16)
    rows, keys, start = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([0, n], [0, 3], [n]))
    status = ps.new_status(DEV)
    ps.ps_attention_forward(q, k, k, rows, keys, n, 3, out, None, ps.alloc_workspace(nb, DEV), causal=True, q_start=start, status=status)
    assert ps.ps_status_read(status) == (0, -1)
    for some in (out[:1000], out[n // 2:n // 2 + 1000], out[-1000:]):
        assert torch.all(some == 1.0)
