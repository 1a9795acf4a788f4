"""ps_attention_forward / ps_attention_backward where the kernels go other ways than at the sizes of test_gpu_attention.py, whose
bounds these are: scores stay under 30 in powers of two here too."""
import numpy as np
import pytest
import torch

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
