"""The operators as functions with gradients, one after the other in a layer: against the same layer in 64 bits on the CPU, and as
the example uses them.

Bounds: fp32, each operator keeps 1e-5 of its result's norm and the layer has four in a row, forwards and backwards: 1e-4.  bf16 rounds
each of a dozen tensors on the way to 2^-8 of a value at most (1.7e-3 in the mean square): 12 * 1.7e-3 = 2e-2, were they all to add up."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import layer as ol
from paper_2504_03702_amd import binding as ps
from paper_2504_03702_amd import layers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def rotate(x, angle):
    n = angle.shape[1]
    a, b, c, s = x[..., :n], x[..., n:2 * n], angle.cos()[:, None], angle.sin()[:, None]
    return torch.cat((a * c - b * s, a * s + b * c, x[..., 2 * n:]), -1)


@pytest.mark.parametrize("dtype,bound", [(torch.float32, 1e-4), (torch.bfloat16, 2e-2)])
def test_a_layer_and_its_gradients(dtype, bound):
    g = torch.Generator().manual_seed(3)
    heads, kv, size, lens = 4, 2, 32, [70, 1, 40]
    n, hidden = sum(lens), heads * size
    made = lambda *s: (torch.randn(s, generator=g) * 0.5).to(dtype)
    x, w_qkv, w_out, bias, dy = made(n, hidden), made(hidden, (heads + 2 * kv) * size) * 0.2, made(hidden, hidden) * 0.2, made(hidden), made(n, hidden)
    pos = torch.cat([torch.arange(m) for m in lens])
    f = ps.ps_rotary_frequencies(8)
    offsets = np.cumsum([0] + lens)
    slopes = torch.tensor([0.5, 0.25, 0.125, 0.0625])

    # in 64 bits
    leaves = [t.double().requires_grad_() for t in (x, w_qkv, w_out, bias)]
    xd, wd, od, bd = leaves
    q, k, v = (xd @ wd).view(n, heads + 2 * kv, size).split((heads, kv, kv), 1)
    angle = pos[:, None].double() * f.double()
    q, k = rotate(q, angle), rotate(k, angle)
    rows = []
    for s in range(3):
        i = slice(offsets[s], offsets[s + 1])
        m = lens[s]
        at = torch.arange(m)
        z = torch.einsum("ihd,jhd->hij", q[i], k[i].repeat_interleave(heads // kv, 1)) * size ** -0.5
        z = 20 * torch.tanh(z / 20) - slopes.double()[:, None, None] * (at[:, None] - at).abs()
        z = z.masked_fill(at[None] > at[:, None], -torch.inf)
        rows.append(torch.einsum("hij,jhd->ihd", z.softmax(-1), v[i].repeat_interleave(heads // kv, 1)))
    keep, by = ol.kept(n, hidden, 11, 5, 0.2)
    want = xd + (torch.cat(rows).reshape(n, hidden) @ od + bd) * torch.tensor(keep) * by
    want.backward(dy.double())

    on = [t.to(DEV).requires_grad_() for t in (x, w_qkv, w_out, bias)]
    xg, wg, og, bg = on
    i32 = lambda t: torch.as_tensor(t).to(DEV, torch.int32)
    rng = torch.tensor([11, 5], dtype=torch.int64, device=DEV)
    q, k, v = (xg @ wg).view(n, heads + 2 * kv, size).split((heads, kv, kv), 1)
    q, k = layers.rotary(q, k, i32(pos), f.to(DEV))
    a = layers.attention(q, k, v, layers.Sequences(i32(offsets), i32(offsets), max(lens), max(lens)), softcap=20.0, causal=True, slopes=slopes.to(DEV))
    y = layers.dropout_add(a.reshape(n, hidden) @ og, bg, xg, rng, 0.2)
    y.backward(dy.to(DEV))
    assert rng.tolist() == [11, 6]
    for got, ref, name in zip((y, *(t.grad for t in on)), (want, *(t.grad for t in leaves)), ("y", "dx", "dqkv", "dout", "dbias")):
        assert got.dtype == dtype
        off = (got.detach().double().cpu() - ref.detach()).norm() / ref.detach().norm()
        assert off < bound, (name, float(off))


def test_rows_of_no_sequence_get_no_gradient():
    q, k, v = (torch.randn(10, 2, 16, device=DEV, requires_grad=True) for _ in range(3))
    offs = torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    out = layers.attention(q, k, v, layers.Sequences(offs, offs, 4, 4))
    out[:4].sum().backward()
    for t in (q, k, v):
        assert torch.all(t.grad[4:] == 0)
    assert torch.any(v.grad[:4] != 0)


@pytest.mark.parametrize("dtype,same", [(torch.float32, 1e-4), (torch.bfloat16, 6e-2)])
def test_the_example_learns_and_scores_by_first_rows(dtype, same):
    """Scores by all rows and by first rows differ by roundings of a row of unit size (2^-8 in bf16, twice) times a head of length 16."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import finetune_long_prompts as example
    finally:
        sys.path.pop(0)
    first, last, off = example.main(40, dtype)
    assert last < 0.5 * first and off < same
