"""ps_dropout_forward / ps_dropout_backward against their 64-bit definition: which values are kept is exact, a value is a sum, a
product and a sum in fp32 (3 * 2^-24 of what goes into it) and rounded once more in bf16 (2^-8); a column's sum of n values in fp32,
in parts, is good to 2^-24 times the parts' length (at most 64 + 256 values) in the worst case, of the sum of their sizes."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from paper_2504_03702_amd import binding as ps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rng_of(seed, offset):
    return torch.tensor([seed, offset], dtype=torch.int64, device=DEV)


def c(t):
    return None if t is None else t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 767), (577, 128), (33, 1000), (64, 7), (1025, 64), (2, 4096), (40, 250)])
@pytest.mark.parametrize("p,bias,residual", [(0.1, True, True), (0.5, False, True), (0.0, True, False), (1.0, True, True), (0.3, False, False)])
def test_both_directions(dtype, rows, cols, p, bias, residual):
    g = torch.Generator(device=DEV)
    g.manual_seed(rows + cols)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)
    x, b, r, dout = normal(rows, cols), normal(cols) if bias else None, normal(rows, cols) if residual else None, normal(rows, cols)
    seed, offset = -(2 ** 62) + 12345 * rows, 2 ** 33 + cols
    out, dx, db = torch.full_like(x, 7.0), torch.full_like(x, 7.0), torch.full((cols,), 7.0, device=DEV)
    rng = rng_of(seed, offset)
    ps.ps_dropout_forward(x, b, r, rng, p, out)
    ws = ps.alloc_workspace(ps.ps_dropout_workspace_bytes(rows, cols), DEV)
    ws.fill_(0xFF)
    ps.ps_dropout_backward(dout, rng, p, dx, db, ws)
    eps = 3 * 2.0 ** -24 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    keep, by = ol.kept(rows, cols, seed, offset, p)
    size = np.where(keep, (np.abs(c(x)) + (np.abs(c(b)) if bias else 0)) * by, 0) + (np.abs(c(r)) if residual else 0)
    ref = ol.dropout(c(x), c(b), c(r), seed, offset, p)
    assert np.all(np.abs(c(out) - ref) <= 3 * 2.0 ** -24 * size + eps * np.abs(ref))
    rdx, rdb = ol.dropout_gradients(c(dout), seed, offset, p)
    assert np.all(np.abs(c(dx) - rdx) <= eps * np.abs(rdx)) and np.array_equal(c(dx) == 0, rdx == 0)
    assert np.all(np.abs(c(db) - rdb) <= 320 * 2.0 ** -24 * np.abs(rdx).sum(0) + 1e-30)
    alone = torch.full_like(x, 7.0)
    ps.ps_dropout_backward(dout, rng, p, alone, None, None)
    assert torch.equal(alone, dx)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_columns(dtype):
    rows, cols = 20011, 72
    dout = torch.randn(rows, cols, device=DEV).to(dtype)
    dx, db, rng = torch.empty_like(dout), torch.empty(cols, device=DEV), rng_of(5, 6)
    ps.ps_dropout_backward(dout, rng, 0.2, dx, db, ps.alloc_workspace(ps.ps_dropout_workspace_bytes(rows, cols), DEV))
    rdx, rdb = ol.dropout_gradients(c(dout), 5, 6, 0.2)
    assert np.all(np.abs(c(db) - rdb) <= 320 * 2.0 ** -24 * np.abs(rdx).sum(0))
    again = torch.empty_like(db)
    ps.ps_dropout_backward(dout, rng, 0.2, dx, again, ps.alloc_workspace(ps.ps_dropout_workspace_bytes(rows, cols), DEV))
    assert torch.equal(db, again)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(767, 20), (768, 8), (769, 100), (800, 1030)])
def test_one_row_block_and_more(dtype, rows, cols):
    test_both_directions(dtype, rows, cols, 0.25, True, True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_places(dtype):
    """Rows apart, at any element, in place over x or the residual: the mask goes by row and column alone."""
    x, r, b = torch.randn(50, 96, device=DEV).to(dtype), torch.randn(50, 96, device=DEV).to(dtype), torch.randn(96, device=DEV).to(dtype)
    rng = rng_of(77, 3)
    want = torch.empty_like(x)
    ps.ps_dropout_forward(x, b, r, rng, 0.25, want)
    wide = torch.full((50, 131), 5.0, dtype=dtype, device=DEV)
    wide[:, 3:99] = x
    out = torch.full((50, 200), 5.0, dtype=dtype, device=DEV)
    ps.ps_dropout_forward(wide[:, 3:99], b, r, rng, 0.25, out[:, 8:104])
    assert torch.equal(out[:, 8:104], want) and torch.all(out[:, :8] == 5.0) and torch.all(out[:, 104:] == 5.0)
    xx, rr = x.clone(), r.clone()
    ps.ps_dropout_forward(xx, b, rr, rng, 0.25, xx)
    ps.ps_dropout_forward(x, b, rr, rng, 0.25, rr)
    assert torch.equal(xx, want) and torch.equal(rr, want)
    dx, inplace = torch.empty_like(x), x.clone()
    ps.ps_dropout_backward(x, rng, 0.25, dx, None, None)
    ps.ps_dropout_backward(inplace, rng, 0.25, inplace, None, None)
    assert torch.equal(dx, inplace)


def test_what_is_dropped_may_be_anything():
    x = torch.randn(64, 64, device=DEV)
    rng = rng_of(9, 9)
    keep = torch.tensor(ol.kept(64, 64, 9, 9, 0.5)[0], device=DEV)
    want, got = torch.empty_like(x), torch.empty_like(x)
    ps.ps_dropout_forward(x, None, None, rng, 0.5, want)
    bad = torch.where(keep, x, torch.full_like(x, float("nan")))
    ps.ps_dropout_forward(bad, None, None, rng, 0.5, got)
    assert torch.equal(got, want)


def test_gradient_against_differences():
    """Linear in x where it is kept: the difference of two calls is the gradient."""
    x, dout = torch.randn(40, 24, device=DEV), torch.randn(40, 24, device=DEV)
    rng, dx, db = rng_of(1, 2), torch.empty(40, 24, device=DEV), torch.empty(24, device=DEV)
    ps.ps_dropout_backward(dout, rng, 0.4, dx, db, ps.alloc_workspace(ps.ps_dropout_workspace_bytes(40, 24), DEV))
    bias = torch.zeros(24, device=DEV)

    def loss(x, bias):
        out = torch.empty_like(x)
        ps.ps_dropout_forward(x, bias, None, rng, 0.4, out)
        return (out.double() * dout.double()).sum().item()

    for i in ((0, 0), (39, 23), (17, 5)):
        up = x.clone()
        up[i] += 0.5
        assert abs((loss(up, bias) - loss(x, bias)) / (up[i].double() - x[i].double()).item() - dx[i].item()) < 1e-5
    bias[3] = 0.5
    assert abs((loss(x, bias) - loss(x, torch.zeros_like(bias))) / 0.5 - db[3].item()) < 1e-4


def test_masks_move_on_inside_a_graph():
    x, rng, out = torch.ones(30, 64, device=DEV), rng_of(4, 0), torch.empty(30, 64, device=DEV)
    ps.ps_dropout_forward(x, None, None, rng, 0.5, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ps.ps_dropout_forward(x, None, None, rng, 0.5, out)
        rng[1:].add_(1)
    for step in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(c(out), ol.dropout(c(x), None, None, 4, step, 0.5))


def test_nothing_to_do():
    for shape in ((0, 5), (5, 0), (0, 0)):
        x = torch.empty(shape, device=DEV)
        db = torch.full((shape[1],), 7.0, device=DEV)
        ps.ps_dropout_forward(x, None, None, rng_of(1, 1), 0.1, x)
        ps.ps_dropout_backward(x, rng_of(1, 1), 0.1, x, db, ps.alloc_workspace(0, DEV))
        assert torch.all(db == 0)


@pytest.mark.parametrize("change,error", [
    (dict(x=lambda t: t.half()), TypeError), (dict(x=lambda t: t.cpu()), TypeError), (dict(x=lambda t: t[:, ::2]), ValueError),
    (dict(bias=lambda t: torch.ones(15, device=DEV)), ValueError), (dict(residual=lambda t: torch.ones(8, 16, device=DEV).bfloat16()), TypeError),
    (dict(rng=lambda t: t[:1]), ValueError), (dict(rng=lambda t: t.int()), TypeError), (dict(p=lambda t: 1.5), ps.PsError),
    (dict(p=lambda t: -0.1), ps.PsError), (dict(p=lambda t: float("nan")), ps.PsError), (dict(out=lambda t: t[:1].expand(8, -1)), ps.PsError),
    (dict(out=lambda t: None), TypeError)])
def test_refusals(change, error):
    args = dict(x=torch.ones(8, 16, device=DEV), bias=None, residual=None, rng=rng_of(1, 1), p=0.1, out=torch.empty(8, 16, device=DEV))
    ps.ps_dropout_forward(**args)
    args.update({n: f(args[n]) for n, f in change.items()})
    with pytest.raises(error):
        ps.ps_dropout_forward(**args)


def test_backward_refusals():
    x, db = torch.ones(8, 16, device=DEV), torch.empty(16, device=DEV)
    ws = ps.alloc_workspace(ps.ps_dropout_workspace_bytes(8, 16), DEV)
    for args, code in (((x, rng_of(1, 1), 0.1, x, db, None), -5), ((x, rng_of(1, 1), 0.1, x, db, ws[:128]), -5), ((x, rng_of(1, 1), 2.0, x, None, None), -1)):
        with pytest.raises(ps.PsError) as e:
            ps.ps_dropout_backward(*args)
        assert e.value.code == code
    with pytest.raises(TypeError):
        ps.ps_dropout_backward(x, rng_of(1, 1), 0.1, None, None, None)
