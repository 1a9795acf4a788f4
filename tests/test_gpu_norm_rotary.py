"""ps_norm_rotary_forward and _backward against their 64-bit definition.

Bounds, C = 2^-20 standing for 16 roundings of 2^-24: the sum of a head's squares is a chain of at most 16 terms and a tree of 6 levels, its root
and quotient add four roundings, of which the root halves the sum's: 15; cosine and sine are good to 2^-22, a turned element is a sum of two
products, 4 * 2^-22 = C of the pair's length.  So `out` is within 2 C and two roundings, 2.25 C, of the pair's length, and half a step of
its type.  Backwards, g is within 1.25 C of its pair's length L; the mean of g w u adds 22 roundings: within 4 C of (L w + |u| mean(L w |u|)) r, and
half a step.  dweight: 3.5 C of the sum of L |u| for what is added up, and what adding up leaves: chains of some terms in a lane, 256 groups of
lanes at most, 32 and 32 of the workgroups' sums, 352 roundings."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from paper_2504_03702_amd import binding as ps
from paper_2504_03702_amd import layers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
C = 2.0 ** -20
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def numpy(t):
    return None if t is None else t.detach().double().cpu().numpy()


def lengths(x, n, interleaved):
    """Every element's, or the length of the pair that it turns in."""
    x = np.abs(x)
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    size = np.hypot(a, b)
    a[...], b[...] = size, size
    return x


def check_forward(x, w, pos, f, out, eps, interleaved, magnitude):
    ref = ol.norm_rotate(numpy(x), numpy(w), numpy(pos), numpy(f), eps, interleaved, magnitude)
    length = lengths(ref, f.numel(), interleaved)
    assert np.all(np.abs(numpy(out) - ref) <= 2.25 * C * length + HALF[out.dtype] * (1 + C) * np.abs(ref) + HALF[out.dtype] * 2.25 * C * length + 1e-38)


def check_backward(x, w, pos, f, dout, dx, dw, eps, interleaved, magnitude):
    x64, w64 = numpy(x), np.ones(x.shape[2]) if w is None else numpy(w)
    rdx, rdw = ol.norm_rotate(x64, w64, numpy(pos), numpy(f), eps, interleaved, magnitude, numpy(dout))
    by = 1.0 / np.sqrt((x64 ** 2).mean(-1, keepdims=True) + eps)
    u = np.abs(x64 * by)
    g = lengths(ol.rotate(numpy(dout), numpy(pos), numpy(f), interleaved, magnitude, inverse=True), f.numel(), interleaved)
    lw = g * np.abs(w64)
    bound = 4 * C * by * (lw + u * (lw * u).mean(-1, keepdims=True))
    assert np.all(np.abs(numpy(dx) - rdx) <= bound * (1 + HALF[dx.dtype]) + HALF[dx.dtype] * np.abs(rdx) + 1e-38)
    if dw is not None:
        assert np.all(np.abs(numpy(dw) - rdw) <= (3.5 * C + 352 * 2.0 ** -24) * (g * u).sum((0, 1)) + 1e-38)


def made(rows, heads, size, dtype, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return [torch.randn(rows, h, size, generator=g, device=DEV).to(dtype) for h in heads]


def places(rows, top=4096):
    return torch.tensor(np.random.default_rng(rows).integers(0, top, rows), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("size,pairs", [(64, 32), (128, 32), (128, 64), (80, 20), (64, 4), (7, 2), (6, 3), (256, 128), (2, 1), (1, 0), (40, 0), (512, 256),
                                        (511, 255), (508, 126), (300, 25)])
@pytest.mark.parametrize("rows", [1, 5, 1030])
def test_sizes(dtype, interleaved, size, pairs, rows):
    x, y, gx, gy = made(rows, (3, 2, 3, 2), size, dtype, size + rows)
    w, w2 = (1 + 0.3 * torch.randn(size, device=DEV) for _ in range(2))
    w, w2 = w.to(dtype), w2.to(dtype)
    pos, f = places(rows), ps.ps_rotary_frequencies(pairs).to(DEV) if pairs else torch.empty(0, device=DEV)
    how = dict(eps=1e-5, interleaved=interleaved, magnitude=1.25)
    ox, oy = torch.full_like(x, 7.0), torch.full_like(y, 7.0)
    ps.ps_norm_rotary_forward(x, w, pos, f, ox, y, w2, oy, **how)
    check_forward(x, w, pos, f, ox, **how)
    check_forward(y, w2, pos, f, oy, **how)
    alone = x.clone()
    ps.ps_norm_rotary_forward(alone, w, pos, f, alone, **how)              # one tensor, in place
    assert torch.equal(alone, ox)
    ws = ps.alloc_workspace(ps.ps_norm_rotary_workspace_bytes(rows, 3, 2, size), DEV)
    ws.fill_(0xA5)
    dx, dy, dw, dw2 = torch.full_like(x, 7.0), torch.full_like(y, 7.0), torch.full((size,), 7.0, device=DEV), torch.full((size,), 7.0, device=DEV)
    ps.ps_norm_rotary_backward(x, w, pos, f, gx, dx, dw, ws, y, w2, gy, dy, dw2, **how)
    check_backward(x, w, pos, f, gx, dx, dw, **how)
    check_backward(y, w2, pos, f, gy, dy, dw2, **how)
    again, dw_again = gx.clone(), torch.empty_like(dw)                      # one tensor, in place of dout, without a weight
    ps.ps_norm_rotary_backward(x, None, pos, f, again, again, dw_again, ws, **how)
    check_backward(x, None, pos, f, gx, again, dw_again, **how)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_rows_add_up_the_same_every_time(dtype):
    rows = 9001
    x, y, gx, gy = made(rows, (4, 1, 4, 1), 64, dtype, 3)
    w, pos, f = torch.ones(64, device=DEV, dtype=dtype), places(rows, 1 << 20), ps.ps_rotary_frequencies(32).to(DEV)
    ws = ps.alloc_workspace(ps.ps_norm_rotary_workspace_bytes(rows, 4, 1, 64), DEV)
    seen = []
    for fill in (0, 0xFF):
        ws.fill_(fill)
        dx, dy, dw, dw2 = torch.empty_like(x), torch.empty_like(y), torch.empty(64, device=DEV), torch.empty(64, device=DEV)
        ps.ps_norm_rotary_backward(x, w, pos, f, gx, dx, dw, ws, y, w, gy, dy, dw2)
        seen.append((dx, dy, dw, dw2))
    assert all(torch.equal(a, b) for a, b in zip(*seen))
    check_backward(x, w, pos, f, gx, dx, dw, 1e-6, False, 1.0)
    check_backward(y, w, pos, f, gy, dy, dw2, 1e-6, False, 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
def test_slices_of_a_projection(dtype, offset):
    """Queries and keys inside the output of one map, from any element on; what lies between stays as it was."""
    n, size = 37, 64
    packed = torch.randn(n, 8 * size + 8, device=DEV).to(dtype)
    before = packed.clone()
    q, k = (packed[:, at:at + h * size].unflatten(1, (h, size)) for at, h in ((offset, 4), (offset + 5 * size, 2)))
    w, pos, f = torch.randn(size, device=DEV).to(dtype), places(n), ps.ps_rotary_frequencies(16).to(DEV)
    q0, k0 = q.clone(), k.clone()
    ps.ps_norm_rotary_forward(q, w, pos, f, q, k, w, k)
    check_forward(q0, w, pos, f, q, 1e-6, False, 1.0)
    check_forward(k0, w, pos, f, k, 1e-6, False, 1.0)
    q.copy_(q0), k.copy_(k0)
    assert torch.equal(packed, before)
    by_head = torch.randn(4, n, size, device=DEV).to(dtype).transpose(0, 1)   # heads further apart than rows
    out = torch.empty(4, n, size, device=DEV, dtype=dtype).transpose(0, 1)
    ps.ps_norm_rotary_forward(by_head, w, pos, f, out)
    check_forward(by_head, w, pos, f, out, 1e-6, False, 1.0)


def test_nothing_to_do_and_nothing_to_go_by():
    f, pos = ps.ps_rotary_frequencies(4).to(DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    x = torch.empty(0, 2, 8, device=DEV)
    ws, dw = ps.alloc_workspace(ps.ps_norm_rotary_workspace_bytes(0, 2, 0, 8), DEV), torch.full((8,), 7.0, device=DEV)
    ps.ps_norm_rotary_forward(x, None, pos, f, x)
    ps.ps_norm_rotary_backward(x, None, pos, f, x, x, dw, ws)
    assert torch.equal(dw, torch.zeros(8, device=DEV))
    # rows of zeros, of the smallest and of the largest values; a row that is none, alone
    x = torch.ones(5, 1, 64, device=DEV)
    x[0], x[1], x[2], x[3, 0, 5] = 0.0, 1e-20, 1e18, float("nan")
    out = torch.empty_like(x)
    ps.ps_norm_rotary_forward(x, None, None, None, out)
    assert torch.equal(out[0], torch.zeros_like(out[0])) and torch.allclose(out[2], torch.ones_like(out[2])) and torch.isnan(out[3]).all()
    assert torch.allclose(out[1], torch.full_like(out[1], 1e-17)) and torch.isfinite(out[4]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layer_function_has_the_gradients(dtype):
    x, y, gx, gy = made(50, (4, 2, 4, 2), 32, dtype, 8)
    x, y = x.requires_grad_(), y.requires_grad_()
    w, w2 = torch.randn(32, device=DEV).to(dtype).requires_grad_(), torch.randn(32, device=DEV).to(dtype).requires_grad_()
    pos, f = places(50), ps.ps_rotary_frequencies(16).to(DEV)
    q, k = layers.norm_rotary(x, y, w, w2, pos, f)
    dx, dy, dw, dw2 = torch.autograd.grad((q, k), (x, y, w, w2), (gx, gy))
    check_forward(x, w, pos, f, q, 1e-6, False, 1.0)
    check_backward(x, w, pos, f, gx, dx, None, 1e-6, False, 1.0)
    check_backward(y, w2, pos, f, gy, dy, None, 1e-6, False, 1.0)
    rdw = [ol.norm_rotate(numpy(a), numpy(b), numpy(pos), numpy(f), dout=numpy(g))[1] for a, b, g in ((x, w, gx), (y, w2, gy))]
    for got, ref in zip((dw, dw2), rdw):
        assert got.dtype == dtype and np.abs(numpy(got) - ref).max() <= (HALF[dtype] + 1e-5) * np.abs(ref).max() + 1e-4
    q, k = layers.norm_rotary(x, y, None, None, None, None)                # the keys' part of the gradients alone
    (dy,) = torch.autograd.grad(k, y, gy)
    check_backward(y, None, pos, f[:0], gy, dy, None, 1e-6, False, 1.0)
    with pytest.raises(ValueError):
        layers.norm_rotary(x, y, w, w2, pos, f.clone().requires_grad_())


@pytest.mark.parametrize("direction", ["forward", "backward"])
def test_another_stream_and_a_graph(direction):
    n, size = 300, 64
    x, g = made(n, (4, 4), size, torch.bfloat16, 2)
    w, pos, f = torch.randn(size, device=DEV).bfloat16(), places(n), ps.ps_rotary_frequencies(32).to(DEV)
    out, dw = torch.empty_like(x), torch.empty(size, device=DEV)
    ws = ps.alloc_workspace(ps.ps_norm_rotary_workspace_bytes(n, 4, 0, size), DEV)

    def call():
        if direction == "forward":
            ps.ps_norm_rotary_forward(x, w, pos, f, out)
        else:
            ps.ps_norm_rotary_backward(x, w, pos, f, g, out, dw, ws)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        x.copy_(made(n, (4,), size, torch.bfloat16, 10 + seed)[0])
        out.zero_(), dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), dw.clone()
        out.zero_(), dw.zero_()
        call()
        assert torch.equal(got[0], out) and torch.equal(got[1], dw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("place", ["x", "dout"])
def test_gradients_past_all_numbers_in_place(dtype, place):
    """A head of zeros under a small eps has a dx that no number holds and adds nothing to dweight, in place as elsewhere.  (80 heads of a tile are 64 and 16: lanes without
    one read the tile's last head again, whose dx may be there by then.)"""
    rows = 16 * 512
    x, g = made(rows, (5, 5), 64, dtype, 12)
    x[15::16, 4] = 0.0
    g[15::16, 4] *= 1e25
    w, pos, f = torch.ones(64, device=DEV, dtype=dtype), places(rows), ps.ps_rotary_frequencies(32).to(DEV)
    ws = ps.alloc_workspace(ps.ps_norm_rotary_workspace_bytes(rows, 5, 0, 64), DEV)
    dx, dw, dw_again = torch.empty_like(x), torch.empty(64, device=DEV), torch.empty(64, device=DEV)
    ps.ps_norm_rotary_backward(x, w, pos, f, g, dx, dw, ws, eps=1e-37)
    assert torch.isfinite(dw).all() and not torch.isfinite(dx[15::16, 4]).any()
    own = {"x": x, "dout": g}[place].clone()
    ps.ps_norm_rotary_backward(own if place == "x" else x, w, pos, f, own if place == "dout" else g, own, dw_again, ws, eps=1e-37)
    assert torch.equal(dw, dw_again) and torch.equal(dx.nan_to_num(), own.nan_to_num())
