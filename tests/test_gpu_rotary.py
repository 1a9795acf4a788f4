"""ps_rotary against its 64-bit definition.

Bounds: cosine and sine of a reduced angle are good to 2^-22 (the angle's float, the function's last places), a result is a sum of
two products: 4 * 2^-22 of the pair's length in fp32, and one rounding, 2^-8, more in bf16."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from paper_2504_03702_amd import binding as ps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def positions(n, top, seed=0):
    return torch.tensor(np.random.default_rng(seed).integers(0, top, n), dtype=torch.int32, device=DEV)


def check(x, pos, f, out, interleaved, magnitude, inverse):
    ref = ol.rotate(x, pos.cpu().numpy(), f.cpu().numpy(), interleaved, magnitude, inverse)
    got = out.double().cpu().numpy()
    n = f.numel()
    length = np.abs(ref).copy()
    a, b = (length[..., 0:2 * n:2], length[..., 1:2 * n:2]) if interleaved else (length[..., :n], length[..., n:2 * n])
    size = np.hypot(a, b)
    a[...], b[...] = size, size
    bound = 4 * 2.0 ** -22 + (2.0 ** -8 if out.dtype == torch.bfloat16 else 0.0)
    assert np.all(np.abs(got - ref)[..., :2 * n] <= bound * length[..., :2 * n] + 1e-30)
    assert np.array_equal(got[..., 2 * n:], ref[..., 2 * n:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("size,pairs", [(64, 32), (128, 32), (128, 64), (80, 40), (64, 4), (6, 3), (7, 2), (256, 128), (2, 1), (10, 0)])
@pytest.mark.parametrize("rows", [1, 5, 1030])
def test_sizes(dtype, interleaved, size, pairs, rows):
    g = torch.Generator(device=DEV)
    g.manual_seed(size + rows)
    x, y = (torch.randn(rows, h, size, generator=g, device=DEV).to(dtype) for h in (3, 2))
    pos, f = positions(rows, 4096), ps.ps_rotary_frequencies(pairs).to(DEV) if pairs else torch.empty(0, device=DEV)
    for inverse in (False, True):
        ox, oy = torch.full_like(x, 7.0), torch.full_like(y, 7.0)
        ps.ps_rotary(x, pos, f, ox, y, oy, interleaved, 1.25, inverse)
        check(x.double().cpu().numpy(), pos, f, ox, interleaved, 1.25, inverse)
        check(y.double().cpu().numpy(), pos, f, oy, interleaved, 1.25, inverse)
        alone = torch.full_like(x, 7.0)
        ps.ps_rotary(x, pos, f, alone, interleaved=interleaved, magnitude=1.25, inverse=inverse)
        assert torch.equal(alone, ox)
        where = x.clone()
        ps.ps_rotary(where, pos, f, where, interleaved=interleaved, magnitude=1.25, inverse=inverse)
        assert torch.equal(where, ox)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("size,pairs", [(80, 20), (12, 4), (20, 2), (6, 2), (4, 2)])
@pytest.mark.parametrize("rows", [3, 700])
def test_sizes_of_eight_bytes(dtype, interleaved, size, pairs, rows):
    test_sizes(dtype, interleaved, size, pairs, rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_positions_anywhere(dtype):
    """The fastest pair turns 2^31 radians: the fraction of a turn is what counts."""
    pos = torch.tensor([0, 1, -1, 131071, 16777217, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV)
    x = torch.randn(7, 2, 64, device=DEV).to(dtype)
    f = ps.ps_rotary_frequencies(32).to(DEV)
    out = torch.empty_like(x)
    ps.ps_rotary(x, pos, f, out)
    check(x.double().cpu().numpy(), pos, f, out, False, 1.0, False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
def test_strides_and_alignment(dtype, offset):
    """Queries and keys inside a packed projection, in place; a head that starts at any element."""
    n, size = 37, 64
    packed = torch.randn(n, 8 * size + 8, device=DEV).to(dtype)
    before = packed.clone()
    view = packed[:, offset:offset + 6 * size].view(n, 6, size) if offset == 0 else packed.as_strided((n, 6, size), (8 * size + 8, size, 1), offset)
    q, k = view[:, :4], view[:, 4:]
    pos, f = positions(n, 1000), ps.ps_rotary_frequencies(16).to(DEV)
    want = [torch.empty(t.shape, dtype=dtype, device=DEV) for t in (q, k)]
    ps.ps_rotary(q.contiguous(), pos, f, want[0], k.contiguous(), want[1], True)
    ps.ps_rotary(q, pos, f, q, k, k, True)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    q.copy_(before.as_strided(q.shape, q.stride(), q.storage_offset()))
    k.copy_(before.as_strided(k.shape, k.stride(), k.storage_offset()))
    assert torch.equal(packed, before)
    heads_first = torch.randn(3, n, size, device=DEV).to(dtype).transpose(0, 1)
    out = torch.empty(3, n, size, dtype=dtype, device=DEV).transpose(0, 1)
    ps.ps_rotary(heads_first, pos, f, out)
    check(heads_first.double().cpu().numpy(), pos, f, out, False, 1.0, False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_is_the_turn_back(dtype):
    """<R x, y> = <x, R^T y> to the rounding of the results, and by differences of the fp32 call."""
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    x, y = (torch.randn(50, 4, 64, generator=g, device=DEV).to(dtype) for _ in range(2))
    pos, f = positions(50, 100000), ps.ps_rotary_frequencies(32, scaling=ps.PS_ROTARY_PARTS, factor=8.0, trained_len=4096).to(DEV)
    rx, ry = torch.empty_like(x), torch.empty_like(y)
    ps.ps_rotary(x, pos, f, rx, magnitude=1.2)
    ps.ps_rotary(y, pos, f, ry, magnitude=1.2, inverse=True)
    left, right = (rx.double() * y.double()).sum().item(), (x.double() * ry.double()).sum().item()
    eps = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -20
    assert abs(left - right) <= 4 * eps * (rx.double() * y.double()).norm().item()
    if dtype == torch.float32:
        for i in ((0, 0, 0), (7, 3, 40), (49, 2, 63)):
            up = x.clone()
            up[i] += 1.0                                   # (linear: any step does)
            out = torch.empty_like(x)
            ps.ps_rotary(up, pos, f, out, magnitude=1.2)
            assert abs(((out.double() - rx.double()) * y.double()).sum().item() - ry[i].item()) < 1e-4


def test_no_rows_and_a_graph():
    f = ps.ps_rotary_frequencies(32).to(DEV)
    x = torch.empty(0, 2, 64, device=DEV)
    ps.ps_rotary(x, positions(0, 5), f, torch.empty_like(x))
    x, pos = torch.randn(9, 2, 64, device=DEV), positions(9, 100)
    out = torch.empty_like(x)
    ps.ps_rotary(x, pos, f, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ps.ps_rotary(x, pos, f, out)
    for step in range(3):
        pos += 1
        want = torch.empty_like(x)
        ps.ps_rotary(x, pos, f, want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("change,error", [
    (dict(x=lambda t: t.half()), TypeError), (dict(x=lambda t: t.cpu()), TypeError), (dict(out=lambda t: t.float()), TypeError),
    (dict(out=lambda t: t[:-1]), ValueError), (dict(positions=lambda t: t[:-1]), ValueError), (dict(positions=lambda t: t.long()), TypeError),
    (dict(frequencies=lambda t: torch.ones(33, device=DEV)), ps.PsError), (dict(x2=lambda t: torch.empty(9, 2, 64, device=DEV)), TypeError),
    (dict(out=lambda t: t[:, :1].expand(-1, 2, -1)), ps.PsError), (dict(frequencies=lambda t: t.double()), TypeError)])
def test_refusals(change, error):
    args = dict(x=torch.ones(9, 2, 64, device=DEV, dtype=torch.bfloat16), positions=positions(9, 5), frequencies=ps.ps_rotary_frequencies(32).to(DEV),
                out=torch.empty(9, 2, 64, device=DEV, dtype=torch.bfloat16), x2=None)
    ps.ps_rotary(**args)
    args.update({n: f(args[n]) for n, f in change.items()})
    with pytest.raises(error):
        ps.ps_rotary(**args)
