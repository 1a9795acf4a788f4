"""The layer functions with the kernels behind them: rows that no sequence has, faulty sequences, recomputed passes, what is written
again before the gradients are taken.  What they do is exact: zeros, flags, errors, the same bits."""
import numpy as np
import pytest
import torch
from torch.utils.checkpoint import checkpoint

from oracle import layer as ol
from paper_2504_03702_amd import binding as ps
from paper_2504_03702_amd import layers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def drawn(*shapes, dtype=torch.float32, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return [torch.randn(s, generator=g, device=DEV).to(dtype).requires_grad_() for s in shapes]


def gradients_of(out, inputs, g):
    """By backward(): a region that is made again the older way takes no other."""
    for t in inputs:
        t.grad = None
    out.backward(g)
    return [t.grad for t in inputs]


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


def test_faulty_sequences_are_told():
    q, k, v = drawn((10, 2, 16), (10, 2, 16), (10, 2, 16))
    status = ps.new_status(DEV)
    leave_nan(q.shape, dtype=torch.float32)
    out = layers.attention(q, k, v, layers.Sequences(offsets(0, 4, 10), offsets(0, 4, 10), 5, 5, status=status))
    assert ps.ps_status_read(status) == (ps.PS_ST_BAD_LENGTH, 1) and torch.all(out[4:] == 0) and torch.all(out[:4] != 0)
    status.zero_()
    out.sum().backward()
    assert ps.ps_status_read(status)[0] == ps.PS_ST_BAD_LENGTH
    assert all(torch.all(t.grad[4:] == 0) for t in (q, k, v))


@pytest.mark.parametrize("reentrant", [False, True])
def test_recomputed_passes_draw_the_same_masks(reentrant):
    """Two masks in a region whose activations are made again: the gradients are those of the pass that was kept, bit for bit."""
    (x, b), g = drawn((40, 24), (24,)), torch.randn(40, 24, device=DEV)

    def region(x, b, rng):
        y = layers.dropout_add(x, b, x, rng, 0.5, move_on=False)
        return layers.dropout_add(y * y, None, y, rng + rng.new_tensor([0, 1]), 0.5, move_on=False)

    grads = []
    for again in (False, True):
        rng = torch.tensor([3, 7], device=DEV)
        out = checkpoint(region, x, b, rng, use_reentrant=reentrant) if again else region(x, b, rng)
        grads.append((out, *gradients_of(out, (x, b), g)))
        assert rng.tolist() == [3, 7]
    assert all(torch.equal(a, c) for a, c in zip(*grads))


@pytest.mark.parametrize("reentrant", [False, True])
def test_recomputed_passes_do_not_move_on(reentrant):
    (x,), rng = drawn((40, 24)), torch.tensor([3, 7], device=DEV)
    out = checkpoint(lambda x: layers.dropout_add(x, None, None, rng, 0.5), x, use_reentrant=reentrant)
    assert rng.tolist() == [3, 8]
    with pytest.raises(RuntimeError, match="move_on=False"):
        out.sum().backward()
    assert rng.tolist() == [3, 8]


def test_masks_stay_until_the_gradients_are_taken():
    (x,), rng = drawn((40, 24)), torch.tensor([3, 7], device=DEV)
    kept = layers.dropout_add(x, None, None, rng, 0.5)
    rng[1:].add_(1)
    kept.sum().backward()                                      # (of a number of its own)
    assert torch.equal(x.grad, torch.tensor(ol.dropout_gradients(np.ones((40, 24)), 3, 7, 0.5)[0]).to(x.grad))
    kept = layers.dropout_add(x, None, None, rng, 0.5, move_on=False)
    rng[1:].add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.sum().backward()


@pytest.mark.parametrize("what", ["attention", "rotary", "dropout"])
@pytest.mark.parametrize("weight", [False, True])
def test_second_derivatives_are_refused(what, weight):
    """Gradients with a graph can be had, and are right; to differentiate them is an error, not nothing."""
    q, k, v = drawn((4, 2, 16), (4, 2, 16), (4, 2, 16))
    (w,) = drawn((4, 2, 16), seed=1)
    if what == "attention":
        out = layers.attention(q, k, v, layers.Sequences(offsets(0, 4), offsets(0, 4), 4, 4))
    elif what == "rotary":
        out = sum(layers.rotary(q, k, offsets(0, 1, 2, 3), torch.ones(8, device=DEV)))
    else:
        out = layers.dropout_add(q.view(8, 16), None, None, torch.tensor([1, 1], device=DEV), 0.1).view(4, 2, 16)
    loss = (out * w).sum() if weight else out.sum()
    (plain,) = torch.autograd.grad(loss, q, retain_graph=True)
    (again,) = torch.autograd.grad(loss, q, create_graph=True)
    assert torch.equal(plain, again)
    with pytest.raises(RuntimeError, match="no second derivatives"):
        (loss + again.square().sum()).backward()


@pytest.mark.parametrize("name", ["q_offsets", "k_offsets", "k_lengths", "q_start", "prefix", "q_docs", "k_docs", "slopes"])
def test_what_gradients_depend_on_may_not_be_written_again(name):
    q, k, v = drawn((4, 2, 16), (4, 2, 16), (4, 2, 16))
    more = dict(k_lengths=offsets(3), q_start=offsets(0), prefix=offsets(1), q_docs=offsets(0, 0, 1, 1), k_docs=offsets(0, 0, 1, 1))
    seqs, slopes = layers.Sequences(offsets(0, 4), offsets(0, 4), 4, 4, **more), torch.ones(2, device=DEV)
    for change in (False, True):
        out = layers.attention(q, k, v, seqs, causal=True, slopes=slopes)
        if not change:
            out.sum().backward()
            continue
        (slopes if name == "slopes" else getattr(seqs, name)).add_(1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.sum().backward()


def test_constants_that_want_a_gradient_are_refused():
    q, k, v, slopes, f = drawn((4, 2, 16), (4, 2, 16), (4, 2, 16), (2,), (8,))
    seqs = layers.Sequences(offsets(0, 4), offsets(0, 4), 4, 4)
    with pytest.raises(ValueError, match="slopes"):
        layers.attention(q, k, v, seqs, slopes=slopes)
    with pytest.raises(ValueError, match="frequencies"):
        layers.rotary(q, k, offsets(0, 1, 2, 3), f)
    layers.attention(q, k, v, seqs, slopes=slopes.detach())
    with torch.no_grad():
        layers.attention(q, k, v, seqs, slopes=slopes)
        layers.rotary(q, k, offsets(0, 1, 2, 3), f)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_incoming_gradients_lie_at_any_address(dtype):
    (q, k, v, first), seqs = drawn((4, 2, 16), (4, 2, 16), (4, 2, 16), (1,), dtype=dtype), layers.Sequences(offsets(0, 4), offsets(0, 4), 4, 4)
    (w,) = drawn((129,), dtype=dtype, seed=1)
    want = torch.autograd.grad((layers.attention(q, k, v, seqs).reshape(-1) * w[1:]).sum(), (q, k, v))
    got = torch.autograd.grad((torch.cat((first, layers.attention(q, k, v, seqs).reshape(-1))) * w).sum(), (q, k, v))
    assert all(torch.equal(a, b) for a, b in zip(want, got))
