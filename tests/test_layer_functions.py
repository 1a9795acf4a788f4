"""The layer functions around the kernels: what they hand over, keep for the gradients and refuse.  The 64-bit definitions stand in
for the kernels, on the CPU, and write what those write: rows of sequences that keep the rules, no others."""
import numpy as np
import pytest
import torch
from torch.utils.checkpoint import checkpoint

from oracle import layer as ol
from paper_2504_03702_amd import binding as ps
from paper_2504_03702_amd import layers


def of(t):
    return None if t is None else t.detach().double().numpy()


def put(to, rows):
    """Rows that the definition has (the others are NaN there) into a call's tensor."""
    rows = torch.from_numpy(rows)
    there = ~rows.isnan()
    to[there] = rows[there].to(to.dtype)


def attention(q, k, v, q_offsets, k_offsets, max_q, max_k, softcap, causal, slopes, status, **how):
    """A call's sequences that keep the rules: (out, lse) or the gradients too."""
    dout = how.pop("dout", None)
    n = q_offsets.diff().tolist()
    good = [i for i in range(len(n)) if n[i] <= max_q and k_offsets.diff()[i] <= max_k]
    if len(good) < len(n) and status is not None:
        status[0] = ps.PS_ST_BAD_LENGTH
    q_docs, k_docs = how.pop("q_docs"), how.pop("k_docs")
    got = None
    for i in good:
        rows, keys = slice(*q_offsets[i:i + 2].tolist()), slice(*k_offsets[i:i + 2].tolist())
        one = {m: None if t is None else t[i:i + 1].numpy() for m, t in how.items()}
        offsets = ([0, rows.stop - rows.start], [0, keys.stop - keys.start])
        parts = ol.attention(of(q)[rows], of(k)[keys], of(v)[keys], *offsets, causal=causal, cap=softcap, slopes=of(slopes),
                             q_docs=None if q_docs is None else q_docs[rows].numpy(), k_docs=None if k_docs is None else k_docs[keys].numpy(),
                             dout=None if dout is None else of(dout)[rows], **one)
        if got is None:
            got = [np.full(s, np.nan) for s in (q.shape, (q.shape[1], q.shape[0]), q.shape, k.shape, k.shape)][:len(parts)]
        for to, part, at in zip(got, parts, (rows, (slice(None), rows), rows, keys, keys)):
            to[at] = part
    return got


@pytest.fixture
def stand_ins(monkeypatch):
    """The calls made, by name; tensors that are not filled on purpose hold NaN."""
    calls = []

    def forward(q, k, v, q_offsets, k_offsets, max_q, max_k, out, lse, workspace, scale=None, softcap=0.0, causal=False, slopes=None,
                status=None, out_rest=None, **how):
        calls.append(("forward", status))
        for to, rows in zip((out, lse), attention(q, k, v, q_offsets, k_offsets, max_q, max_k, softcap, causal, slopes, status, **how) or ()):
            put(to, rows)
        if out_rest is not None:
            out_rest.zero_()

    def backward(q, k, v, out, lse, dout, q_offsets, k_offsets, max_q, max_k, dq, dk, dv, workspace, scale=None, softcap=0.0, causal=False,
                 slopes=None, status=None, out_rest=None, **how):
        calls.append(("backward", status))
        if dout.data_ptr() % 16:
            raise ps.PsError(-1, "dout")
        got = attention(q, k, v, q_offsets, k_offsets, max_q, max_k, softcap, causal, slopes, status, dout=dout, **how)
        for to, rows in zip((dq, dk, dv), got[2:] if got else ()):
            put(to, rows)

    def rotary(x, positions, frequencies, out, x2=None, out2=None, interleaved=False, magnitude=1.0, inverse=False):
        for t, to in ((x, out), (x2, out2)):
            put(to, ol.rotate(of(t), positions.numpy(), of(frequencies), interleaved, magnitude, inverse))

    def dropout(x, bias, residual, rng, p, out):
        calls.append(("dropout", tuple(rng.tolist())))
        put(out, ol.dropout(of(x), of(bias), of(residual), *rng.tolist(), p))

    def dropout_gradients(dout, rng, p, dx, dbias, workspace):
        calls.append(("dropout gradients", tuple(rng.tolist())))
        for to, rows in zip((dx, dbias), ol.dropout_gradients(of(dout), *rng.tolist(), p)):
            if to is not None:
                put(to, rows)

    for name, f in (("attention_forward", forward), ("attention_backward", backward), ("rotary", rotary), ("dropout_forward", dropout),
                    ("dropout_backward", dropout_gradients)):
        monkeypatch.setattr(ps, "ps_" + name, f)
    real = torch.empty

    def empty(*a, **k):
        t = real(*a, **k)
        return t.fill_(float("nan")) if t.is_floating_point() and not t.requires_grad else t

    monkeypatch.setattr(torch, "empty", empty)
    return calls


def drawn(*shapes, dtype=torch.float32, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g).to(dtype).requires_grad_() for s in shapes]


def gradients_of(out, inputs, g):
    """By backward(): a region that is made again the older way takes no other."""
    for t in inputs:
        t.grad = None
    out.backward(g)
    return [t.grad for t in inputs]


def offsets(*at):
    return torch.tensor(at, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_no_sequence_are_zeros(stand_ins, dtype):
    """And what follows on them stays finite: their gradient is zero, but zero times NaN is not."""
    q, k, v = drawn((10, 2, 16), (10, 2, 16), (10, 2, 16), dtype=dtype)
    (w,) = drawn((32, 8), dtype=dtype, seed=1)
    out = layers.attention(q, k, v, layers.Sequences(offsets(2, 6), offsets(0, 4), 4, 4))
    assert torch.all(out[:2] == 0) and torch.all(out[6:] == 0) and torch.all(out[2:6] != 0)
    (out.reshape(10, 32) @ w)[2:6].sum().backward()
    assert all(torch.isfinite(t.grad).all() for t in (q, k, v, w))


def test_faulty_sequences_are_told(stand_ins):
    q, k, v = drawn((10, 2, 16), (10, 2, 16), (10, 2, 16))
    status = torch.zeros(2, dtype=torch.int64)
    out = layers.attention(q, k, v, layers.Sequences(offsets(0, 4, 10), offsets(0, 4, 10), 5, 5, status=status))
    assert status[0] == ps.PS_ST_BAD_LENGTH and torch.all(out[4:] == 0) and torch.all(out[:4] != 0)
    out.sum().backward()
    assert [s is status for _, s in stand_ins] == [True, True]
    assert all(torch.all(t.grad[4:] == 0) for t in (q, k, v))


@pytest.mark.parametrize("reentrant", [False, True])
def test_recomputed_passes_draw_the_same_masks(stand_ins, reentrant):
    """Two masks in a region whose activations are made again: the gradients are those of the pass that was kept, bit for bit."""
    (x, b), g = drawn((40, 24), (24,)), torch.randn(40, 24)

    def region(x, b, rng):
        y = layers.dropout_add(x, b, x, rng, 0.5, move_on=False)
        return layers.dropout_add(y * y, None, y, rng + rng.new_tensor([0, 1]), 0.5, move_on=False)

    grads = []
    for again in (False, True):
        rng = torch.tensor([3, 7])
        out = checkpoint(region, x, b, rng, use_reentrant=reentrant) if again else region(x, b, rng)
        grads.append((out, *gradients_of(out, (x, b), g)))
        assert rng.tolist() == [3, 7]
    assert all(torch.equal(a, c) for a, c in zip(*grads))


@pytest.mark.parametrize("reentrant", [False, True])
def test_recomputed_passes_do_not_move_on(stand_ins, reentrant):
    (x,), rng = drawn((40, 24)), torch.tensor([3, 7])
    out = checkpoint(lambda x: layers.dropout_add(x, None, None, rng, 0.5), x, use_reentrant=reentrant)
    assert rng.tolist() == [3, 8]
    with pytest.raises(RuntimeError, match="move_on=False"):
        out.sum().backward()
    assert rng.tolist() == [3, 8]


def test_masks_stay_until_the_gradients_are_taken(stand_ins):
    (x,), rng = drawn((40, 24)), torch.tensor([3, 7])
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
def test_second_derivatives_are_refused(stand_ins, what, weight):
    """Gradients with a graph can be had, and are right; to differentiate them is an error, not nothing."""
    q, k, v = drawn((4, 2, 16), (4, 2, 16), (4, 2, 16))
    (w,) = drawn((4, 2, 16), seed=1)
    if what == "attention":
        out = layers.attention(q, k, v, layers.Sequences(offsets(0, 4), offsets(0, 4), 4, 4))
    elif what == "rotary":
        out = sum(layers.rotary(q, k, offsets(0, 1, 2, 3), torch.ones(8)))
    else:
        out = layers.dropout_add(q.view(8, 16), None, None, torch.tensor([1, 1]), 0.1).view(4, 2, 16)
    loss = (out * w).sum() if weight else out.sum()
    (plain,) = torch.autograd.grad(loss, q, retain_graph=True)
    (again,) = torch.autograd.grad(loss, q, create_graph=True)
    assert torch.equal(plain, again)
    with pytest.raises(RuntimeError, match="no second derivatives"):
        (loss + again.square().sum()).backward()


@pytest.mark.parametrize("name", ["q_offsets", "k_offsets", "k_lengths", "q_start", "prefix", "q_docs", "k_docs", "slopes"])
def test_what_gradients_depend_on_may_not_be_written_again(stand_ins, name):
    q, k, v = drawn((4, 2, 16), (4, 2, 16), (4, 2, 16))
    more = dict(k_lengths=offsets(3), q_start=offsets(0), prefix=offsets(1), q_docs=offsets(0, 0, 1, 1), k_docs=offsets(0, 0, 1, 1))
    seqs, slopes = layers.Sequences(offsets(0, 4), offsets(0, 4), 4, 4, **more), torch.ones(2)
    for change in (False, True):
        out = layers.attention(q, k, v, seqs, causal=True, slopes=slopes)
        if not change:
            out.sum().backward()
            continue
        (slopes if name == "slopes" else getattr(seqs, name)).add_(1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.sum().backward()


def test_constants_that_want_a_gradient_are_refused(stand_ins):
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
def test_incoming_gradients_lie_at_any_address(stand_ins, dtype):
    (q, k, v, first), seqs = drawn((4, 2, 16), (4, 2, 16), (4, 2, 16), (1,), dtype=dtype), layers.Sequences(offsets(0, 4), offsets(0, 4), 4, 4)
    (w,) = drawn((129,), dtype=dtype, seed=1)
    want = torch.autograd.grad((layers.attention(q, k, v, seqs).reshape(-1) * w[1:]).sum(), (q, k, v))
    got = torch.autograd.grad((torch.cat((first, layers.attention(q, k, v, seqs).reshape(-1))) * w).sum(), (q, k, v))
    assert all(torch.equal(a, b) for a, b in zip(want, got))
