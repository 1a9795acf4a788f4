"""ps_attention_forward / ps_attention_backward against their 64-bit definition.

Bounds, from the arithmetic: fp32 calls keep scores to a few units of 2^-24 of their size (up to 30 here, in powers of two), which
is the relative error of a weight: 30 * 3 * 2^-24 = 5e-6, and twice that where a gradient takes the difference of two sums.  bf16
calls round each weight and each output, 2^-8 at most each and 1.7e-3 in the mean square, and g once more: 5e-3 forwards and 8e-3
backwards of the tensor's norm, and 8 times that of any single value against the tensor's root mean square (a value that cancels
keeps the rounding of what it was made of)."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from paper_2504_03702_amd import binding as ps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BOUNDS = {torch.float32: (5e-6, 1e-5), torch.bfloat16: (5e-3, 8e-3)}


def near(got, ref, bound, what):
    got, ref = got.detach().double().cpu().numpy(), np.asarray(ref, np.float64)
    fine = np.isfinite(ref)
    assert np.array_equal(fine, np.isfinite(got)), what
    assert np.array_equal(got[~fine], ref[~fine]), what
    d, r = got[fine] - ref[fine], ref[fine]
    if r.size == 0:
        return
    rms = np.sqrt(np.mean(r ** 2))
    if rms == 0:
        assert np.all(d == 0), what
        return
    assert np.linalg.norm(d) <= bound * np.linalg.norm(r), (what, np.linalg.norm(d) / np.linalg.norm(r))
    assert np.max(np.abs(d) / np.maximum(np.abs(r), rms)) <= 8 * bound, (what, np.max(np.abs(d) / np.maximum(np.abs(r), rms)))


def i32(v):
    return None if v is None else torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


class Problem:
    """Sequences of given lengths, contents drawn; tensors as a call takes them."""

    def __init__(self, dtype, q_lens, k_lens, heads=4, kv_heads=2, size=64, seed=0, room=None, big=1.0, **how):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        spans = k_lens if room is None else [n + r for n, r in zip(k_lens, room)]
        self.dtype, self.how = dtype, how
        self.qo, self.ko = np.cumsum([0] + list(q_lens)), np.cumsum([0] + list(spans))
        self.k_lengths = None if room is None else np.array(k_lens)
        self.max_q, self.max_k = max([0, *q_lens]), max([0, *k_lens])
        normal = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)
        nq, nk = int(self.qo[-1]), int(self.ko[-1])
        self.q, self.k, self.v, self.dout = normal(nq, heads, size) * big, normal(nk, kv_heads, size), normal(nk, kv_heads, size), normal(nq, heads, size)
        self.status = ps.new_status(DEV)

    def arguments(self):
        h = self.how
        slopes = h.get("slopes")
        return dict(scale=h.get("scale"), softcap=h.get("cap", 0.0), causal=h.get("causal", False), k_lengths=i32(self.k_lengths),
                    q_start=i32(h.get("q_start")), prefix=i32(h.get("prefix")), q_docs=i32(h.get("q_docs")), k_docs=i32(h.get("k_docs")),
                    slopes=None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device=DEV), status=self.status)

    def workspace(self, backward):
        nb = ps.ps_attention_workspace_bytes(len(self.qo) - 1, self.q.shape[0], self.k.shape[0], self.max_q, self.max_k, self.q.shape[1],
                                             self.k.shape[1], self.q.shape[2], self.dtype, backward)
        assert nb > 0
        return torch.full((nb,), 0xFF, dtype=torch.uint8, device=DEV)        # (NaN wherever it is read before it is written)

    def forward(self, q=None, k=None, v=None, out=None):
        q, k, v = (a if b is None else b for a, b in ((self.q, q), (self.k, k), (self.v, v)))
        out = torch.full_like(self.q, 7.0) if out is None else out
        lse = torch.full((q.shape[1], q.shape[0]), 7.0, device=DEV)
        self.rest = torch.full(self.q.shape, 0.5, dtype=self.dtype, device=DEV) if self.dtype == torch.bfloat16 else None
        ps.ps_attention_forward(q, k, v, i32(self.qo), i32(self.ko), self.max_q, self.max_k, out, lse, self.workspace(False),
                                out_rest=self.rest, **self.arguments())
        return out, lse

    def backward(self, out, lse, dq=None, dk=None, dv=None):
        dq, dk, dv = (torch.full_like(a, 7.0) if b is None else b for a, b in ((self.q, dq), (self.k, dk), (self.v, dv)))
        ps.ps_attention_backward(self.q, self.k, self.v, out, lse, self.dout, i32(self.qo), i32(self.ko), self.max_q, self.max_k, dq, dk,
                                 dv, self.workspace(True), out_rest=self.rest, **self.arguments())
        return dq, dk, dv

    def both(self):
        """(out, lse, dq, dk, dv)"""
        o = self.forward()
        return (*o, *self.backward(*o))

    def reference(self, backward=True):
        h = dict(self.how)
        c = lambda t: t.float().cpu().numpy()
        if "slopes" in h:
            h["slopes"] = np.float32(h["slopes"])
        return ol.attention(c(self.q), c(self.k), c(self.v), self.qo, self.ko, k_lengths=self.k_lengths, dout=c(self.dout) if backward else None, **h)

    def check(self, backward=True):
        got = self.forward()
        if backward:
            got = (*got, *self.backward(*got))
        assert ps.ps_status_read(self.status) == (0, -1)
        ref = self.reference(backward)
        f, b = BOUNDS[self.dtype]
        for name, x, r, bound in zip(("out", "lse", "dq", "dk", "dv"), got, ref, (f, BOUNDS[torch.float32][0], b, b, b)):
            # rows that no sequence has are left alone
            keep = np.isnan(r) & (x.float().cpu().numpy() == 7.0)
            near(torch.where(torch.tensor(keep, device=DEV), torch.zeros_like(x, dtype=torch.float32), x.float()), np.where(keep, 0.0, r), bound, name)
        return got


SLOPES = [0.5, 0.25, 0.125, 0.0625]
LENGTHS = [1, 130, 0, 63, 64, 65, 2, 127, 129]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [8, 40, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("how", [dict(), dict(causal=True), dict(causal=True, cap=5.0, slopes=SLOPES)], ids=["all", "causal", "capped"])
def test_lengths_and_sizes(dtype, size, how):
    Problem(dtype, LENGTHS, LENGTHS, size=size, **how).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (5, 1), (6, 2), (12, 4)])
def test_shared_heads(dtype, heads, kv_heads):
    Problem(dtype, [70, 33, 1], [70, 33, 1], heads, kv_heads, causal=True, slopes=[0.5 / (h + 1) for h in range(heads)]).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("q_lens,k_lens", [([5, 1, 40], [200, 129, 40]), ([100, 7], [3, 0]), ([0, 3], [9, 5])])
def test_rows_at_the_end_of_longer_keys_and_before_shorter_ones(dtype, q_lens, k_lens):
    """More rows than keys: under a causal mask the first of them see nothing."""
    got = Problem(dtype, q_lens, k_lens, causal=True).check()
    if q_lens[0] == 100:
        assert torch.all(got[0][:97] == 0) and torch.all(got[1][:, :97] == -np.inf) and torch.all(got[2][:97] == 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_prefixes(dtype):
    Problem(dtype, [150, 64, 30, 90], [150, 64, 30, 90], causal=True, prefix=[97, 0, 30, 1000], slopes=SLOPES).check()
    Problem(dtype, [150, 20], [150, 90], causal=True, prefix=[-4, 75], q_start=[-30, 3]).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("order", ["sorted", "shuffled", "padding"])
def test_documents(dtype, causal, order):
    rng = np.random.default_rng(3)
    n = [300, 77, 128]
    docs = np.concatenate([np.sort(rng.integers(0, 5, m)) for m in n])
    if order == "shuffled":
        docs = rng.permutation(docs)
    if order == "padding":
        docs[100:170] = -1
        docs[300:377] = -5                                       # a whole sequence of it
    Problem(dtype, n, n, q_docs=docs, k_docs=docs, causal=causal).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_documents_of_rows_and_keys_apart(dtype):
    """A row may look for a document that no key has, and for one among other keys."""
    q_docs, k_docs = np.array([3, 4, 9, 3] + [0] * 60), np.array([4] * 40 + [3] * 50 + [0] * 10)
    Problem(dtype, [4, 60], [90, 10], q_docs=q_docs, k_docs=k_docs, slopes=SLOPES, heads=4, kv_heads=1).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("how", [dict(causal=True), dict(causal=True, cap=20.0, slopes=SLOPES), dict()], ids=["causal", "capped", "all"])
def test_single_tokens_over_long_keys(dtype, how):
    """Keys shared out over workgroups, some of which have none of a short sequence."""
    Problem(dtype, [1, 1, 3, 0], [5000, 700, 1, 64], **how).check(backward=False)
    Problem(dtype, [1], [2049], heads=16, kv_heads=1, size=128, **{**how, **({"slopes": [0.01 * h for h in range(16)]} if "slopes" in how else {})}).check(False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_scores_and_large_distances(dtype):
    """Weights that overflow without the running maximum, and a bias that leaves one key."""
    Problem(dtype, [100], [100], big=40.0, causal=True, cap=30.0).check()
    Problem(dtype, [130, 1], [130, 3000], slopes=[64.0, 8.0, 1.0, 0.01], causal=True).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), torch.finfo(torch.bfloat16).min])
def test_what_nobody_sees_does_not_matter(dtype, bad):
    """Room behind a cache's keys, and padding, hold anything."""
    p = Problem(dtype, [5, 70, 1], [90, 70, 1], room=[38, 1, 70], causal=True, slopes=SLOPES)
    for s in range(3):
        p.k[p.ko[s] + p.k_lengths[s]:p.ko[s + 1]] = bad
        p.v[p.ko[s] + p.k_lengths[s]:p.ko[s + 1]] = bad
    out, lse = p.forward()
    grads = p.backward(out, lse)
    ref = p.reference()
    f, b = BOUNDS[dtype]
    near(out, ref[0], f, "out")
    near(grads[0], ref[2], b, "dq")
    for g, r, name in zip(grads[1:], ref[3:], ("dk", "dv")):
        keep = np.isnan(r[:, 0, 0])
        assert torch.all(g[torch.tensor(keep)] == 7.0)
        near(g[torch.tensor(~keep)], r[~keep], b, name)

    docs = np.array([0] * 50 + [-1] * 30 + [1] * 60)
    p = Problem(dtype, [140], [140], q_docs=docs, k_docs=docs)
    clean = [t.clone() for t in p.both()]
    for t in (p.q, p.k, p.v, p.dout):
        t[50:80] = bad
    dirty = p.both()
    for a, c in zip(clean, dirty):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_scores_may_be_anything(dtype):
    """A key of NaN is seen by the rows from its own on: the rows in front of it have clean results, the others do not."""
    p = Problem(dtype, [200], [200], causal=True)
    p.k[150, 0, 3] = float("nan")
    out, lse = p.forward()
    ref = p.reference(False)
    near(out[:150], ref[0][:150], BOUNDS[dtype][0], "out")
    assert torch.isnan(out[150:, :2]).all() and torch.isnan(lse[:2, 150:]).all() and torch.isfinite(out[:, 2:]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides(dtype):
    """Slices of a packed projection, keys spread over heads first, gradients into one packed tensor."""
    p = Problem(dtype, [90, 41], [90, 41], heads=4, kv_heads=2, causal=True)
    plain = p.both()
    n, size = 131, 64
    packed = torch.full((n, 8 + 3, size), 5.0, dtype=dtype, device=DEV)
    packed[:, :4], packed[:, 4:6], packed[:, 6:8] = p.q, p.k, p.v
    keys_first = p.k.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.full((4, n, size), 5.0, dtype=dtype, device=DEV).transpose(0, 1)
    p.q, p.k, p.v = packed[:, :4], keys_first, packed[:, 6:8]
    o, lse = p.forward(out=out)
    grads = torch.full((n, 9, size), 5.0, dtype=dtype, device=DEV)
    p.dout = torch.nn.functional.pad(p.dout, (0, 8))[..., :size]
    p.backward(o, lse, grads[:, :4], grads[:, 4:6], grads[:, 6:8])
    for a, b in zip(plain, (o, lse, grads[:, :4], grads[:, 4:6], grads[:, 6:8])):
        assert torch.equal(a, b)
    assert torch.all(packed[:, 8:] == 5.0) and torch.all(grads[:, 8] == 5.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_key_tensor_for_all_heads(dtype):
    """A head stride of 0: inputs expanded over heads."""
    p = Problem(dtype, [40], [40], heads=2, kv_heads=2)
    p.k = p.k[:, :1].expand(-1, 2, -1)
    near(p.forward()[0], p.reference(False)[0], BOUNDS[dtype][0], "out")


def test_faulty_sequences_are_left_out():
    p = Problem(torch.float32, [10, 20, 30], [10, 20, 30])
    good, _ = p.forward()
    p.max_q = p.max_k = 25
    out, lse = p.forward()
    assert torch.equal(out[:30], good[:30]) and torch.all(out[30:] == 7.0)
    assert ps.ps_status_read(p.status) == (ps.PS_ST_BAD_LENGTH, 2)
    p = Problem(torch.bfloat16, [10, 20, 30], [10, 20, 30])
    good, lse = p.forward()
    p.ko[1] = 1 << 20
    out, _ = p.forward()
    grads = p.backward(good, lse)
    assert torch.all(out[:30] == 7.0) and torch.equal(out[30:], good[30:]) and ps.ps_status_read(p.status) == (ps.PS_ST_BAD_LENGTH, 0)
    assert torch.all(grads[0][:30] == 7.0) and torch.all(grads[1][:30] == 7.0) and torch.all(grads[1][30:] != 7.0)


def test_nothing_to_do():
    for q, k in (([], []), ([0, 0], [0, 0]), ([0], [5])):
        p = Problem(torch.float32, q, k)
        out, lse = p.forward()
        dq, dk, dv = p.backward(out, lse)
        assert torch.all(dk == 0) and torch.all(dv == 0)
    p = Problem(torch.bfloat16, [3], [0])
    out, lse = p.forward()
    assert torch.all(out == 0) and torch.all(lse == -np.inf) and torch.all(p.backward(out, lse)[0] == 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_same_call_gives_the_same_bits(dtype):
    p = Problem(dtype, [1, 300, 77], [2000, 300, 77], causal=True, cap=10.0)
    first = p.both()
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda.current_stream().wait_stream(torch.cuda.default_stream())
        second = p.both()
        torch.cuda.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def test_sequences_do_not_disturb_one_another():
    """Alone or among others, up to how the keys are shared out."""
    p = Problem(torch.float32, [100, 200], [100, 200], causal=True)
    both = p.both()
    p.q, p.k, p.v, p.dout = (t[100:].contiguous() for t in (p.q, p.k, p.v, p.dout))
    p.qo = p.ko = np.array([0, 200])
    alone = p.both()
    for a, b, name in zip(both, alone, ("out", "lse", "dq", "dk", "dv")):
        near(b, (a[:, 100:] if name == "lse" else a[100:]).double().cpu().numpy(), 1e-6, name)


def test_in_a_graph():
    p = Problem(torch.bfloat16, [1, 150], [900, 150], causal=True, q_docs=np.zeros(151, int), k_docs=np.zeros(1050, int))
    args, qo, ko, w = p.arguments(), i32(p.qo), i32(p.ko), p.workspace(True)
    out, lse, grads = torch.empty_like(p.q), torch.empty(4, 151, device=DEV), [torch.empty_like(t) for t in (p.q, p.k, p.v)]

    def step():
        ps.ps_attention_forward(p.q, p.k, p.v, qo, ko, p.max_q, p.max_k, out, lse, w, **args)
        ps.ps_attention_backward(p.q, p.k, p.v, out, lse, p.dout, qo, ko, p.max_q, p.max_k, *grads, w, **args)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        p.q.copy_(torch.randn(p.q.shape, generator=torch.Generator().manual_seed(seed)))
        step()
        want = [t.clone() for t in (out, lse, *grads)]
        for t in (out, lse, *grads):
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (out, lse, *grads)):
            assert torch.equal(a, b)


def test_offsets_past_32_bits():
    """A cache of 4.6 GB: the last keys lie 2^31 elements and more behind the first."""
    n, size = 17_000_000, 64
    k = torch.empty(n, 2, size, dtype=torch.bfloat16, device=DEV)
    tail = 300
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    k[-tail:] = torch.randn(tail, 2, size, generator=g, device=DEV).bfloat16()
    q = torch.randn(2, 2, size, generator=g, device=DEV).bfloat16()
    out, lse = torch.empty_like(q), torch.empty(2, 2, device=DEV)
    # two sequences, the first of no rows and nearly all keys: too long for max_k, so left out
    status = ps.new_status(DEV)
    ps.ps_attention_forward(q, k, k, i32([0, 0, 2]), i32([0, n - tail, n]), 2, tail, out, lse, ps.alloc_workspace(
        ps.ps_attention_workspace_bytes(2, 2, n, 2, tail, 2, 2, size, torch.bfloat16), DEV), causal=True, status=status)
    assert ps.ps_status_read(status) == (ps.PS_ST_BAD_LENGTH, 0)
    c = lambda t: t.float().cpu().numpy()
    ref, _ = ol.attention(c(q), c(k[-tail:]), c(k[-tail:]), [0, 2], [0, tail], causal=True)
    near(out, ref, 5e-3, "out")


GOOD = dict(heads=4, kv_heads=2, size=64)


@pytest.mark.parametrize("change,error", [
    (dict(q=lambda p: p.q.half()), TypeError), (dict(k=lambda p: p.k.float()), TypeError), (dict(q=lambda p: p.q.cpu()), TypeError),
    (dict(v=lambda p: p.v[:-1]), ValueError), (dict(out=lambda p: torch.empty(60, 4, 32, dtype=p.dtype, device=DEV)), ValueError),
    (dict(q=lambda p: p.q.transpose(1, 2).contiguous().transpose(1, 2)), ValueError),
    (dict(lse=lambda p: torch.empty(3, device=DEV)), ValueError), (dict(lse=lambda p: torch.empty(4, 60, device=DEV).double()), TypeError),
    (dict(k_offsets=lambda p: i32([0, 60])), ValueError), (dict(q_docs=lambda p: i32([0] * 60)), ValueError),
    (dict(slopes=lambda p: torch.ones(3, device=DEV)), ValueError), (dict(prefix=lambda p: i32([1])), ValueError),
    (dict(scale=lambda p: 0.0), ps.PsError), (dict(scale=lambda p: float("nan")), ps.PsError), (dict(scale=lambda p: float("inf")), ps.PsError),
    (dict(softcap=lambda p: -1.0), ps.PsError), (dict(max_q=lambda p: -1), ps.PsError),
    (dict(workspace=lambda p: p.workspace(False)[:-1]), ps.PsError), (dict(workspace=lambda p: torch.empty(1 << 20, dtype=torch.uint8, device=DEV)[8:]), ps.PsError),
    (dict(q=lambda p: torch.empty(60 * 256 + 8, dtype=p.dtype, device=DEV)[1:60 * 256 + 1].view(60, 4, 64)), ps.PsError),
    (dict(q=lambda p: torch.empty(60, 4, 68, dtype=p.dtype, device=DEV)[..., :64]), ps.PsError),
    (dict(out=lambda p: torch.empty(60, 1, 64, dtype=p.dtype, device=DEV).expand(-1, 4, -1)), ps.PsError),
])
def test_refusals(change, error):
    p = Problem(torch.bfloat16, [25, 35], [25, 35], **GOOD)
    args = dict(q=p.q, k=p.k, v=p.v, q_offsets=i32(p.qo), k_offsets=i32(p.ko), max_q=35, max_k=35, out=torch.empty_like(p.q),
                lse=torch.empty(4, 60, device=DEV), workspace=p.workspace(False))
    ps.ps_attention_forward(**args)
    args.update({n: f(p) for n, f in change.items()})
    with pytest.raises(error):
        ps.ps_attention_forward(**args)


def test_sizes_that_are_not_built():
    for size in (4, 12, 136, 256):
        assert ps.ps_attention_workspace_bytes(1, 10, 10, 10, 10, 1, 1, size, torch.bfloat16) == 0
    assert ps.ps_attention_workspace_bytes(1, 10, 10, 10, 10, 3, 2, 64, torch.bfloat16) == 0
    assert ps.ps_attention_workspace_bytes(1, 10, 10, 1 << 22, 10, 64, 1, 64, torch.bfloat16) == 0
    p = Problem(torch.float32, [4], [4], size=64)
    q = torch.empty(4, 4, 136, device=DEV)
    k = torch.empty(4, 2, 136, device=DEV)
    with pytest.raises(ps.PsError) as e:
        ps.ps_attention_forward(q, k, k, i32(p.qo), i32(p.ko), 4, 4, torch.empty_like(q), None, p.workspace(False))
    assert e.value.code == -6


def test_both_ways_through_the_binding(monkeypatch):
    p = Problem(torch.bfloat16, [30, 1], [30, 400], causal=True, cap=5.0, slopes=SLOPES, prefix=[3, 4])
    ps.load_library()
    assert ps._native is not None
    made = []
    real = ps._made
    monkeypatch.setattr(ps, "_made", lambda name, *a: made.append(real(name, *a)) or made[-1])
    one = p.both()
    assert made == [True, True]
    monkeypatch.setattr(ps, "_made", lambda name, *a: False)
    for a, b in zip(one, p.both()):
        assert torch.equal(a, b)
