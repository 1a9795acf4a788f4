"""ps_local_attention_forward and _backward against their 64-bit definition.

Bounds as of ps_attention_forward and _backward (test_gpu_attention.py): a bias adds to the score what it adds to its size, up to 4 of 30 here.  dbias is
made of fp32 values and sums in calls of both types: a weight is good to 5e-6 (fp32's bound); the row's sum that is taken off has what two bf16 pieces of
out leave, 2^-17, in bf16 calls; both stand against values that cancel, so twice that of the norm of what is added up, which is compared with the norm
of dbias.

Rows that see one key have weight 1 and no gradient of their score: dout . v less the same as dout . out, two sums of head_dim products in other orders,
each off by at most head_dim / 2 roundings of 2^-23 of the sum of their sizes S.  What is left of dq and dk is that times scale and k or q: below
scale head_dim 2^-23 S |k|, for dk once for each head of the group, and of dbias below head_dim 2^-23 S for every row.  The same
holds for dbias where all distances have one bucket: a row's weights sum to one, and its terms to zero."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from paper_2504_03702_amd import binding as ps
from tests.test_gpu_attention import BOUNDS, DEV, LENGTHS, SLOPES, Problem, i32, near

pytestmark = pytest.mark.gpu


class Local(Problem):
    def __init__(self, dtype, q_lens, k_lens, *a, left=-1, right=-1, sinks=0, buckets=None, n_buckets=0, **how):
        super().__init__(dtype, q_lens, k_lens, *a, **how)
        g = torch.Generator(device=DEV)
        g.manual_seed(how.get("seed", 0) + 99)
        self.local = dict(left=left, right=right, sinks=sinks)
        self.buckets = None if buckets is None else np.asarray(buckets)
        self.bias = None if buckets is None else torch.randn(n_buckets, self.q.shape[1], generator=g, device=DEV)

    def more(self):
        return dict(self.local, buckets=i32(self.buckets), bias=self.bias)

    def workspace(self, backward):
        nb = ps.ps_local_attention_workspace_bytes(len(self.qo) - 1, self.q.shape[0], self.k.shape[0], self.max_q, self.max_k, self.q.shape[1],
                                                   self.k.shape[1], self.q.shape[2], self.dtype, backward, **self.local,
                                                   n_buckets=0 if self.bias is None else self.bias.shape[0],
                                                   reach=0 if self.bias is None else len(self.buckets) // 2)
        assert nb > 0
        return torch.full((nb,), 0xFF, dtype=torch.uint8, device=DEV)        # (NaN wherever it is read before it is written)

    def forward(self):
        out, lse = torch.full_like(self.q, 7.0), torch.full((self.q.shape[1], self.q.shape[0]), 7.0, device=DEV)
        self.rest = torch.full(self.q.shape, 0.5, dtype=self.dtype, device=DEV) if self.dtype == torch.bfloat16 else None
        ps.ps_local_attention_forward(self.q, self.k, self.v, i32(self.qo), i32(self.ko), self.max_q, self.max_k, out, lse, self.workspace(False),
                                      out_rest=self.rest, **self.more(), **self.arguments())
        return out, lse

    def backward(self, out, lse):
        dq, dk, dv = (torch.full_like(a, 7.0) for a in (self.q, self.k, self.v))
        dbias = None if self.bias is None else torch.full_like(self.bias, 7.0)
        ps.ps_local_attention_backward(self.q, self.k, self.v, out, lse, self.dout, i32(self.qo), i32(self.ko), self.max_q, self.max_k, dq, dk, dv,
                                       self.workspace(True), dbias=dbias, out_rest=self.rest, **self.more(), **self.arguments())
        return (dq, dk, dv) if dbias is None else (dq, dk, dv, dbias)

    def reference(self, backward=True):
        self.how = dict(self.how, **self.local)
        if self.bias is not None:
            self.how.update(buckets=self.buckets, bias=self.bias.double().cpu().numpy())
        return super().reference(backward)

    def arguments(self):
        own = {n: v for n, v in self.how.items() if n not in ("left", "right", "sinks", "buckets", "bias")}
        keep, self.how = self.how, own
        try:
            return super().arguments()
        finally:
            self.how = keep

    def check(self, backward=True):
        got = self.both() if backward else self.forward()
        assert ps.ps_status_read(self.status) == (0, -1)
        ref = self.reference(backward)
        f, b = BOUNDS[self.dtype]
        bounds = (f, BOUNDS[torch.float32][0], b, b, b, 3e-5 if self.dtype == torch.bfloat16 else 1e-5)
        for name, x, r, bound in zip(("out", "lse", "dq", "dk", "dv", "dbias"), got, ref, bounds):
            # rows that no sequence has are left alone
            keep = np.isnan(r) & (x.float().cpu().numpy() == 7.0)
            r = np.where(keep, 0.0, r)
            x = torch.where(torch.tensor(keep, device=DEV), torch.zeros_like(x, dtype=torch.float32), x.float())
            if name in ("dq", "dk", "dbias") and np.abs(r).max(initial=0.0) < 1e-12:   # (one key a row, or one bucket)
                size, group = self.q.shape[2], self.q.shape[1] // self.k.shape[1]
                sums = float((self.dout.float().abs().amax((0, 1)) * self.v.float().abs().amax((0, 1))).sum())
                by = {"dq": float(self.k.float().abs().max()), "dk": group * float(self.q.float().abs().max()), "dbias": size ** 0.5 * self.q.shape[0]}[name]
                assert float(x.abs().max()) <= size ** 0.5 * 2.0 ** -23 * sums * by, name
                continue
            near(x, r, bound, name)
        return got


BUCKETS = [5, 5, 4, 3, 3, 2, 1, 0, 1, 2, 6, 6, 7, 8, 8]                      # (reach 7)
T5 = ol.buckets(32, 128)
KINDS = {"window": dict(left=20, right=9, sinks=3), "causal": dict(causal=True, left=33, sinks=70), "narrow": dict(left=0, right=0),
         "ahead": dict(left=0, right=40, sinks=1, slopes=SLOPES), "bias": dict(buckets=T5, n_buckets=32),
         "both": dict(causal=True, left=64, sinks=2, buckets=BUCKETS, n_buckets=9, cap=5.0), "gaps": dict(buckets=[1, -1, 0, 9, 2], n_buckets=3, right=50)}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [8, 40, 64, 72, 96, 104, 128])
@pytest.mark.parametrize("kind", list(KINDS))
def test_lengths_and_sizes(dtype, size, kind):
    Local(dtype, LENGTHS, LENGTHS, size=size, **KINDS[kind]).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (5, 1), (6, 2), (12, 4), (32, 1), (7, 1)])
@pytest.mark.parametrize("kind", ["window", "bias", "both"])
def test_shared_heads(dtype, heads, kv_heads, kind):
    Local(dtype, [70, 33, 1, 150], [70, 33, 1, 150], heads, kv_heads, **KINDS[kind]).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("how", [dict(left=100, right=50, sinks=5), dict(causal=True, left=255, sinks=4, buckets=T5, n_buckets=32),
                                 dict(causal=True, left=99, sinks=200, cap=30.0), dict(buckets=T5, n_buckets=32, sinks=9),
                                 dict(left=-1, right=3, sinks=1), dict(left=3, right=-1, sinks=700)],
                         ids=["window", "causal-bias", "many-sinks", "bias", "ends", "begins"])
def test_long_rows(dtype, how):
    """Several blocks of rows and keys, windows that skip tiles, first keys seen from far away; shares, where blocks are few."""
    Local(dtype, [1300], [1300], 2, 1, **how).check()
    Local(dtype, [700, 20, 513], [700, 20, 513], 3, 3, size=72, **how).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_places_and_lengths(dtype):
    """Rows at the end of longer keys, in front of them, behind them; room behind the keys; prefixes inside windows; more rows than keys."""
    for how in (dict(left=30, right=10, sinks=2), dict(causal=True, left=60, sinks=1, buckets=BUCKETS, n_buckets=9), dict(left=5, right=5)):
        Local(dtype, [5, 1, 40], [200, 129, 40], **how).check()
        Local(dtype, [100, 7], [3, 0], **how).check()
        Local(dtype, [0, 3], [9, 5], **how).check()
        Local(dtype, [60, 20, 9], [150, 90, 30], room=[38, 0, 7], q_start=[-20, 80, 2000], **how).check()
        Local(dtype, [60, 20], [150, 90], q_start=[-(1 << 30), 1 << 30], **how).check()
        Local(dtype, [150, 64, 30], [150, 64, 30], prefix=[97, 0, 30], **dict(how, causal=True)).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("order", ["sorted", "shuffled", "padding"])
def test_documents(dtype, order):
    rng = np.random.default_rng(3)
    n = [300, 77, 128]
    docs = np.concatenate([np.sort(rng.integers(0, 5, m)) for m in n])
    if order == "shuffled":
        docs = rng.permutation(docs)
    if order == "padding":
        docs[100:170] = -1
        docs[300:377] = -5                                       # a whole sequence of it
    for how in (dict(left=30, right=40, sinks=20), dict(causal=True, left=90, buckets=T5, n_buckets=32)):
        Local(dtype, n, n, q_docs=docs, k_docs=docs, **how).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("how", [dict(causal=True, left=1023, sinks=4), dict(causal=True, buckets=T5, n_buckets=32, cap=20.0), dict(causal=True, left=70, sinks=40, buckets=T5, n_buckets=32),
                                 dict(left=2, right=0)], ids=["window", "bias", "both", "narrow"])
def test_single_tokens_over_long_keys(dtype, how):
    Local(dtype, [1, 1, 3, 0], [5000, 700, 1, 64], **how).check(backward=False)
    Local(dtype, [1, 2], [2049, 3000], heads=16, kv_heads=1, size=128, **how).check(False)
    Local(dtype, [1, 1], [2049, 40], room=[63, 5], q_start=[1000, 45], heads=4, kv_heads=4, size=72, **how).check(False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_without_any_of_it_as_ps_attention(dtype):
    """The same sums in the same order: equal to the bit."""
    for how in (dict(), dict(causal=True, cap=5.0, slopes=SLOPES)):
        p, q = Local(dtype, [130, 9, 300], [130, 9, 300], **how), Problem(dtype, [130, 9, 300], [130, 9, 300], **how)
        assert all(torch.equal(a, b) for a, b in zip(p.both(), q.both()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_faulty_sequences(dtype):
    """Left out of everything, the bias's gradient too."""
    p = Local(dtype, [40, 30, 20], [40, 30, 20], left=9, right=9, buckets=T5, n_buckets=32)
    whole = p.both()
    p.max_q = 35
    p.status = ps.new_status(DEV)
    got = p.both()
    assert ps.ps_status_read(p.status) == (ps.PS_ST_BAD_LENGTH, 0)
    assert torch.all(got[0][:40] == 7.0) and torch.all(got[2][:40] == 7.0)
    for x, y in zip(got[:1] + got[2:5], whole[:1] + whole[2:5]):
        assert torch.equal(x[40:], y[40:])
    q = Local(dtype, [30, 20], [30, 20], left=9, right=9, buckets=T5, n_buckets=32)
    q.q, q.k, q.v, q.dout = (t[40:].contiguous() for t in (p.q, p.k, p.v, p.dout))
    q.bias = p.bias
    assert torch.allclose(q.both()[5], got[5], rtol=1e-4, atol=1e-5)
    none = Local(dtype, [], [], buckets=T5, n_buckets=32)
    assert torch.equal(none.backward(*none.forward())[3], torch.zeros_like(none.bias))


def many(seed, n, longest):
    """Lengths of n sequences: none, one, the longest and others in no order."""
    r = np.random.RandomState(seed)
    lens = [int(x) for x in r.randint(1, 1 + longest // 4, n)]
    for i, m in zip(r.permutation(n)[:7], (0, 0, 1, longest, longest, longest - 1, longest // 2)):
        lens[i] = m
    return lens


# More blocks than units: of 64 sequences and fewer workgroups add up what there is, the longest first without a window; of more they count as the grid does.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,longest", [(64, 300), (33, 300), (67, 200)])
@pytest.mark.parametrize("how", [dict(buckets=T5, n_buckets=32), dict(causal=True, left=30, sinks=3, buckets=BUCKETS, n_buckets=9), dict(causal=True, left=1000)], ids=["bias", "both", "causal"])
def test_many_sequences(dtype, n, longest, how):
    lens = many(n, n, longest)
    Local(dtype, lens, lens, 4, 4, 64, **how).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("how", [dict(buckets=T5, n_buckets=32), dict(left=30, right=20, sinks=3)], ids=["bias", "window"])
def test_faulty_ones_among_many(dtype, how):
    lens = many(5, 64, 300)
    p = Local(dtype, lens, lens, 4, 4, 64, **how)
    whole = p.both()
    p.max_q, p.status = 298, ps.new_status(DEV)
    got = p.both()
    bad = [s for s in range(64) if lens[s] > 298]
    code, which = ps.ps_status_read(p.status)
    assert len(bad) == 3 and code == ps.PS_ST_BAD_LENGTH and which in bad
    # (their shares may be others, for other bounds: fp32 sums in another order, rounded once)
    for i in (0, 2, 3, 4):
        for s in range(64):
            x, y = (t[i][p.qo[s]:p.qo[s + 1]].float() for t in (got, whole))
            assert torch.all(x == 7.0) if s in bad else torch.allclose(x, y, rtol=2.0 ** -7, atol=1e-5), (i, s)


# Biases that hide a bucket's pairs: near ones and those of all that is further behind than reach, in tiles of one bias and of many.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lowest", [float("-inf"), torch.finfo(torch.float32).min])
@pytest.mark.parametrize("how", [dict(), dict(causal=True, cap=20.0), dict(left=200, right=150, sinks=3)], ids=["all", "cap", "window"])
def test_a_bias_that_hides(dtype, lowest, how):
    p = Local(dtype, [300, 7, 1], [300, 260, 260], 4, 2, 64, buckets=ol.buckets(32, 32), n_buckets=32, **how)
    p.bias[3], p.bias[15], p.bias[17, 1], p.bias[31] = lowest, lowest, lowest, lowest
    got = p.check()
    assert not got[-1][3].any() and not got[-1][15].any()
    p.bias[:] = lowest                                                       # nothing is left
    out, lse, *grads = p.both()
    assert not out.any() and (lse == -np.inf).all() and not any(g.any() for g in grads)


# Calls whose bounds say that no sequence has a key, or a row.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_bounds_of_zero(dtype):
    p = Local(dtype, [700, 0, 40], [0, 0, 0], 4, 2, 64, left=3, right=2, sinks=5, buckets=BUCKETS, n_buckets=9)
    p.max_k = 0
    out, lse, dq, dk, dv, dbias = p.both()
    assert not out.any() and (lse == -np.inf).all() and not dq.any() and not dbias.any()
    p = Local(dtype, [0, 0], [700, 40], 4, 2, 64, left=3, right=2, sinks=5, buckets=BUCKETS, n_buckets=9)
    p.max_q = 0
    out, lse, dq, dk, dv, dbias = p.both()
    assert not dk.any() and not dv.any() and not dbias.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_same_bits_every_time(dtype):
    p = Local(dtype, [900, 333], [900, 333], 8, 2, left=200, right=100, sinks=4, buckets=T5, n_buckets=32)
    first = p.both()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, p.both()))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), torch.finfo(torch.bfloat16).min])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_what_nobody_sees_does_not_matter(dtype, bad):
    """Room behind a cache's keys and tiles outside of the windows hold anything."""
    p = Local(dtype, [5, 70, 1], [90, 70, 400], room=[38, 1, 70], causal=True, left=60, sinks=2, buckets=T5, n_buckets=32)
    clean = p.both()
    for s in range(3):
        p.k[p.ko[s] + p.k_lengths[s]:p.ko[s + 1]] = bad
        p.v[p.ko[s] + p.k_lengths[s]:p.ko[s + 1]] = bad
    got = p.both()
    assert all(torch.equal(a, b) for a, b in zip(clean, got))


def test_a_graph_is_played_again():
    p = Local(torch.bfloat16, [600, 33], [600, 33], 4, 2, left=100, right=60, sinks=4, buckets=T5, n_buckets=32)
    q_offsets, k_offsets, args, more = i32(p.qo), i32(p.ko), p.arguments(), p.more()
    out, lse, rest = torch.empty_like(p.q), torch.empty(4, p.q.shape[0], device=DEV), torch.empty_like(p.q)
    grads, ws = [torch.empty_like(t) for t in (p.q, p.k, p.v, p.bias)], p.workspace(True)

    def call():
        ps.ps_local_attention_forward(p.q, p.k, p.v, q_offsets, k_offsets, p.max_q, p.max_k, out, lse, ws, out_rest=rest, **more, **args)
        ps.ps_local_attention_backward(p.q, p.k, p.v, out, lse, p.dout, q_offsets, k_offsets, p.max_q, p.max_k, *grads[:3], ws, dbias=grads[3], out_rest=rest,
                                       **more, **args)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        for t in (p.q, p.k, p.v, p.dout, p.bias):
            t.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, lse, *grads)]
        for t in (out, lse, *grads):
            t.zero_()
        call()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, *grads)))
