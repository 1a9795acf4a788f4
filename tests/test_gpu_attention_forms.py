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


class Large(Problem):
    """With its definition in 64 bits taken a head at a time on the GPU: sequences too long for a row at a time."""

    def reference(self, backward=True):
        h = self.how
        group, scale, cap = self.q.shape[1] // self.k.shape[1], self.q.shape[2] ** -0.5, h.get("cap", 0.0)
        nan = lambda *shape: torch.full(shape, float("nan"), dtype=torch.float64, device=DEV)
        out, lse, dq, dk, dv = nan(*self.q.shape), nan(self.q.shape[1], self.q.shape[0]), nan(*self.q.shape), nan(*self.k.shape), nan(*self.k.shape)
        docs = [None if h.get(n) is None else torch.tensor(np.asarray(h[n]), device=DEV) for n in ("q_docs", "k_docs")]
        for s in range(len(self.qo) - 1):
            rows, keys = slice(int(self.qo[s]), int(self.qo[s + 1])), slice(int(self.ko[s]), int(self.ko[s + 1]))
            m, n = rows.stop - rows.start, keys.stop - keys.start
            place, key = torch.arange(n - m, n, device=DEV)[:, None], torch.arange(n, device=DEV)[None]
            seen = torch.ones(m, n, dtype=torch.bool, device=DEV)
            if h.get("causal"):
                seen = (key <= place) | (key < (0 if h.get("prefix") is None else h["prefix"][s]))
            if docs[0] is not None:
                a, b = docs[0][rows][:, None], docs[1][keys][None]
                seen = seen & (a == b) & (a >= 0)
            dk[keys] = dv[keys] = 0.0
            for head in range(self.q.shape[1]):
                c = head // group
                q, k, v, g = (t.double().contiguous() for t in (self.q[rows, head], self.k[keys, c], self.v[keys, c], self.dout[rows, head]))
                x = scale * (q @ k.t().contiguous())
                bent = torch.tanh(x / cap) if cap else None
                y = cap * bent if cap else x
                if h.get("slopes") is not None:
                    y = y - float(np.float32(h["slopes"][head])) * (place - key).abs()
                y = y.masked_fill(~seen, -torch.inf)
                total = y.logsumexp(1) if n else torch.full((m,), -torch.inf, dtype=torch.float64, device=DEV)
                p = torch.where(seen, (y - total[:, None]).exp(), 0.0)
                o = p @ v
                out[rows, head], lse[head, rows] = o, total
                if not backward:
                    continue
                d = p * (g @ v.t().contiguous() - (g * o).sum(1, keepdim=True))
                if cap:
                    d = d * (1 - bent * bent)
                dq[rows, head] = scale * (d @ k)
                dk[keys, c] += scale * (d.t().contiguous() @ q)
                dv[keys, c] += p.t().contiguous() @ g
        return [t.cpu().numpy() for t in ((out, lse, dq, dk, dv) if backward else (out, lse))]

    def shares(self, backward):
        """Whether the call's workspace holds shares of out, or of dk and dv."""
        rows = self.k.numel() * 2 if backward else self.q.numel()
        return self.workspace(backward).numel() >= 2 * 4 * rows


def lengths(n, top, seed=0):
    return np.random.default_rng(seed).integers(1, top + 1, n).tolist()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_reference_of_long_sequences(dtype):
    """It agrees with the definition that goes a row at a time."""
    docs = np.repeat([0, 1, -1, 0], [30, 50, 20, 33])
    p = Large(dtype, [100, 33], [100, 33], causal=True, prefix=[10, 0], cap=5.0, slopes=SLOPES, q_docs=docs, k_docs=docs)
    for a, b in zip(p.reference(), Problem.reference(p)):
        assert np.array_equal(np.isfinite(a), np.isfinite(b)) and np.allclose(a[np.isfinite(a)], b[np.isfinite(b)], rtol=1e-9, atol=1e-9)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shares_of_many_single_rows(dtype):
    """More than 4096 rows in shares, of which most have one: a long cache among 600 short ones."""
    k = [2500, *lengths(599, 40)]
    p = Large(dtype, [1] * 600, k, heads=8, kv_heads=8, causal=True, slopes=[0.5 / (h + 1) for h in range(8)])
    assert p.shares(False)
    p.check(backward=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [64, 96, 128])
@pytest.mark.parametrize("lens", [[700], [90, 700, 3]], ids=str)
def test_shares_of_many_rows(dtype, size, lens):
    """More than 4096 rows of several shares each, and the gradients' shares."""
    p = Large(dtype, lens, lens, heads=8, kv_heads=8, size=size, causal=True, cap=20.0)
    assert p.shares(False) and p.shares(True)
    p.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("how", ["all", "causal", "documents"])
def test_more_than_64_tiles(dtype, how):
    """Tiles are looked through 64 at a time: rows that see more of them, in whole blocks and in shares."""
    n = 4300
    docs = np.repeat(np.arange(6), [700, 1, 1900, 64, 1500, 135])
    masks = dict(all=dict(), causal=dict(causal=True, prefix=[4200]), documents=dict(causal=True, q_docs=docs, k_docs=docs))[how]
    p = Large(dtype, [n], [n], heads=16, kv_heads=16, size=8, **masks)
    assert not p.shares(False) and not p.shares(True)
    p.check()
    if how == "documents":
        docs = np.random.default_rng(1).integers(0, 3, n)
        masks = dict(q_docs=docs, k_docs=docs)
    p = Large(dtype, [n], [n], heads=2, kv_heads=1, size=40, **masks)
    assert p.shares(False) and p.shares(True)
    p.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sequences_that_take_turns(dtype):
    """More than 2048 blocks: some of the sequences at a time."""
    lens = lengths(64, 260)
    Large(dtype, lens, lens, heads=12, kv_heads=12, size=16, causal=True).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_shares_among_many_sequences(dtype):
    """More than 64 sequences, whose shares are counted as the grid counts."""
    lens = [1200, *lengths(69, 20), 0]
    p = Large(dtype, lens, lens, heads=2, kv_heads=1, causal=True)
    assert p.shares(False) and p.shares(True)
    p.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [72, 80, 96])
@pytest.mark.parametrize("causal", [False, True])
def test_single_tokens_with_heads_between_64_and_128(dtype, size, causal):
    """Documents or none, key counts that end inside a tile, and shares."""
    k = [1500, 300, 33, 1]
    docs = np.random.default_rng(2).integers(-1, 3, sum(k))
    Large(dtype, [1, 3, 2, 1], k, size=size, causal=causal, slopes=SLOPES).check(backward=False)
    Large(dtype, [1, 3, 2, 1], k, size=size, causal=causal, q_docs=[0, 1, 2, -1, 0, 1, 2], k_docs=docs).check(backward=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("group", [3, 5, 6, 7])
def test_groups_that_do_not_divide_a_tile(dtype, group):
    docs = np.repeat([0, 1, 2], [150, 80, 131])
    Large(dtype, [300, 61], [300, 61], heads=2 * group, kv_heads=2, causal=True, q_docs=docs, k_docs=docs).check()
    Large(dtype, [300, 61], [300, 61], heads=2 * group, kv_heads=2, size=96, causal=True, cap=10.0).check()
