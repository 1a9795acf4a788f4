"""Local attention where a window, a causal end or documents leave keys that nobody sees among those of a partly read tile, and where rows see few keys at the
far end of a window.  Bounds as in test_gpu_local_attention.py, or equality."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from tests.test_gpu_local_attention import BUCKETS, DEV, T5, Local

pytestmark = pytest.mark.gpu

BIASES = dict(buckets=T5, n_buckets=32)
# Rows at the end of longer keys, in front of them, among keys of other documents: (lengths of rows, of keys, and what they see).
UNSEEN = {"window": ([5, 1, 40], [200, 129, 300], dict(left=30, right=10, sinks=3)),
          "causal": ([60, 20], [150, 90], dict(causal=True, left=45, sinks=1, q_start=[-20, 30])),
          "ahead": ([50, 9], [300, 77], dict(left=20, right=33, q_start=[101, 12])),
          "documents": ([70, 150], [70, 150], dict(left=90, sinks=2, q_docs=[0] * 220, k_docs=[0, 0, 3, 0] * 55))}


def nobody_sees(p):
    """Rows of k and v that none of their sequence's rows sees."""
    found, h = [], p.how
    for s in range(len(p.qo) - 1):
        rows, keys = slice(p.qo[s], p.qo[s + 1]), slice(p.ko[s], p.ko[s + 1])
        m, n = rows.stop - rows.start, keys.stop - keys.start
        docs = (np.asarray(h["q_docs"])[rows], np.asarray(h["k_docs"])[keys]) if "q_docs" in h else (None, None)
        seen = ol.visible(m, n, h["q_start"][s] if "q_start" in h else n - m, h.get("causal", False), 0, *docs, **p.local)
        found += (p.ko[s] + np.flatnonzero(~seen.any(0))).tolist()
    assert len(found) > 40
    return torch.tensor(found, device=DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("kind", list(UNSEEN))
def test_hidden_values_may_be_the_largest(dtype, cap, kind):
    """dout . v of a hidden pair overflows, and adds nothing to the bias's gradient either."""
    q_lens, k_lens, how = UNSEEN[kind]
    for bias in (BIASES, dict(buckets=BUCKETS, n_buckets=9)):
        p = Local(dtype, q_lens, k_lens, cap=cap, **bias, **how)
        clean, gone = p.both(), nobody_sees(p)
        p.v[gone] = torch.finfo(dtype).max * torch.sign(p.v[gone])
        for name, x, y in zip(("out", "lse", "dq", "dk", "dv", "dbias"), p.both(), clean):
            assert torch.equal(x, y), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("kind", ["window", "causal", "ahead"])
@pytest.mark.parametrize("bias", [{}, BIASES], ids=["plain", "bias"])
def test_keys_outside_of_all_windows_may_be_anything(dtype, bad, kind, bias):
    """Forwards: rows of a cache that were never written, or are somebody else's by now, in front of all windows, behind all, in tiles that are read and
    in such that are not."""
    q_lens, k_lens, how = UNSEEN[kind]
    for heads, kv_heads, size in ((4, 2, 64), (3, 3, 80), (16, 4, 128)):
        p = Local(dtype, q_lens, k_lens, heads, kv_heads, size, **bias, **how)
        clean, gone = p.forward(), nobody_sees(p)
        p.k[gone] = p.v[gone] = bad
        assert all(torch.equal(x, y) for x, y in zip(p.forward(), clean)), (heads, size)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("bias", [{}, BIASES], ids=["plain", "bias"])
def test_single_tokens_over_freed_keys(dtype, causal, bias):
    """One token a sequence, or a few: by one workgroup for all keys and by several."""
    for q_lens, k_lens, left in (([1, 1, 3], [5000, 700, 301], 1500), ([1, 1], [129, 4001], 60)):
        for heads, kv_heads, size in ((4, 2, 64), (3, 3, 80), (8, 2, 128)):
            p = Local(dtype, q_lens, k_lens, heads, kv_heads, size, causal=causal, left=left, right=0, sinks=5, **bias)
            clean, gone = p.forward(), nobody_sees(p)
            p.k[gone] = p.v[gone] = float("nan")
            assert all(torch.equal(x, y) for x, y in zip(p.forward(), clean))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,kv_heads", [(2, 1), (4, 4)])
def test_rows_of_far_tiles_are_not_read(dtype, heads, kv_heads):
    """A key's gradients come from the rows in whose windows its block is: others', of tiles further on, may be anything.  (Blocks of 128 keys, tiles of at most 64 tokens: rows
    from 700 on are in no tile of a window of keys in front of 512; blocks of rows in front of 640 have none of them.)"""
    p = Local(dtype, [1300, 40], [1300, 40], heads, kv_heads, left=30, right=20)
    clean = p.both()
    p.q[700:1300] = p.dout[700:1300] = float("nan")
    for name, x, y in zip(("out", "lse", "dq", "dk", "dv"), p.both(), clean):
        if name == "lse":
            x, y = x.t(), y.t()
        n = 512 if name in ("dk", "dv") else 640
        assert torch.equal(x[:n], y[:n]) and torch.equal(x[1300:], y[1300:]), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bias", [{}, BIASES], ids=["plain", "bias"])
def test_keys_of_far_tiles_are_not_read(dtype, bias):
    """Both directions, where keys in front of all windows fill their tiles (keys in front of 256 for rows from 400 on, which see 60)."""
    p = Local(dtype, [40, 5], [440, 5], causal=True, left=60, **bias)
    clean = p.both()
    p.k[:256] = p.v[:256] = float("nan")
    for name, x, y in zip(("out", "lse", "dq", "dk", "dv", "dbias"), p.both(), clean):
        assert torch.equal(x, y), name


@pytest.mark.parametrize("kind", ["window", "bias"])
@pytest.mark.parametrize("size", [64, 128])
def test_a_window_that_ends_at_its_row_is_a_causal_one(kind, size):
    """The same pairs, so the same sums, with what the rounding of d leaves where rows see few keys: equal to the bit.  (All rows see the first key either way.)"""
    for lens in ([700], [1100, 30]):
        how = dict(BIASES if kind == "bias" else {}, sinks=1)
        one, other = (Local(torch.bfloat16, lens, lens, size=size, left=600, **how, **end) for end in (dict(causal=True), dict(right=0)))
        for name, x, y in zip(("out", "lse", "dq", "dk", "dv", "dbias"), one.both(), other.both()):
            assert torch.equal(x, y), name


@pytest.mark.parametrize("size", [64, 128])
@pytest.mark.parametrize("how", [dict(left=600, right=0), dict(left=0, right=600)], ids=["first", "last"])
def test_rows_that_see_few_keys_of_a_long_window(how, size):
    """A row's dq is scale sum d_j k_j, and where keys have much in common (here `far`, besides what they differ by) it stays small because sum d_j is 0: of d's rounding
    it may keep no more than two bf16 pieces leave, 2^-16 of every term.  Besides: D = dout . out from two pieces of out, 2^-16 of S = sum |dout| |out|; weights p from fp32
    scores of size `far` |q| (at most 2^-24 log2(head_dim) + 1 = 8 roundings of that, 2^-17 here), in d twice, by D and by itself.  So an element of
    dq is off by less than scale max |k| sum_j p_j 2^-15 (|dp_j| + |D| + S), and its own rounding 2^-8."""
    far, n, few = 8.0, 1000, 60 if size == 64 else 30                        # (rows whose keys are all in one tile, which their end cuts: of 64 keys, of 32 for heads of 128 under a bias)
    p = Local(torch.bfloat16, [n], [n], 2, 1, size, seed=4, **BIASES, **how)
    p.k += far
    p.bias.zero_()
    out, lse, dq, *_ = p.both()
    scale, k, v = size ** -0.5, p.k[:, 0].double(), p.v[:, 0].double()
    rows = torch.arange(few, device=DEV) if how["left"] else torch.arange(n - few, n, device=DEV)
    apart = torch.arange(n, device=DEV)[None] - rows[:, None]
    seen = (apart >= -how["left"]) & (apart <= how["right"])
    for h in range(2):
        q, do = p.q[rows, h].double(), p.dout[rows, h].double()
        w = (q @ k.t().contiguous() * scale).masked_fill(~seen, -torch.inf).softmax(1)
        o, dp = w @ v, do @ v.t().contiguous()
        big_d = (do * o).sum(1, keepdim=True)
        want = scale * ((w * (dp - big_d)) @ k)
        bound = scale * k.abs().max() * (w * (dp.abs() + big_d.abs() + (do * o).abs().sum(1, keepdim=True))).sum(1, keepdim=True) * 2.0 ** -15 + 2.0 ** -8 * want.abs()
        off = (dq[rows, h].double() - want).abs()
        assert torch.all(off <= bound), float((off / bound).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2), (5, 1), (32, 1)])
@pytest.mark.parametrize("size", [64, 128])
def test_as_many_buckets_as_there_may_be(dtype, heads, kv_heads, size):
    """64, of which a row's lanes share a column, and the most LDS that a call asks for (32 heads to a key head)."""
    Local(dtype, [150, 33, 1], [150, 33, 1], heads, kv_heads, size, buckets=ol.buckets(64, 100), n_buckets=64).check()
    Local(dtype, [260], [260], heads, kv_heads, size, causal=True, left=150, sinks=2, buckets=ol.buckets(64, 90, False), n_buckets=64).check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_buckets", [32, 64])
def test_a_bias_gradient_of_many_blocks(dtype, n_buckets):
    """8 sequences of up to 1100 tokens, 4 heads to a key head, are 280 blocks of 128 rows and more, whose sums are added up in two launches."""
    lens = [1100, 1100, 1099, 1100, 1000, 1100, 1100, 1100]
    p = Local(dtype, lens, lens, 4, 1, 64, causal=True, left=40, buckets=ol.buckets(n_buckets, 128, False), n_buckets=n_buckets)
    # (in 64 bits on the card, a sequence at a time: the same definition as the oracle's)
    got, want = p.both()[5].double(), torch.zeros(n_buckets, 4, dtype=torch.float64, device=DEV)
    buckets = torch.tensor(p.buckets, device=DEV)
    for s, n in enumerate(lens):
        i = slice(p.qo[s], p.qo[s + 1])
        apart = torch.arange(n, device=DEV)[None] - torch.arange(n, device=DEV)[:, None]
        of, seen = buckets[apart.clamp(-128, 128) + 128], (apart <= 0) & (apart >= -40)
        k, v = p.k[i, 0].double().t().contiguous(), p.v[i, 0].double().t().contiguous()
        for h in range(4):
            q, do = p.q[i, h].double(), p.dout[i, h].double()
            w = (q @ k * 0.125 + p.bias[:, h].double()[of]).masked_fill(~seen, -torch.inf).softmax(1)
            dp = do @ v
            want[:, h].index_add_(0, of.flatten(), (w * (dp - (w * dp).sum(1, keepdim=True))).flatten())
    assert float((got - want).norm()) <= (3e-5 if dtype == torch.bfloat16 else 1e-5) * float(want.norm())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", [-1e30, -1e9, -2.0 ** 20])
@pytest.mark.parametrize("how", [dict(), dict(causal=True, cap=20.0), dict(left=200, right=150, sinks=3)], ids=["all", "cap", "window"])
def test_a_large_negative_bias_hides_too(dtype, value, how):
    """As -infinity does, rows that see nothing else included: equal to the bit."""
    p = Local(dtype, [300, 7, 1, 40], [300, 260, 260, 20], 4, 2, 64, buckets=ol.buckets(32, 32), n_buckets=32, **how)
    for gone in ((3, 15, 31), (0, 1), tuple(range(32))):
        p.bias[list(gone)] = -torch.inf
        want = p.both()
        assert all(torch.isfinite(t).all() for t in (want[0], *want[2:])), gone
        p.bias[list(gone)] = value
        assert all(torch.equal(x, y) for x, y in zip(p.both(), want)), gone
