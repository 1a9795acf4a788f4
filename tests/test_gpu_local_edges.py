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
