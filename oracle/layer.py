"""64-bit definitions of the operators of a layer that is fine-tuned or takes long prompts: attention with capped scores, distance
bias, document and prefix masks, and its gradients; rotary positions; dropout from a counter-based generator.  Plain numpy, a
sequence and a head at a time."""
from __future__ import annotations

import numpy as np


def visible(nq, nk, start, causal=False, prefix=0, q_docs=None, k_docs=None):
    """[nq, nk] truth: which keys row i, at position start + i, sees."""
    place, key = start + np.arange(nq)[:, None], np.arange(nk)[None]
    seen = np.ones((nq, nk), bool)
    if causal:
        seen = (key <= place) | (key < prefix)
    if q_docs is not None:
        seen &= (q_docs[:, None] == k_docs[None]) & (q_docs[:, None] >= 0)
    return seen


def attend(q, k, v, seen, start, scale, cap=0.0, slope=0.0, dout=None):
    """One head of one sequence: (out, lse) and, with dout, (dq, dk, dv).  Only what is seen is ever touched."""
    nq, nk = seen.shape
    out, lse = np.zeros((nq, v.shape[1])), np.full(nq, -np.inf)
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for i in range(nq):
        j = np.flatnonzero(seen[i])
        if j.size == 0:
            continue
        x = scale * (k[j] @ q[i])
        bent = np.tanh(x / cap) if cap > 0 else None
        y = (cap * bent if cap > 0 else x) - slope * np.abs(start + i - j)
        top = y.max()
        e = np.exp(y - top)
        p = e / e.sum()
        out[i] = p @ v[j]
        lse[i] = top + np.log(e.sum())
        if dout is not None:
            dv[j] += p[:, None] * dout[i]
            g = p * (v[j] @ dout[i] - dout[i] @ out[i])
            if cap > 0:
                g = g * (1 - bent * bent)
            dq[i] = scale * (g @ k[j])
            dk[j] += scale * g[:, None] * q[i]
    return (out, lse) if dout is None else (out, lse, dq, dk, dv)


def attention(q, k, v, q_offsets, k_offsets, k_lengths=None, q_start=None, prefix=None, q_docs=None, k_docs=None, slopes=None,
              causal=False, scale=None, cap=0.0, dout=None):
    """Packed tensors [rows, heads, size]: (out, lse [heads, rows]) and, with dout, (dq, dk, dv).  Rows outside the sequences: NaN."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    heads, kv_heads, scale = q.shape[1], k.shape[1], q.shape[2] ** -0.5 if scale is None else scale
    out, lse = np.full(q.shape, np.nan), np.full((heads, q.shape[0]), np.nan)
    dq, dk, dv = np.full(q.shape, np.nan), np.full(k.shape, np.nan), np.full(v.shape, np.nan)
    for s in range(len(q_offsets) - 1):
        rows = slice(q_offsets[s], q_offsets[s + 1])
        n = k_offsets[s + 1] - k_offsets[s] if k_lengths is None else k_lengths[s]
        keys = slice(k_offsets[s], k_offsets[s] + n)
        nq = rows.stop - rows.start
        start = n - nq if q_start is None else q_start[s]
        seen = visible(nq, n, start, causal, 0 if prefix is None else prefix[s], None if q_docs is None else q_docs[rows],
                       None if k_docs is None else k_docs[keys])
        dk[keys], dv[keys] = 0.0, 0.0
        for h in range(heads):
            c = h * kv_heads // heads
            got = attend(q[rows, h], k[keys, c], v[keys, c], seen, start, scale, cap, 0.0 if slopes is None else float(slopes[h]),
                         None if dout is None else np.asarray(dout, np.float64)[rows, h])
            out[rows, h], lse[h, rows] = got[:2]
            if dout is not None:
                dq[rows, h] = got[2]
                dk[keys, c] += got[3]
                dv[keys, c] += got[4]
    return (out, lse) if dout is None else (out, lse, dq, dk, dv)


def rotate(x, positions, frequencies, interleaved=False, magnitude=1.0, inverse=False):
    """x [rows, heads, size]; frequencies [pairs]."""
    x = np.array(x, np.float64)
    n = len(frequencies)
    first = np.arange(n) * 2 if interleaved else np.arange(n)
    second = first + 1 if interleaved else first + n
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(frequencies, np.float64)[None]
    turn = magnitude * np.exp((-1j if inverse else 1j) * angle)[:, None]
    y = (x[..., first] + 1j * x[..., second]) * turn
    x[..., first], x[..., second] = y.real, y.imag
    return x


def philox(counter, key):
    """Philox4x32-10 (Salmon et al. 2011): four words of 32 bits from arrays (or numbers) of four and two."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(rows, cols, seed, offset, p):
    """([rows, cols] truth, the factor of what is kept)."""
    lost = int(np.rint(np.float32(p) * 65536))
    groups = (cols + 7) // 8
    r, g = np.meshgrid(np.arange(rows), np.arange(groups), indexing="ij")
    zero = np.zeros_like(r)
    seed, offset = seed & (2 ** 64 - 1), offset & (2 ** 64 - 1)
    words = philox((g, r, zero + (offset & 0xFFFFFFFF), zero + (offset >> 32)), (seed & 0xFFFFFFFF, seed >> 32))
    pieces = np.stack([half for w in words for half in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1)
    return pieces.reshape(rows, groups * 8)[:, :cols] >= lost, 65536 / (65536 - lost) if lost < 65536 else 0.0


def dropout(x, bias, residual, seed, offset, p):
    x = np.asarray(x, np.float64)
    keep, by = kept(*x.shape, seed, offset, p)
    y = np.where(keep, (x if bias is None else x + np.asarray(bias, np.float64)) * by, 0.0)
    return y if residual is None else y + np.asarray(residual, np.float64)


def dropout_gradients(dout, seed, offset, p):
    dout = np.asarray(dout, np.float64)
    keep, by = kept(*dout.shape, seed, offset, p)
    dx = np.where(keep, dout * by, 0.0)
    return dx, dx.sum(0)
