"""Fine-tunes the last layer of a response-length predictor on synthetic prompts longer than a table of learned positions would take,
and scores new prompts with it.

    python examples/finetune_long_prompts.py [--steps N] [--fp32]

Prompts are packed several to a row, as documents that do not see one another, and cut off from the padding at the row's end.  A
layer is: queries, keys and values; rotary positions within the document, for contexts 8 times the trained one; attention with
capped scores; output projection; dropout with bias and residual; and, of every document's first row, the regression head.  Scoring
attends with the first rows alone.  The maps are torch's; rotary positions, attention and dropout, with their gradients, are the
library's."""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2504_03702_amd import binding as ps  # noqa: E402
from paper_2504_03702_amd import layers  # noqa: E402

DEV = "cuda:0"
HIDDEN, HEADS, KV_HEADS, VOCAB, ROW = 256, 4, 2, 512, 1024
SIZE = HIDDEN // HEADS


class Layer(torch.nn.Module):
    def __init__(self, dtype, generator):
        super().__init__()
        made = lambda *s: torch.nn.Parameter((torch.randn(s, generator=generator) * s[0] ** -0.5).to(DEV, dtype))
        self.embed = torch.nn.Parameter(torch.randn(VOCAB, HIDDEN, generator=generator).to(DEV, dtype))
        self.qkv, self.out = made(HIDDEN, (HEADS + 2 * KV_HEADS) * SIZE), made(HIDDEN, HIDDEN)
        self.bias = torch.nn.Parameter(torch.zeros(HIDDEN, device=DEV, dtype=dtype))
        self.head = torch.nn.Parameter(torch.zeros(HIDDEN, device=DEV))
        self.frequencies = ps.ps_rotary_frequencies(SIZE // 2, scaling=ps.PS_ROTARY_PARTS, factor=8.0, trained_len=ROW // 8).to(DEV)

    def forward(self, tokens, positions, firsts, seqs, rng, p, first_rows=None):
        """Length predictions of the documents that start at rows `firsts`; first_rows: the sequences whose queries are those rows alone."""
        x = self.embed[tokens]
        q, k, v = (x @ self.qkv).view(-1, HEADS + 2 * KV_HEADS, SIZE).split((HEADS, KV_HEADS, KV_HEADS), 1)
        q, k = layers.rotary(q, k, positions, self.frequencies)
        if first_rows is not None:
            q, x = q[firsts], x[firsts]
        a = layers.attention(q, k, v, seqs if first_rows is None else first_rows, softcap=30.0)
        y = layers.dropout_add(a.reshape(-1, HIDDEN) @ self.out, self.bias, x, rng, p)
        return (y if first_rows is not None else y[firsts]).float() @ self.head


def draw(rows, generator, status=None):
    """Documents packed into rows of ROW tokens: a log-length is one of four, said by the second token.  Returns what Layer takes, and
    the log-lengths; status: told of faulty sequences."""
    tokens, docs, positions, firsts, lengths, targets = [], [], [], [], [], []
    for r in range(rows):
        at, doc = 0, 0
        while True:
            n = int(torch.randint(16, 200, (), generator=generator))
            if at + n > ROW - 24:
                break
            kind = int(torch.randint(0, 4, (), generator=generator))
            words = torch.randint(8, VOCAB, (n,), generator=generator)
            words[0], words[1] = 0, 1 + kind                    # the row that is scored, and what it has to find
            tokens.append(words)
            docs.append(torch.full((n,), doc))
            positions.append(torch.arange(n))
            firsts.append(r * ROW + at)
            lengths.append(n)
            targets.append(float(kind) - 1.5)
            at, doc = at + n, doc + 1
        tokens.append(torch.zeros(ROW - at, dtype=torch.long))
        docs.append(torch.full((ROW - at,), -1))
        positions.append(torch.zeros(ROW - at, dtype=torch.long))
    i32 = lambda v: (torch.cat(v) if isinstance(v, list) else v).to(DEV, torch.int32)
    offsets = i32(torch.arange(rows + 1) * ROW)
    docs, firsts, lengths = i32(docs), torch.tensor(firsts), torch.tensor(lengths)
    packed = layers.Sequences(offsets, offsets, ROW, ROW, q_docs=docs, k_docs=docs, status=status)
    # for scoring: a sequence a document, its one query in front of its keys; documents lie one after the other, padding behind the last of
    # a row, so that a document's keys are a span with room at its end
    n = len(firsts)
    single = layers.Sequences(i32(torch.arange(n + 1)), i32(torch.cat((firsts, torch.tensor([rows * ROW])))), 1, int(lengths.max()),
                              k_lengths=i32(lengths), q_start=i32(torch.zeros(n)), status=status)
    return torch.cat(tokens).to(DEV), i32(positions), firsts.to(DEV), packed, single, torch.tensor(targets, device=DEV)


def main(steps=60, dtype=torch.bfloat16, rows=8, seed=0):
    """Trains, and returns (first loss, last loss, largest difference between scores by rows and by first rows)."""
    generator = torch.Generator().manual_seed(seed)
    layer = Layer(dtype, generator)
    rng = torch.tensor([seed, 0], dtype=torch.int64, device=DEV)
    optimizer = torch.optim.Adam(layer.parameters(), lr=3e-3)
    losses, status = [], ps.new_status(DEV)
    for step in range(steps):
        tokens, positions, firsts, packed, _, targets = draw(rows, generator, status)
        loss = torch.nn.functional.mse_loss(layer(tokens, positions, firsts, packed, rng, 0.1), targets)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step}: loss {float(losses[-1]):.4f}", flush=True)
    with torch.no_grad():
        tokens, positions, firsts, packed, single, targets = draw(rows, generator, status)
        by_rows = layer(tokens, positions, firsts, packed, rng, 0.0)
        by_firsts = layer(tokens, positions, firsts, packed, rng, 0.0, first_rows=single)
        off = float((by_rows - by_firsts).abs().max())
        print(f"new prompts: loss {float(torch.nn.functional.mse_loss(by_firsts, targets)):.4f}, scored by their first rows alone to {off:.2g}")
    if ps.ps_status_read(status)[0]:
        raise RuntimeError(f"faulty sequences: {ps.ps_status_read(status)}")
    return float(losses[0]), float(losses[-1]), off


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--fp32", action="store_true")
    args = ap.parse_args()
    main(args.steps, torch.float32 if args.fp32 else torch.bfloat16)
