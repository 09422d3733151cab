"""Learns the dense rows of an index from its documents' texts, holds them in 8 bits, and searches with them.

Every term has a row of a table; a text's dense row is the weighted sum of its terms' rows.  A query is a few terms of a
document, and should find that document among all: the loss is the softmax over all documents.  One step:

    docs, x  = embed(table, texts), embed(table, queries)
    loss     = softmax_loss(x, docs, labels)
    gradient = embed_grad of softmax_loss_grad's two gradients, into the one table; embed_grad_weights for the weights of the
               documents' terms

    python examples/learn_rows.py [--docs 4000] [--dim 128] [--steps 60] [--bf16]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2511_00855_amd import binding as B  # noqa: E402
from paper_2511_00855_amd.synth import make_workload  # noqa: E402

DEVICE = torch.device("cuda:0")


def queries_of(docs, rng, count, terms=5):
    """`count` queries of a few terms of a random document each: (indptr, tokens, labels) on the GPU."""
    labels = rng.integers(0, docs.n, count)
    lists = [rng.choice(row, min(terms, len(row)), replace=False) for row in (docs.tx_idx[docs.tx_indptr[d]:docs.tx_indptr[d + 1]] for d in labels)]
    indptr = np.concatenate([[0], np.cumsum([len(t) for t in lists])]).astype(np.int64)
    return tuple(torch.from_numpy(a).to(DEVICE) for a in (indptr, np.concatenate(lists).astype(np.int32), labels.astype(np.int32)))


def learn(docs, dim, steps, batch=512, bf16=False, rate=0.02, temperature=0.5, say=print):
    """Returns (table, the terms' weights in the documents, losses)."""
    rng = np.random.default_rng(0)
    dtype = torch.bfloat16 if bf16 else torch.float32
    indptr, tokens = torch.from_numpy(docs.tx_indptr).to(DEVICE), torch.from_numpy(docs.tx_idx).to(DEVICE)
    # rarer terms weigh more to begin with; both are learned from there on, in f32
    df = torch.bincount(tokens.long(), minlength=docs.tx_vocab).float()
    weights = torch.log1p(docs.n / df)[tokens.long()].mul_(0.05).contiguous()
    master = torch.randn((docs.tx_vocab, dim), device=DEVICE, generator=torch.Generator(DEVICE).manual_seed(0)) * dim ** -0.5
    moments = torch.zeros_like(master), torch.zeros_like(master)
    losses = []
    for step in range(steps):
        q_indptr, q_tokens, labels = queries_of(docs, rng, batch)
        table = master.to(dtype)
        rows = B.embed(table, tokens, weights, indptr)
        x = B.embed(table, q_tokens, None, q_indptr)
        loss, lse = B.softmax_loss(x, rows, labels, scale=1 / temperature)
        mean = torch.full((batch,), 1 / batch, device=DEVICE)
        grad_x, grad_rows = B.softmax_loss_grad(x, rows, labels, lse, mean, scale=1 / temperature)
        grad = B.embed_grad(grad_rows, tokens, docs.tx_vocab, weights, indptr, dtype=torch.float32)
        grad += B.embed_grad(grad_x, q_tokens, docs.tx_vocab, None, q_indptr, dtype=torch.float32)
        weights -= 0.1 * rate * B.embed_grad_weights(grad_rows, table, tokens, indptr)
        # Adam
        moments[0].lerp_(grad, 0.1)
        moments[1].lerp_(grad.square(), 0.01)
        first, second = moments[0] / (1 - 0.9 ** (step + 1)), moments[1] / (1 - 0.99 ** (step + 1))
        master -= rate * first / (second.sqrt() + 1e-8)
        losses.append(float(loss.mean()))
        if step % 10 == 0 or step + 1 == steps:
            say(f"step {step}: loss {losses[-1]:.3f}")
    return master.to(dtype), weights, losses


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--docs", type=int, default=4000)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--bf16", action="store_true")
    a = ap.parse_args(argv)
    w = make_workload("tiny", seed=0, n=a.docs, nq=200, dim=a.dim)
    table, weights, losses = learn(w.docs, a.dim, a.steps, bf16=a.bf16)

    # how often a new query's document is the best of all: with the rows as they are, and in 8 bits
    indptr, tokens = torch.from_numpy(w.docs.tx_indptr).to(DEVICE), torch.from_numpy(w.docs.tx_idx).to(DEVICE)
    rows = B.embed(table, tokens, weights, indptr, out_dtype=torch.float32)
    q_indptr, q_tokens, labels = queries_of(w.docs, np.random.default_rng(1), 200)
    x = B.embed(table, q_tokens, None, q_indptr, out_dtype=torch.float32)
    q, scale = B.quantize_rows(rows)
    exact, eight = (x @ rows.T).argmax(1), B.scores_int8(x, q, scale).argmax(1)
    found, found8 = float((exact == labels).float().mean()), float((eight == labels).float().mean())
    print(f"found first: {found:.3f}, in 8 bits {found8:.3f}; loss {losses[0]:.3f} -> {losses[-1]:.3f}")

    # the learned rows in the index: dense weight alone
    docs, queries = B.DeviceVecs(w.docs, DEVICE), B.DeviceVecs(w.queries, DEVICE)
    docs.dense, queries.dense = rows, x
    ix = B.Index.build(docs, B.build_params(32))
    ids, _ = ix.search_batch(queries, 10, 256, np.tile(np.float32([1, 0, 0]), (200, 1)))
    found_ix = float((ids == exact[:, None]).any(1).float().mean())
    ix.close()
    print(f"the index's ten best hold the exact best: {found_ix:.3f}")
    return dict(losses=losses, found=found, found8=found8, found_ix=found_ix)


if __name__ == "__main__":
    main()
