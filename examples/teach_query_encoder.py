"""A query encoder taught by a reader, from the retrieval it drives: the operators of hr_scores.h around an IVF index.

    python examples/teach_query_encoder.py [--passages N] [--steps S]

Every step is what a service that learns from its own traffic does: encode a batch of questions, search the index for passages
(IvfIndex.search), let the reader score what came back (here: its own, better view of the question), score the questions
against the whole corpus kept in 8 bits (i8_linear), take the loss against the reader's scores of the retrieved passages and its gradient
in one call (distill_step; places that the search left empty, -1, do not count), and update the encoder.  Before and
after, the scores are read as distributions (logprobs): how likely the right passage is, how sure the encoder is, what else it
would have returned; the questions it is least sure of are searched again with more probes.

Synthetic data: unit vectors around centroids; a question is a passage seen through noise and a rotation that the
encoder, a matrix, has to undo.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_09138_amd as hr  # noqa: E402

SCALE = 20.0                            # of the scores: inverse temperature of student and reader


def unit(x):
    return x / x.norm(dim=1, keepdim=True)


def corpus(passages, d, nlist, g):
    """Passages list by list, their lists, and the index over them; a passage's label is its row."""
    centroids = unit(torch.randn(nlist, d, generator=g, device="cuda"))
    size = passages // nlist
    rows = unit(centroids.repeat_interleave(size, 0) + 0.6 / d ** 0.5 * torch.randn(nlist * size, d, generator=g, device="cuda"))
    offsets = torch.arange(0, nlist * size + 1, size, dtype=torch.int64)
    return hr.IvfIndex(centroids, offsets, rows.half(), torch.arange(nlist * size, device="cuda")), rows


def questions(rows, n, turn, g):
    """(what the encoder sees, what the reader makes of it, the passage it is about)"""
    gold = torch.randint(len(rows), (n, 1), generator=g, device="cuda")
    clean = unit(rows[gold[:, 0]] + 0.3 / rows.shape[1] ** 0.5 * torch.randn(n, rows.shape[1], generator=g, device="cuda"))
    return clean @ turn, clean, gold


def report(name, ix, rows8, scale8, encoder, seen, gold, probes):
    q = unit(seen @ encoder)
    r = hr.logprobs(hr.i8_linear(q, rows8, scale8), gold, k=5, scale=SCALE)
    found = (ix.search(q, probes, 10)[0] == gold).any(1).float()
    unsure = r.entropy.topk(len(q) // 4).indices
    again = (ix.search(q[unsure].contiguous(), min(4 * probes, ix.nlist), 10)[0] == gold[unsure]).any(1).float()
    print(f"{name}: ln p of the right passage {r.logprobs.mean():.3f}, entropy {r.entropy.mean():.3f}, best of all {(r.top_ids[:, :1] == gold).float().mean():.3f}, "
          f"found by the search {found.mean():.3f}; least sure quarter {found[unsure].mean():.3f}, searched again {again.mean():.3f}")
    return float(r.logprobs.mean())


def main(passages=65536, d=256, nlist=256, batch=512, k=32, probes=8, steps=60, rate=200.0, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ix, rows = corpus(passages, d, nlist, g)
    rows8, scale8 = hr.quantize_rows(rows)
    skew = torch.randn(d, d, generator=g, device="cuda")
    turn = torch.matrix_exp(1.35 * (skew - skew.T) / (2 * d) ** 0.5)
    encoder = torch.eye(d, device="cuda")
    test = questions(rows, batch, turn, g)
    before = report("before", ix, rows8, scale8, encoder, test[0], test[2], probes)
    weights = torch.full((batch,), 1.0 / batch, device="cuda")
    losses = []
    for step in range(steps):
        seen, clean, _ = questions(rows, batch, turn, g)
        raw = seen @ encoder
        norm = raw.norm(dim=1, keepdim=True)
        q = raw / norm
        ids, _ = ix.search(q, probes, k)
        reader = (rows[ids.clamp(min=0)] * clean[:, None, :]).sum(2)
        scores = hr.i8_linear(q, rows8, scale8)
        loss, grad = hr.distill_step(scores, ids, reader, weights, scale=SCALE, out=scores)
        dq = grad @ rows
        draw = (dq - q * (dq * q).sum(1, keepdim=True)) / norm
        encoder -= rate / SCALE * (seen.T @ draw)
        losses.append(loss.mean())
        if step % 20 == 0 or step == steps - 1:
            print(f"step {step}: loss {float(losses[-1]):.4f}", flush=True)
    after = report("after", ix, rows8, scale8, encoder, test[0], test[2], probes)
    ix.close()
    return before, after, [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--passages", type=int, default=65536)
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    main(passages=a.passages, steps=a.steps)
