"""A bigram language model trained with the library's operators around its optimizer step.

One token table (fp32 [vocab, dim]) and one output matrix (fp32 [dim, vocab]) are two blocks of a handle.  Every step looks
the tokens up (``Embedding.lookup``), forms the logits and the gradients of the cross entropy with torch products, sums the
table's gradient by token (``Embedding.grad``) into the block's bf16 array, clips all blocks by the global norm
(``Baoc.clip_grads``) and hands them on: to the sampling window first, and after the allocation to the optimizer step.

    python examples/bigram_lm.py [--steps 60]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_04711_b200 import binding as B, harness as H, workloads as W  # noqa: E402

VOCAB, DIM, BATCH, LENGTH, PAD = 512, 128, 16, 65, 0


def sequences(gen: torch.Generator) -> torch.Tensor:
    """Sequences in which token t is followed by 3 t + 1 most of the time; each is padded from a random length on."""
    ids = torch.randint(1, VOCAB, (BATCH, LENGTH), generator=gen)
    keep = torch.rand((BATCH, LENGTH), generator=gen) < 0.9
    for t in range(1, LENGTH):
        follow = (3 * ids[:, t - 1] + 1) % (VOCAB - 1) + 1
        ids[:, t] = torch.where(keep[:, t], follow, ids[:, t])
    lengths = torch.randint(LENGTH // 2, LENGTH + 1, (BATCH, 1), generator=gen)
    return torch.where(torch.arange(LENGTH) < lengths, ids, PAD).to("cuda:0")


def train(steps: int = 60, window: int = 8, max_norm: float = 0.25, seed: int = 0):
    """Returns (losses, global gradient norms before the clip) as lists, one entry per step after the window."""
    wl = W.Workload("bigram_lm", [W.Block("tok_emb", VOCAB, DIM), W.Block("out.w", DIM, VOCAB)], window=window, mem_budget_frac=0.6,
                    time_budget=1.3, seed=seed)
    sess = H.Session(wl, [B.make_config(1, 1, 1, 0, bits, lr=5e-3, weight_decay=0.0) for bits in (32, 16)], n_grad_sets=1)
    sess.init_params()
    table, weight = sess.param_views[0].view(VOCAB, DIM), sess.param_views[1].view(DIM, VOCAB)
    dtable, dweight = sess.grad_views[0][0].view(VOCAB, DIM), sess.grad_views[0][1].view(DIM, VOCAB)
    embed = B.Embedding(VOCAB, DIM, scale=DIM ** 0.5, pad_id=PAD)
    gen = torch.Generator().manual_seed(seed)
    losses, norms = [], []
    for t in range(1 - window, steps + 1):
        ids = sequences(gen)
        inputs, targets = ids[:, :-1], ids[:, 1:]
        kept = ((inputs != PAD) & (targets != PAD)).reshape(-1, 1)
        h = embed.lookup(table, inputs, out_dtype=torch.float32).view(-1, DIM)
        logp = torch.log_softmax(h @ weight, -1)
        count = kept.sum()
        loss = -(logp.gather(1, targets.reshape(-1, 1)) * kept).sum() / count
        dlogits = logp.exp()
        dlogits.scatter_add_(1, targets.reshape(-1, 1), -torch.ones_like(kept, dtype=torch.float32))
        dlogits *= kept / count
        dweight.copy_(h.t() @ dlogits)
        embed.grad(inputs, (dlogits @ weight.t()).view(*inputs.shape, DIM), dtable)
        norm = sess.clip_grads(0, max_norm)[0]
        if t <= 0:
            sess.sample_stats(0)
            if t == 0:                                      # the window is over: risk, allocation, optimizer
                risk, _ = sess.risk()
                assign, _, _ = sess.allocate(risk)
                sess.configure(assign)
        else:
            losses.append(float(loss))
            norms.append(float(norm))
            sess.step(0, t)
    return losses, norms


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    for i, (loss, norm) in enumerate(zip(*train(ap.parse_args().steps))):
        if i % 10 == 9:
            print(f"step {i + 1}: loss {loss:.3f}, gradient norm {norm:.3f}")
