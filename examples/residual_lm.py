"""A language model of residual feed-forward blocks, built from the library's operators alone and trained by its optimizer step.

    emb  = table[ids]                                                       Embedding.lookup
    y, h = 0 + emb, pre_0(y)                                                Join.join
    for every block:  f = gelu(h w1^T + b1) w2^T                            Linear.product, twice
                      y, h = y + gate * post(f), pre(y)                     Join.join
    logp = log softmax(h table^T)[next token]                               Linear.product, LogProbs.logprobs

and back through the same operators' gradients, the table's from both of its ends.  Parameters are fp32 blocks of a handle; the
products read bf16 copies of the matrices, activations are bf16 on an fp32 residual stream.  Gradients are written into the
blocks' bf16 arrays, clipped by their global norm and handed to the sampling window, then to the optimizer step.

    python examples/residual_lm.py [--steps 60]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_04711_b200 import binding as B, harness as H, workloads as W  # noqa: E402

VOCAB, DIM, FF, LAYERS, BATCH, LENGTH, PAD = 512, 128, 320, 2, 16, 65, 0
BF = torch.bfloat16


def blocks():
    """Names and shapes of the parameter blocks."""
    out = [("table", (VOCAB, DIM)), ("pre.0", (DIM,))]
    for i in range(LAYERS):
        out += [(f"w1.{i}", (FF, DIM)), (f"b1.{i}", (FF,)), (f"w2.{i}", (DIM, FF)), (f"post.{i}", (DIM,)), (f"gate.{i}", (DIM,)), (f"pre.{i + 1}", (DIM,))]
    return out


class Model:
    def __init__(self):
        self.embed, self.join, self.answer = B.Embedding(VOCAB, DIM, scale=DIM ** 0.5, pad_id=PAD), B.Join(DIM), B.LogProbs(VOCAB)
        self.up, self.down, self.head = B.Linear(DIM, FF, act="gelu"), B.Linear(FF, DIM), B.Linear(DIM, VOCAB)

    def loss_and_gradients(self, p, g, ids, follow):
        """The mean loss of the positions whose next token `follow` is not -1.  p: fp32 parameters by name; g: bf16 gradients by
        name, written."""
        n, count = ids.numel(), (follow >= 0).sum()
        half = {k: v.to(BF) for k, v in p.items() if v.dim() == 2}
        emb = self.embed.lookup(half["table"], ids)
        y, h = self.join.join(None, emb, p["pre.0"])
        kept = []
        for i in range(LAYERS):
            pre = torch.empty((n, FF), dtype=BF, device=ids.device)
            a = self.up.product(h, half[f"w1.{i}"], bias=p[f"b1.{i}"], pre=pre)
            f = self.down.product(a, half[f"w2.{i}"])
            kept.append((h, pre, a, f))
            y, h = self.join.join(y, f, p[f"pre.{i + 1}"], post_w=p[f"post.{i}"], gate=p[f"gate.{i}"])
            kept[-1] += (y,)
        logits = self.head.product(h, half["table"])
        out = self.answer.logprobs(logits, follow)
        loss = -out.logp.sum() / count

        dlogits = self.answer.grad(logits, follow, out.stats, torch.where(follow >= 0, -1.0 / count, 0.0), dlogits=logits)
        dh, dy = torch.empty_like(h), None
        self.head.grad(h, half["table"], dlogits, dx=dh, dw=g["table"])
        for i in reversed(range(LAYERS)):
            h, pre, a, f, y = kept[i]
            dy, df = self.join.grad(y, f, dh, p[f"pre.{i + 1}"], dy=dy, post_w=p[f"post.{i}"], gate=p[f"gate.{i}"], dx=dy, df=dh,
                                    dpre_w=g[f"pre.{i + 1}"], dpost_w=g[f"post.{i}"], dgate=g[f"gate.{i}"])
            da = torch.empty_like(a)
            self.down.grad(a, half[f"w2.{i}"], df, dx=da, dw=g[f"w2.{i}"])
            dh = torch.empty_like(h)
            self.up.grad(h, half[f"w1.{i}"], da, pre=pre, dx=dh, dw=g[f"w1.{i}"], db=g[f"b1.{i}"])
        _, demb = self.join.grad(emb.float(), None, dh, p["pre.0"], dy=dy, want_dx=False, dpre_w=g["pre.0"])
        self.embed.grad(ids, demb, g["table"], accumulate=True)            # on top of the head's share
        return loss


def sequences(gen: torch.Generator) -> torch.Tensor:
    """Sequences in which token t is followed by 3 t + 1 most of the time; each is padded from a random length on."""
    ids = torch.randint(1, VOCAB, (BATCH, LENGTH), generator=gen)
    keep = torch.rand((BATCH, LENGTH), generator=gen) < 0.9
    for t in range(1, LENGTH):
        ids[:, t] = torch.where(keep[:, t], (3 * ids[:, t - 1] + 1) % (VOCAB - 1) + 1, ids[:, t])
    lengths = torch.randint(LENGTH // 2, LENGTH + 1, (BATCH, 1), generator=gen)
    return torch.where(torch.arange(LENGTH) < lengths, ids, PAD).to("cuda:0")


def initialise(p, gen: torch.Generator):
    for name, v in p.items():
        if v.dim() == 2:
            v.copy_(torch.randn(v.shape, generator=gen) * v.shape[1] ** -0.5)
        else:
            v.fill_(0.0 if name.startswith("b1") else 1.0)


def train(steps: int = 60, window: int = 8, max_norm: float = 1.0, seed: int = 0):
    """Returns (losses, global gradient norms before the clip), one of each per step after the window."""
    shapes = blocks()
    wl = W.Workload("residual_lm", [W.Block(name, s[0], s[1] if len(s) == 2 else 1) for name, s in shapes], window=window, mem_budget_frac=0.7,
                    time_budget=1.3, seed=seed)
    sess = H.Session(wl, [B.make_config(1, 1, 1, 0, bits, lr=3e-3, weight_decay=0.0) for bits in (32, 16)], n_grad_sets=1)
    named = lambda views: {name: v.view(s) for (name, s), v in zip(shapes, views)}
    p, g, model, gen = named(sess.param_views), named(sess.grad_views[0]), Model(), torch.Generator().manual_seed(seed)
    initialise(p, gen)
    losses, norms = [], []
    for t in range(1 - window, steps + 1):
        ids = sequences(gen)
        inputs, targets = ids[:, :-1].reshape(-1), ids[:, 1:].reshape(-1)
        loss = model.loss_and_gradients(p, g, inputs, torch.where((inputs != PAD) & (targets != PAD), targets, -1))
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
