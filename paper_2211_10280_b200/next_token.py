"""A small next-token model trained on from streamed word embeddings: the language-model operators used together.

    python -m paper_2211_10280_b200.next_token [--steps 200] [--state-bits 8] [--dense]

1. A stream of token batches trains the SGNS tables (`binding.Context`), as a streaming job does.
2. Their input rows become the embedding table of a next-token model: scaled lookup of a window of tokens, mean over the
   window, two linear layers, softmax over the vocabulary.
3. Each step looks rows up (`Embedding.lookup`), takes gradients, clips them by their global norm on the device, and
   updates the layers with `AdamW` (one launch for all of them) and the table with `Embedding.adamw`, which reads the
   batch's gradient rows and touches only the rows of its tokens; the table's share of the norm is that of its touched rows
   (`Embedding.gradient_rows`, the form that a message has).  With --dense the table's whole gradient is made
   (autograd through `Embedding.__call__`) and the table is one more tensor of the AdamW step.
Nothing in a step waits for the device; the loss is read every `report` steps.
"""
from __future__ import annotations

import argparse
import math

import numpy as np
import torch

from . import binding, operators


def token_stream(V: int, length: int, seed: int) -> np.ndarray:
    """Tokens that follow their predecessor by a fixed table seven times in ten and are Zipf draws otherwise."""
    r = np.random.default_rng(seed)
    follows = np.random.default_rng(0).permutation(V)
    drawn = np.minimum(np.exp(r.random(length) * math.log(V + 1)) - 1, V - 1).astype(np.int64)
    use = r.random(length) < 0.7
    out = drawn.copy()
    for i in range(1, length):
        if use[i]:
            out[i] = follows[out[i - 1]]
    return out


def streamed_table(V: int, d: int, batches: int = 20, batch: int = 2048) -> torch.Tensor:
    """Input rows of an SGNS model trained on `batches` mini-batches of the stream."""
    ctx = binding.Context(V=V, d=d, window=5, k=5, batch=batch, reduction=binding.MEAN)
    tokens = token_stream(V, batches * batch, seed=1).astype(np.int32).reshape(batches, batch)
    for t in range(batches):
        ctx.tensair_train_batch_host(0, np.ascontiguousarray(tokens[t]), t)
    table = torch.from_numpy(ctx.tensair_read_embeddings(0, 0)).cuda()
    ctx.close()
    return table


def clip_factor(grads, max_norm: float) -> torch.Tensor:
    """The factor, on the device, that brings the gradients' global norm down to max_norm; not finite where the norm is not (max_norm
    over an infinite norm would be a zero like any other), so that the optimizers leave the step out."""
    norm = torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()
    return torch.where(torch.isfinite(norm), (max_norm / (norm + 1e-6)).clamp(max=1.0), norm)


def rows_slot(most: int, d: int):
    """Room for the touched rows of a batch of up to `most` tokens, as `Embedding.gradient_rows` fills it."""
    return (torch.empty(most, dtype=torch.int32, device="cuda"), torch.zeros(most, d, device="cuda"),
            torch.empty(1, dtype=torch.int32, device="cuda"))


def touched_rows(embedding, grad, ids, slot) -> torch.Tensor:
    """The rows of the table's gradient that are not zero, with zeros behind them: their number stays on the device."""
    _, rows, count = embedding.gradient_rows(grad, ids, out=slot)
    return torch.where(torch.arange(rows.shape[0], device="cuda")[:, None] < count, rows, 0.0)


def train(steps: int = 200, V: int = 5000, d: int = 64, hidden: int = 128, rows: int = 1024, window: int = 4, state_bits: int = 8,
          dense: bool = False, lr: float = 3e-3, max_norm: float = 1.0, report: int = 50, quiet: bool = True):
    """Trains the model; returns the table before and after, the ids that occurred, and the reported losses."""
    table = streamed_table(V, d)
    before = table.clone()
    gen = torch.Generator("cuda").manual_seed(0)
    shapes = [(hidden, d), (hidden,), (V, hidden), (V,)]
    layers = [torch.randn(s, device="cuda", generator=gen).mul_(s[-1] ** -0.5 if len(s) > 1 else 0.0).requires_grad_() for s in shapes]
    copies = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    for c, w in zip(copies, layers):
        c.copy_(w.detach())
    params, decay = [w.detach() for w in layers], [1.0, 0.0, 1.0, 0.0]
    embedding = operators.Embedding(V, d, max_tokens=rows * window, scale=math.sqrt(d))
    m, v, slot = torch.zeros_like(table), torch.zeros_like(table), rows_slot(min(V, rows * window), d)
    if dense:
        params, copies, decay = params + [table], copies + [None], decay + [0.0]
    optimizer = operators.AdamW(params, lr=lr, weight_decay=0.01, state_bits=state_bits, copies=copies, decay_factors=decay)
    stream = torch.from_numpy(token_stream(V, steps * rows + window, seed=2)).cuda()
    losses, seen = [], torch.zeros(V, dtype=torch.bool, device="cuda")
    for step in range(1, steps + 1):
        at = torch.arange(rows, device="cuda") + (step - 1) * rows
        ids = stream[at[:, None] + torch.arange(window, device="cuda")]          # [rows, window]
        target = stream[at + window]
        seen[ids] = True
        if dense:
            table.requires_grad_()
            x = embedding(table, ids)
        else:
            x = embedding.lookup(table, ids).requires_grad_()
        w = [c.detach().requires_grad_() for c in copies[:4]]                     # the forward pass runs in 16 bits
        h = torch.nn.functional.gelu(x[:, -1].bfloat16() @ w[0].t() + x.mean(1).bfloat16() @ w[0].t() + w[1])
        loss = torch.nn.functional.cross_entropy((h @ w[2].t() + w[3]).float(), target)
        grads = list(torch.autograd.grad(loss, w + [table if dense else x]))
        table.requires_grad_(False)
        clip = clip_factor(grads if dense else grads[:4] + [touched_rows(embedding, grads[4], ids, slot)], max_norm)
        optimizer.step(grads if dense else grads[:4], grad_scale=clip)
        if not dense:
            embedding.adamw(grads[4], ids, table, m, v, step=step, lr=lr, weight_decay=0.0, grad_scale=clip)
        if step % report == 0 or step == 1:
            losses.append(loss.item())
            embedding.check()
            if not quiet:
                print(f"step {step:5d}  loss {losses[-1]:.4f}")
    return dict(before=before, after=table, seen=seen, losses=losses, optimizer=optimizer)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    ap.add_argument("--dense", action="store_true")
    a = ap.parse_args()
    train(a.steps, state_bits=a.state_bits, dense=a.dense, quiet=False)


if __name__ == "__main__":
    main()
