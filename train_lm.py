#!/usr/bin/env python3
"""A small language model trained with the library's operators on one MI355X.

A token's hidden state is its embedding; each block adds an MLP of the layer-normed state of the token
and of the one before it; the loss is the cross entropy of the next token over the whole vocabulary.
Embedding, layer norm and the loss run in the library's kernels, forward and backward, and their
gradients step two optimizers: Jorge takes the blocks' matrices, AdamW (clipped, with moments in 8
bits unless asked otherwise) the two vocabulary-sized tables, the gains and the biases.

The text is synthetic: a Markov chain over the vocabulary whose next token follows from the last one
nine times in ten, so a model that learns it ends well below log(vocabulary). Prints one JSON line.
"""
import argparse
import json
import math
import os
import sys
import time

ROOT = os.path.dirname(os.path.abspath(__file__))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def build(vocab, width, blocks, seed=0):
    """Parameters of the model: (tables, matrices, vectors), each a dict of fp32 tensors on the GPU."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std):
        return torch.nn.Parameter(torch.randn(shape, generator=gen, device="cuda") * std)
    tables = {"embed": normal((vocab, width), 1.0 / math.sqrt(width)), "head": normal((vocab, width), 0.02)}
    matrices, vectors = {}, {}
    for b in range(blocks):
        matrices[f"{b}.up"] = normal((2 * width, 2 * width), 1.0 / math.sqrt(2 * width))
        matrices[f"{b}.down"] = normal((width, 2 * width), 0.5 / math.sqrt(2 * width))
        for name in (f"{b}", "last") if b == blocks - 1 else (f"{b}",):
            vectors[f"{name}.gain"] = torch.nn.Parameter(torch.ones(width, device="cuda"))
            vectors[f"{name}.bias"] = torch.nn.Parameter(torch.zeros(width, device="cuda"))
    return tables, matrices, vectors


class Operators:
    """The library's operators, as the model calls them."""

    def __init__(self):
        from paper_2310_12298_amd import lm
        self.embedding, self.layer_norm, self.loss = lm.embedding, lm.layer_norm, lm.linear_cross_entropy


def loss_of(ops, tables, matrices, vectors, tokens, targets, dtype):
    """Mean cross entropy of the next tokens. Activations and the tables' working copies are of dtype."""
    import torch
    width = tables["embed"].shape[1]
    h = ops.embedding(tokens, tables["embed"], math.sqrt(width)).to(dtype)
    for b in range(len(matrices) // 2):
        x = ops.layer_norm(h, vectors[f"{b}.gain"], vectors[f"{b}.bias"])
        before = torch.nn.functional.pad(x, (0, 0, 1, 0))[:, :-1]
        u = torch.nn.functional.gelu(torch.cat([x, before], 2) @ matrices[f"{b}.up"].to(dtype).t())
        h = h + u @ matrices[f"{b}.down"].to(dtype).t()
    h = ops.layer_norm(h, vectors["last.gain"], vectors["last.bias"])
    return ops.loss(h, tables["head"].to(dtype), targets)


class Text:
    """Seeded batches of a Markov chain: the next token is (a * token + b) mod vocab nine times in ten, else any."""

    def __init__(self, vocab, seed=0):
        import torch
        self.vocab, self.gen = vocab, torch.Generator(device="cuda").manual_seed(seed + 1)

    def batch(self, rows, length):
        import torch
        tok = torch.empty(rows, length + 1, dtype=torch.int64, device="cuda")
        free = torch.randint(0, self.vocab, tok.shape, generator=self.gen, device="cuda")
        leap = torch.rand(tok.shape, generator=self.gen, device="cuda") < 0.1
        tok[:, 0] = free[:, 0]
        for i in range(1, length + 1):
            tok[:, i] = torch.where(leap[:, i], free[:, i], (tok[:, i - 1] * 31 + 7) % self.vocab)
        targets = tok[:, 1:].contiguous()
        targets[:, 0] = -100                     # nothing is asked of a sequence's first token
        return tok[:, :-1].contiguous(), targets


def train(vocab=8192, width=512, blocks=2, rows=16, length=256, steps=30, lr=3e-3, jorge_lr=0.02, bits=8,
          dtype="bf16", seed=0, say=None):
    """Trains and returns {"losses": one per step, "ms_per_step", ...}."""
    import torch

    from paper_2310_12298_amd.optim import AdamWOptimizer, JorgeOptimizer
    dt = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    tables, matrices, vectors = build(vocab, width, blocks, seed)
    ops, text = Operators(), Text(vocab, seed)
    jorge = JorgeOptimizer(matrices.values(), lr=jorge_lr, beta1=0.9, precond_interval=10)
    adamw = AdamWOptimizer([{"params": list(tables.values())}, {"params": list(vectors.values()), "weight_decay": 0.0}],
                           lr=lr, betas=(0.9, 0.98), max_norm=1.0, bits=bits, seed=seed)
    losses, times = [], []
    for step in range(steps):
        tokens, targets = text.batch(rows, length)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        loss = loss_of(ops, tables, matrices, vectors, tokens, targets, dt)
        loss.backward()
        jorge.step()
        adamw.step()
        for o in (jorge, adamw):
            o.zero_grad()
        losses.append(loss.item())
        times.append((time.perf_counter() - t0) * 1e3)
        if say and (step % 10 == 0 or step == steps - 1):
            say(f"step {step}: loss {losses[-1]:.4f}, {times[-1]:.2f} ms")
    return {"losses": losses, "ms_per_step": sorted(times)[len(times) // 2], "tokens_per_step": rows * length,
            "log_vocab": math.log(vocab)}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--vocab", type=int, default=8192)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--rows", type=int, default=16, help="sequences per step")
    ap.add_argument("--length", type=int, default=256)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32), help="of AdamW's moments")
    ap.add_argument("--dtype", default="bf16", choices=("bf16", "fp32"), help="of the activations")
    a = ap.parse_args()
    out = train(a.vocab, a.width, a.blocks, a.rows, a.length, a.steps, bits=a.bits, dtype=a.dtype,
                say=lambda m: print(m, file=sys.stderr, flush=True))
    print(json.dumps({"metric": "language model training step", "unit": "ms/step", "value": out["ms_per_step"],
                      "data": "synthetic", "first_loss": out["losses"][0], "last_loss": out["losses"][-1],
                      "log_vocab": out["log_vocab"], "config": vars(a)}), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
