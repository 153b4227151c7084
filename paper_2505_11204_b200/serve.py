"""Several fine-tuned models answering together out of one four-bit superposition.

    python -m paper_2505_11204_b200.serve [--width 1024] [--blocks 6] [--vocab 32128] [--tasks 4] [--tokens 8] [--steps 16]

A stack of square layers and a vocabulary head stands in for a language model.  Its fine-tuned versions are compressed into
one superposition; base and superposition are then packed into four bits.  A batch of sequences, each of its own task, is
decoded token by token: every layer is one call for the whole batch (the base read once, each slot of the superposition
once), the head's logits are scored, the best token goes on.  The same sequences are also decoded with the retrieved fp32
weights, and the log probabilities are compared.  Last, one more task learns: a few steps on its head with the gradient of
the token log probabilities, and the result is added to the superposition.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import randes
from .scoring import token_log_probs


def build(width: int, blocks: int, vocab: int, n_tasks: int, seed: int = 0):
    """(plan, base, models, M): `blocks` layers [width, width] of one shuffled group and a head [vocab, width]."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols = [width] * blocks + [vocab], [width] * (blocks + 1)
    plan = randes.Plan(rows, cols, [0] * blocks + [1], [randes.SHUFFLE | randes.FLIP, randes.FLIP], task_ids=range(n_tasks),
                       seeds=[42 + t for t in range(n_tasks)], max_tasks=n_tasks + 1)
    normal = lambda r, c, s: torch.randn(r, c, generator=gen, device="cuda") * s
    base = [normal(r, c, 1 / math.sqrt(c)) for r, c in zip(rows, cols)]
    deltas = [[normal(r, c, 0.1 / math.sqrt(c)) for r, c in zip(rows, cols)] for _ in range(n_tasks)]
    models = [[w + d for w, d in zip(base, delta)] for delta in deltas]
    return plan, base, models, plan.compress(base, models)


def decode(embed, steps, layers, head, top_k: int, forced=None):
    """Greedy decoding: (tokens [steps, n], their log probabilities).  `layers`: functions h -> h; `head`: h -> logits;
    `forced`: tokens to follow in place of the best ones."""
    n = embed.shape[0]
    h, tokens, logprobs = embed, [], []
    for step in range(steps):
        x = h
        for layer in layers:
            x = x + torch.tanh(layer(x))
        logits = head(x / x.pow(2).mean(1, keepdim=True).sqrt())
        target = forced[step] if forced is not None else None
        scores = randes.token_scores(logits, target, top_k=top_k)
        token = scores.top_ids[:, 0] if forced is None else target
        tokens.append(token)
        logprobs.append(scores.top_logprobs[:, 0] if forced is None else scores.logprob)
        # the next input: a fixed pseudo-embedding of the token, mixed with the state
        angle = token.float()[:, None] * torch.arange(1, embed.shape[1] + 1, device=embed.device).float()[None] * 0.37
        h = 0.5 * x + torch.sin(angle)
    return torch.stack(tokens), torch.stack(logprobs)


def serve(width=1024, blocks=6, vocab=32128, n_tasks=4, n_tokens=8, steps=16, group=64, lam=0.5, seed=0):
    """Decodes with packed and with retrieved weights; returns the tokens and both sets of log probabilities."""
    plan, base, models, M = build(width, blocks, vocab, n_tasks, seed)
    tasks = [b % n_tasks for b in range(n_tokens)]
    packed_base, packed_m = randes.pack(base, group=group), plan.pack_superposition(M, group=group)
    embed = torch.randn(n_tokens, width, generator=torch.Generator(device="cuda").manual_seed(seed + 1), device="cuda")
    apply = lambda l: lambda x: plan.packed_linear(tasks, lam, l, x, packed_base[l], packed_m)
    tokens, packed_lp = decode(embed, steps, [apply(l) for l in range(blocks)], apply(blocks), top_k=4)

    # the same tokens through each task's retrieved weights, in their own type
    full = torch.empty_like(packed_lp)
    for t in range(n_tasks):
        mine = [b for b in range(n_tokens) if tasks[b] == t]
        if mine:
            w = plan.retrieve(t, lam, base, M)
            lin = lambda l: lambda x: x @ w[l].t()
            full[:, mine] = decode(embed[mine], steps, [lin(l) for l in range(blocks)], lin(blocks), 1, forced=tokens[:, mine].contiguous())[1]
    full_bytes = sum(r * c * 4 for r, c in zip(plan.rows, plan.cols))
    packed_bytes = sum(p.nbytes for p in packed_base)
    plan.close()
    return {"tokens": tokens, "packed": packed_lp, "full": full, "bytes": (2 * full_bytes, 2 * packed_bytes)}


def learn(width=256, vocab=4096, rows=64, steps=5, rate=50.0, seed=0):
    """A new task's head learns to name given tokens; returns the mean log probability before and after, by its own weights."""
    plan, base, models, M = build(width, 2, vocab, 2, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 2)
    x = torch.randn(rows, width, generator=gen, device="cuda")
    targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    head = base[-1].clone().requires_grad_(True)
    seen = []
    for _ in range(steps + 1):
        logprob, entropy = token_log_probs(x @ head.t(), targets)
        seen.append(float(logprob.detach().mean()))
        loss = -(logprob + 0.01 * entropy).mean()
        (grad,) = torch.autograd.grad(loss, head)
        with torch.no_grad():
            head -= rate * grad
    before = plan.slot(M, 2).clone()
    plan.add_model(2, 99, base, [base[0], base[1], head.detach()], M)
    changed = not torch.equal(plan.slot(M, 2), before)
    plan.close()
    return seen[0], seen[-1], changed


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("width", 1024), ("blocks", 6), ("vocab", 32128), ("tasks", 4), ("tokens", 8), ("steps", 16), ("group", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    r = serve(a.width, a.blocks, a.vocab, a.tasks, a.tokens, a.steps, a.group)
    off = (r["packed"] - r["full"]).abs()
    print("%d sequences of %d tasks, %d tokens each, from %.1f MiB of packed base and superposition (%.1f MiB in fp32)"
          % (a.tokens, a.tasks, a.steps, r["bytes"][1] / 2**20, r["bytes"][0] / 2**20))
    print("mean log probability of the tokens: packed %.3f, retrieved fp32 weights %.3f; largest difference %.3f"
          % (float(r["packed"].mean()), float(r["full"].mean()), float(off.max())))
    first, last, added = learn()
    print("a new task's head: mean log probability of its tokens %.3f before, %.3f after five steps; added to the superposition: %s"
          % (first, last, "yes" if added else "no"))
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
