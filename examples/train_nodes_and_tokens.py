"""Trains a classifier on two embeddings at once: nodes, whose table is held as tensor-train cores, and the tokens
that describe them, whose table is a plain matrix in bf16.

A step: the nodes' lookup, the tokens' lookups, a linear layer and the cross-entropy over two micro-batches, the gradients
of the token table and of the layer added up in fp32, clipping, and the three updates.

The gradients of the cores exist only inside their update, which forms them from the gradients of the rows that were
looked up.  What is clipped is therefore the norm over the token table's gradient, the layer's, and those row gradients
of all micro-batches.  The cores' gradients are linear in the rows', so the factor scales them alike, but their own norm
is another one.

    python examples/train_nodes_and_tokens.py [steps]
"""
from __future__ import annotations

import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2206_10581_amd import DenseEmbedding, GradientClip, TTEmbedding

N, D, R = (12, 12, 12), (4, 4, 4), (16, 16)   # 1,728 nodes of width 64
NODES, WIDTH = 12 ** 3, 64
TOKENS, DIM = 300, 96
CLASSES, BATCH, MICRO = 10, 512, 2


def train(steps: int = 60, lr: float = 0.5, max_norm: float = 0.5, seed: int = 0):
    """Losses of the steps, and the norms that they were clipped by."""
    g = torch.Generator().manual_seed(seed)
    cores = [(torch.randn(s, generator=g) * 0.5) for s in
             ((N[0], D[0], R[0]), (N[1], R[0], D[1], R[1]), (N[2], R[1], D[2]))]
    nodes = TTEmbedding(N, D, R, BATCH * MICRO, cores, device="cuda:0")
    table = (torch.randn((TOKENS, DIM), generator=g) / math.sqrt(DIM)).cuda()      # fp32, looked up in bf16
    low = table.bfloat16()
    tokens = DenseEmbedding(low, BATCH, scale=math.sqrt(DIM), padding_id=0)
    layer = (torch.randn((WIDTH + DIM, CLASSES), generator=g) * 0.05).cuda()
    # what is to be learned: a class for every node and token, the token's being the one of its number
    node_class = torch.randint(0, CLASSES, (NODES,), generator=g)

    table_grad, layer_grad = torch.empty_like(table), torch.empty_like(layer)
    row_grads = torch.empty((BATCH * MICRO, WIDTH), device="cuda")
    clip = GradientClip([table_grad, layer_grad, row_grads])
    losses, norms = [], []
    for step in range(steps):
        total = 0.0
        node = torch.randint(0, NODES, (BATCH * MICRO,), generator=g)
        rows = nodes.forward(node.cuda())      # of all micro-batches: the cores are updated once, with all of these rows
        for micro in range(MICRO):
            part = slice(micro * BATCH, (micro + 1) * BATCH)
            token = torch.randint(0, TOKENS, (BATCH,), generator=g)
            label = torch.where(token % 2 == 0, token % CLASSES, node_class[node[part]]).cuda()
            token = token.cuda()
            features = torch.empty((BATCH, WIDTH + DIM), device="cuda")
            features[:, :WIDTH] = rows[part]
            tokens.forward(token, out=features[:, WIDTH:])
            logits = features @ layer
            loss = torch.logsumexp(logits, 1) - logits.gather(1, label[:, None])[:, 0]
            total = total + loss.mean() / MICRO
            d_logits = torch.softmax(logits, 1)
            d_logits[torch.arange(BATCH, device="cuda"), label] -= 1.0
            d_logits /= BATCH * MICRO
            d_features = d_logits @ layer.t()
            d_layer = features.t() @ d_logits
            layer_grad.copy_(d_layer) if micro == 0 else layer_grad.add_(d_layer)
            tokens.backward(token, d_features[:, WIDTH:], out=table_grad, add=micro > 0)
            row_grads[part] = d_features[:, :WIDTH]
        norms.append(clip.clip(max_norm))
        layer.add_(layer_grad, alpha=-lr)
        table.add_(table_grad, alpha=-lr)
        low.copy_(table)
        nodes.backward_update(row_grads, lr)
        losses.append(total)
    nodes.close()
    return torch.stack(losses).tolist(), torch.stack(norms).tolist()


if __name__ == "__main__":
    losses, norms = train(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
    for k in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {k:4d}  loss {losses[k]:.4f}  gradient norm {norms[k]:.4f}", flush=True)
    print(f"last       loss {losses[-1]:.4f}  gradient norm {norms[-1]:.4f}")
