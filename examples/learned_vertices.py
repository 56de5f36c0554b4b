"""Vertices with learned rows, taught by a teacher's top logits: the operators for learned inputs and large answers around two GraphSAGE layers.

A training step: sample blocks -> rows of the vertex table by id -> RMS norm -> two layers -> distillation loss and its gradient in one
call -> the layers' backward passes -> the norm's gradients -> SGD, that of the table straight from the sorted ids. Afterwards the whole table is
normalised into 8 bits with a scale a row, and answers are scored from that copy: log probability of each vertex's class, entropy, alternatives.

    python examples/learned_vertices.py [steps]
"""
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2311_13225_amd import binding as b  # noqa: E402

VERTICES, DEGREE, DIM, HIDDEN, CLASSES, TOP = 20_000, 12, 64, 64, 47, 8
SEEDS, FANOUTS = 1024, (8, 5, 1)     # (the last hop is not used: input gradients need a block's transpose, which the bottom hop goes without)
LR, EPS, TEMPERATURE, KEY = 2.0, 1e-5, 2.0, 7


def make_graph(rng):
    """Vertices of one class mostly know each other: (edges, class of every vertex)."""
    label = rng.integers(0, CLASSES, VERTICES)
    by_class = [np.flatnonzero(label == c) for c in range(CLASSES)]
    dst = np.repeat(np.arange(VERTICES), DEGREE)
    src = rng.integers(0, VERTICES, dst.size)
    alike = rng.random(dst.size) < 0.8
    mates = np.concatenate([rng.choice(by_class[c], DEGREE) for c in label])
    return np.where(alike, mates, src).astype(np.int32), dst.astype(np.int32), label


class Layer:
    """One GraphSAGE layer over a sampled block, with everything it keeps for its backward pass."""

    def __init__(self, view, d_in, d_out, relu, gen):
        spread = math.sqrt(2.0 / (d_in + d_out))
        e = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
        self.view, self.relu = view, relu
        self.params = [torch.randn((d_in, d_out), generator=gen, device="cuda") * spread for _ in range(2)] + [torch.zeros(d_out, device="cuda")]
        self.grads = [torch.empty_like(p) for p in self.params]
        self.mean, self.h, self.grad_x = e(view.n_dst_cap, d_in), e(view.n_dst_cap, d_out), e(view.n_src_cap, d_in)
        self.ws = torch.empty(b.no_sage_layer_ws_bytes(view.n_dst_cap, view.n_src_cap, d_in, d_out), dtype=torch.uint8, device="cuda")

    def forward(self, x):
        self.x = x
        b.no_sage_layer_fwd(self.view, x, *self.params, self.relu, self.mean, self.h, self.ws)
        return self.h

    def backward(self, grad_h):
        b.no_sage_layer_bwd(self.view, self.x, self.mean, self.h, grad_h, self.params[0], self.params[1], self.relu, *self.grads, self.grad_x, self.ws)
        return self.grad_x

    def update(self):
        for p, g in zip(self.params, self.grads):
            p.add_(g, alpha=-LR)


def main(steps=150, say=print):
    rng = np.random.default_rng(0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    src, dst, label = make_graph(rng)
    graph = b.no_build_csr(src, dst, VERTICES, 32)
    blocks = b.no_blocks_create(graph, SEEDS, FANOUTS)
    views = [b.no_blocks_view(blocks, hop) for hop in (0, 1)]
    # the rows that a block needs: their ids and number stay on the device
    ids, n_ids = b._view(views[1].d_src_global, (views[1].n_src_cap,), "<i4", blocks), b._view(views[1].d_n_src, (1,), "<i4", blocks)
    cap = views[1].n_src_cap

    table, weight = torch.randn((VERTICES, DIM), generator=gen, device="cuda") / math.sqrt(DIM), torch.ones(DIM, device="cuda")
    scale = math.sqrt(DIM)
    lower, upper = Layer(views[1], DIM, HIDDEN, True, gen), Layer(views[0], HIDDEN, CLASSES, False, gen)
    e = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    rows, x, rstd, grad_rows, grad_weight = e(cap, DIM), e(cap, DIM), e(cap), e(cap, DIM), e(DIM)
    grad_z, loss, lse = e(SEEDS, CLASSES), e(SEEDS), e(SEEDS)
    row_weight = torch.full((SEEDS,), 1.0 / SEEDS, device="cuda")
    ws_embed = torch.empty(b.no_embed_ws_bytes(cap, DIM), dtype=torch.uint8, device="cuda")
    ws_norm = torch.empty(b.no_rmsnorm_ws_bytes(cap, DIM), dtype=torch.uint8, device="cuda")
    ws_loss = torch.empty(b.no_distill_ws_bytes(SEEDS, CLASSES), dtype=torch.uint8, device="cuda")
    ws_score = torch.empty(b.no_logprobs_ws_bytes(SEEDS, CLASSES, 3), dtype=torch.uint8, device="cuda")

    # a teacher that knows the classes, but for some noise: its TOP largest logits of every vertex
    teacher = torch.randn((VERTICES, CLASSES), generator=gen, device="cuda")
    labels = torch.from_numpy(label).cuda()
    teacher[torch.arange(VERTICES, device="cuda"), labels] += 6.0
    teacher_logits, teacher_ids = teacher.topk(TOP, dim=1)
    teacher_ids = teacher_ids.to(torch.int32)
    order = torch.from_numpy(rng.permutation(VERTICES).astype(np.int32)).cuda()
    train, held = order[: VERTICES * 3 // 4], order[VERTICES * 3 // 4:]

    first = last = None
    for step in range(steps):
        at = step * SEEDS % (train.numel() - SEEDS)
        seeds = train[at:at + SEEDS].contiguous()
        b.no_sample_blocks(graph, seeds, KEY, step, None, blocks)
        b.no_embed_fwd(table, ids, rows, scale=scale, n_ids=n_ids)
        b.no_rmsnorm_fwd(rows, weight, EPS, x, rstd=rstd, n_rows=n_ids)
        z = upper.forward(lower.forward(x))
        who = seeds.long()
        b.no_distill_fwd_bwd(z[:SEEDS], teacher_ids[who], teacher_logits[who], TEMPERATURE, row_weight, loss, lse, grad_z, ws_loss)
        grad_x = lower.backward(upper.backward(grad_z))
        b.no_rmsnorm_bwd(rows, weight, rstd, grad_x, grad_rows, grad_weight, ws_norm, n_rows=n_ids)
        b.no_embed_bwd(grad_rows, ids, table, ws_embed, scale=-LR * scale, accumulate=True, n_ids=n_ids)
        lower.update()
        upper.update()
        weight.add_(grad_weight, alpha=-LR)
        if step % 50 == 0 or step == steps - 1:
            last = loss.sum().item()
            first = last if first is None else first
            say("step %4d  loss %.4f" % (step, last))

    # answers of held-out vertices, from the fp32 table and from its normalised 8-bit copy
    small, small_scale = torch.empty((VERTICES, DIM), dtype=torch.float8_e4m3fn, device="cuda"), e(VERTICES)
    b.no_rmsnorm_fwd(table * scale, weight, EPS, small, row_scale=small_scale)
    seeds = held[:SEEDS].contiguous()
    b.no_sample_blocks(graph, seeds, KEY, steps, None, blocks)
    tokens = labels[seeds.long()].to(torch.int32)
    found = {}
    for name in ("fp32", "8 bits"):
        if name == "fp32":
            b.no_embed_fwd(table, ids, rows, scale=scale, n_ids=n_ids)
            b.no_rmsnorm_fwd(rows, weight, EPS, x, n_rows=n_ids)
        else:
            b.no_embed_fwd(small, ids, x, row_scale=small_scale, n_ids=n_ids)
        z = upper.forward(lower.forward(x))
        logprob, entropy = e(SEEDS), e(SEEDS)
        top_ids, top_logprobs = torch.empty((SEEDS, 3), dtype=torch.int32, device="cuda"), e(SEEDS, 3)
        b.no_logprobs_fwd(z[:SEEDS], tokens, 1.0, logprob, entropy, lse, ws_score, top_ids=top_ids, top_logprobs=top_logprobs)
        found[name] = dict(logprob=logprob.mean().item(), entropy=entropy.mean().item(), right=(top_ids[:, 0] == tokens).float().mean().item(),
                           among_three=(top_ids == tokens[:, None]).any(1).float().mean().item())
        say("%-6s  log probability of the class %.3f  entropy %.3f  first %.3f  among three %.3f" % ((name,) + tuple(found[name].values())))
    return dict(first=first, last=last, **found)


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 150)
