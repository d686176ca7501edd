"""Training step with every node of the graph as a class: a student embedding learns, from the sampled neighborhood of a seed,
which node comes next (softmax cross entropy against all nodes) and what a frozen teacher embedding thinks of them
(distillation from the teacher's best classes).

The neighborhood mean of the student's table (``fused_sample_mean``, a table that learns) goes through one linear layer; its
answer is scored against the same table (``fused_cross_entropy``, ``fused_distillation``), so that the table gets gradients
from both ends.  The [batch, nodes] scores are never kept, in no direction; the teacher's best classes are looked up once per
step over pieces of its table.

With ``--blocks`` the encoder is deeper: the seed's own row joins the neighborhood mean and goes through gated feed-forward blocks
with a norm before each (``fused_residual_norm``, ``fused_gated_feed_forward``), and a last norm before the linear layer.
``--orthogonal`` gives the encoder's matrices orthogonalised momentum (``OrthogonalMomentum``) in place of Adam.

    python -m paper_2511_13645_amd.entity_step --nodes 169343 --batch 1024 --steps 50 --blocks 2 --orthogonal
"""
from __future__ import annotations

import argparse
import json
import statistics
import sys
import time


def teacher_best(answer, table, k, piece=1 << 16):
    """The k best classes of rows `answer` [T,D] and their scores: torch.topk over pieces of the table."""
    import torch
    ids, best = None, None
    for a in range(0, table.shape[0], piece):
        z = answer @ table[a:a + piece].T
        v, i = z.topk(min(k, z.shape[1]), 1)
        best = v if best is None else torch.cat([best, v], 1)
        ids = i + a if ids is None else torch.cat([ids, i + a], 1)
        best, at = best.topk(min(k, best.shape[1]), 1)
        ids = ids.gather(1, at)
    return ids.int().contiguous(), best.contiguous()


def gated_blocks(count, dim, hidden, device, dtype):
    """Parameters of `count` blocks, four each (the norm's weight, then the gated block's three matrices), and the last norm's."""
    import torch
    new = lambda r, c: torch.nn.Parameter(torch.randn((r, c), device=device).mul_(c ** -0.5).to(dtype))
    one = lambda: torch.nn.Parameter(torch.ones(dim, device=device, dtype=dtype))
    return [p for _ in range(count) for p in (one(), new(hidden, dim), new(hidden, dim), new(dim, hidden))] + [one()]


def encode(context, own, blocks):
    """The context and a seed's own row through the blocks: the sum of both, then of that and each block's answer, normed."""
    from .autograd import fused_gated_feed_forward, fused_residual_norm
    for i in range(0, len(blocks) - 1, 4):
        normed, own = fused_residual_norm(context, blocks[i], own)
        context = fused_gated_feed_forward(normed, *blocks[i + 1:i + 4])
    return fused_residual_norm(context, blocks[-1], own)[0]


def main() -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--nodes", type=int, default=169_343)
    ap.add_argument("--degree", type=float, default=13.7)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--dtype", default="f32", choices=["f32", "bf16", "f16"])
    ap.add_argument("--batch", type=int, default=1024)
    ap.add_argument("--fanouts", default="15,10")
    ap.add_argument("--slots", type=int, default=16)
    ap.add_argument("--temperature", type=float, default=2.0)
    ap.add_argument("--weight", type=float, default=0.5, help="of the distillation")
    ap.add_argument("--rate", type=float, default=0.01)
    ap.add_argument("--blocks", type=int, default=0, help="gated feed-forward blocks of the encoder")
    ap.add_argument("--hidden", type=int, default=512, help="of a block")
    ap.add_argument("--orthogonal", action="store_true", help="orthogonalised momentum for the encoder's matrices")
    ap.add_argument("--orthogonal-rate", type=float, default=0.02)
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--warmup", type=int, default=5)
    args = ap.parse_args()

    import torch
    from . import synth
    from .autograd import fused_cross_entropy, fused_distillation, fused_sample_mean
    from .orthogonal import OrthogonalMomentum

    dev = "cuda:0"
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[args.dtype]
    g = synth.chung_lu_graph(args.nodes, args.degree, min(13_000.0, args.nodes / 8), seed=0)
    indptr, indices = g.indptr.to(dev), g.indices.to(dev)
    fan = [int(k) for k in args.fanouts.split(",")]
    gen = torch.Generator(device=dev).manual_seed(0)
    teacher = torch.randn((args.nodes, args.dim), generator=gen, device=dev) * args.dim ** -0.25
    table = torch.nn.Parameter((teacher + torch.randn(teacher.shape, generator=gen, device=dev)).mul_(0.3).to(dtype))
    layer = torch.nn.Linear(args.dim, args.dim, bias=False, device=dev, dtype=dtype)
    blocks = gated_blocks(args.blocks, args.dim, args.hidden, dev, dtype) if args.blocks else []
    encoder = [*layer.parameters(), *blocks]
    matrices = [p for p in encoder if p.dim() == 2] if args.orthogonal else []
    others = [p for p in encoder if not any(p is m for m in matrices)]
    # Adam's squares of gradients below 2^-12 are zero in fp16, as is 1e-8: the step would be an infinity
    opts = [torch.optim.Adam([table, *others], lr=args.rate, eps=1e-4 if args.dtype == "f16" else 1e-8)]
    if matrices:
        opts.append(OrthogonalMomentum(matrices, args.orthogonal_rate))
    n = args.steps + args.warmup
    seeds = synth.seed_batches(args.nodes, args.batch, n, seed=2).to(dev)
    times, losses = [], []
    for i in range(n):
        start = indptr[seeds[i].long()].long()
        degree = indptr[seeds[i].long() + 1].long() - start
        following = indices[(start + degree // 2).clamp(max=indices.shape[0] - 1)]
        targets = torch.where(degree > 0, following, -1).int()         # a seed without neighbors has no target
        with torch.no_grad():
            ids, logits = teacher_best(teacher[seeds[i].long()], teacher, args.slots)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        context, _, _, _ = fused_sample_mean(table, indptr, indices, seeds[i], fan, seed=i)
        if blocks:
            context = encode(context, table[seeds[i].long()], blocks)
        answer = layer(context)
        hard = fused_cross_entropy(answer, table, targets)
        soft = fused_distillation(answer, table, ids, logits, temperature=args.temperature)
        loss = hard.mean() + args.weight * args.temperature ** 2 * soft.mean()
        for opt in opts:
            opt.zero_grad(set_to_none=True)
        loss.backward()
        for opt in opts:
            opt.step()
        torch.cuda.synchronize()
        times.append((time.perf_counter() - t0) * 1e3)
        losses.append(loss.item())
    what = "training step: sampled mean, %slinear layer, cross entropy and distillation against every node, %s" % (
        "%d gated blocks, " % args.blocks if args.blocks else "", "Adam and orthogonalised momentum" if matrices else "Adam")
    print(json.dumps({"what": what,
                      "nodes": args.nodes, "dim": args.dim, "dtype": args.dtype, "batch": args.batch, "slots": args.slots,
                      "median_ms": statistics.median(times[args.warmup:]), "first_loss": losses[0],
                      "last_loss": statistics.mean(losses[-5:])}), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
