"""Drafting over a pruned prompt: its keys rotated and scored, the selection in pages, and then steps that draft a tree of tokens for each of
its continuations: planned, rotated into the pages, attended over and cut back to the accepted path, the whole step replayed as a graph.

    python examples/draft_pruned.py            # needs an MI355X; random inputs, and coins for the verdict on each drafted token
"""
import os
import random
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2601_07667_amd import asl


def run(Hq=32, Hk=8, d=128, N=8192, W=32, budget=2048, sequences=6, nodes=16, steps=8, page_size=64, seed=0):
    """Returns what came out: the prompt's keys and its kept tokens, of each step the trees, paths, inputs and outputs, the last lengths."""
    dev, n, n_keep = torch.device("cuda:0"), sequences, min(budget, N)
    g, coin = torch.Generator(device=dev).manual_seed(seed), random.Random(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)

    def ints(*x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    ctx = asl.Asl(N, Hk + 1, Hq * W)
    ctx.asl_paged_reserve(n + 1, n * nodes * Hq, d)
    freqs = asl.rotation_freqs(d, base=500000.0, kind=asl.ASL_FREQS_PARTS, factor=8.0, context=8192.0, low=1.0, high=4.0).to(dev)
    place = torch.arange(N, dtype=torch.int32, device=dev)

    # the prompt: rotated, scored by its window, its best tokens and the window kept in row 0
    k, v, q = normal(N, Hk, d), normal(Hk, N, d), normal(W, Hq, d)
    kr, qr = torch.empty((Hk, N, d), dtype=torch.bfloat16, device=dev), torch.empty((Hq, W, d), dtype=torch.bfloat16, device=dev)
    ctx.asl_rotate(asl.make_rotation(0, Hk, d), None, k, place, freqs, None, kr.transpose(0, 1))
    ctx.asl_rotate(asl.make_rotation(Hq, 0, d), q, None, place[N - W:], freqs, qr.transpose(0, 1), None)
    scores = torch.empty((Hk + 1, N - W), dtype=torch.float32, device=dev)
    ring = torch.zeros((8, N - W), dtype=torch.int32, device=dev)
    state, stat = asl.new_state(dev), asl.new_stat(dev)
    idx = torch.empty((Hk + 1, n_keep), dtype=torch.int32, device=dev)
    ctx.asl_layer_step(asl.make_params(Hq, Hk, d, N, W, 7, budget), qr, kr, None, 0, 10, 8, 0.3, scores, ring, state, stat, idx)

    n_rows, width = 1 + n, -(-(n_keep + (steps + 1) * nodes) // page_size) + 1
    n_pages = -(-n_keep // page_size) + n * (2 + (steps + 1) * nodes // page_size) + 1
    k_pages, v_pages = normal(n_pages, Hk, page_size, d), normal(n_pages, Hk, page_size, d)
    table, kv_len = ints(*[0] * (n_rows * width)).view(n_rows, width), ints(*[0] * n_rows)
    refs = ints(*[0] * n_pages)
    pages = asl.make_pages(Hq, Hk, d, page_size, n_pages, n_rows, width)
    ctx.asl_pages_grow(pages, ints(0), ints(n_keep), 1, table, kv_len, refs)
    ctx.asl_pages_write(pages, kr, v, ints(0), ints(0, n_keep), 1, n_keep, table, kv_len, k_pages, v_pages, idx=idx[:Hk])

    # its continuations: the kept tokens in common, and every row's positions ahead of its places by what was taken out
    k_ptrs, v_ptrs = (torch.tensor([x.data_ptr()], dtype=torch.int64, device=dev) for x in (k_pages, v_pages))
    rows, pruned, total = ints(*range(1, 1 + n)), ints(*[N - n_keep] * n_rows), n * nodes
    ctx.asl_pages_fork(pages, k_ptrs, v_ptrs, 1, ints(*[0] * n), rows, n, table, kv_len, refs)
    group, prefix = ints(0, n), ints(n_keep // page_size * page_size)
    add, parent, path, n_path = ints(*[0] * n), ints(*[0] * total), ints(*[0] * total).view(n, nodes), ints(*[0] * n)
    cu, pos, slot = ints(*[0] * (n + 1)), ints(*[0] * total), torch.zeros(total, dtype=torch.int64, device=dev)
    x, qt, out = normal(total, Hq + 2 * Hk, d), normal(total, Hq, d), normal(total, Hq, d)
    rotation = asl.make_rotation(Hq, Hk, d)
    batch = asl.make_attn(n, total, nodes, n_keep + (steps + 1) * nodes, n_groups=1)

    def step():
        ctx.asl_pages_plan(pages, rows, add, n, total, table, kv_len, refs, cu, slot, pos, parent=parent, pruned=pruned)
        ctx.asl_rotate_write(pages, rotation, x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:], pos, slot, freqs, qt, k_pages, v_pages)
        ctx.asl_tree_attention(pages, batch, qt, k_pages, v_pages, table, kv_len, cu, parent, out, rows=rows, group_start=group,
                               prefix_len=prefix)
        ctx.asl_pages_accept(pages, k_ptrs, v_ptrs, 1, rows, cu, path, n_path, n, table, kv_len, refs, slot=slot)

    history, graph = [], None
    for _ in range(steps):
        # trees of up to `nodes` nodes, and a path from a root on for as long as the coins fall well
        trees = [[coin.randrange(-1, i) if i else -1 for i in range(coin.randint(1, nodes))] for _ in range(n)]
        paths = []
        for t in trees:
            kept, at = [], -1
            for i, p in enumerate(t):
                if p == at and coin.random() < 0.6:
                    kept.append(i)
                    at = i
            paths.append(kept)
        flat = [p for t in trees for p in t]
        add.copy_(ints(*[len(t) for t in trees])), parent.copy_(ints(*flat + [-1] * (total - len(flat))))
        path.copy_(torch.stack([ints(*p + [-1] * (nodes - len(p))) for p in paths])), n_path.copy_(ints(*[len(p) for p in paths]))
        x.copy_(normal(*x.shape))
        if graph is None:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        graph.replay()
        history.append(dict(trees=trees, paths=paths, x=x.clone(), q=qt.clone(), out=out.clone(), pos=pos.clone()))
    lengths = kv_len.tolist()
    ctx.asl_pages_free(pages, ints(*range(n_rows)), n_rows, table, kv_len, refs)
    left, fault = int(refs.sum()), ctx.asl_device_fault()
    ctx.close()
    return dict(k=kr, v=v, idx=idx, freqs=freqs, history=history, lengths=lengths, left=left, fault=fault)


if __name__ == "__main__":
    r = run()
    drafted, kept = (sum(len(t) for h in r["history"] for t in h[key]) for key in ("trees", "paths"))
    print("%d tokens kept of the prompt; %d drafted, %d accepted; sequences of %s tokens; pages still held: %d; faults: %d"
          % (r["idx"].shape[1], drafted, kept, r["lengths"][1:], r["left"], r["fault"]))
