"""One layer of a prompt from prefill to decoding: its cache in pages, the attention that hands its normalisers to the scoring, the
selection compacted into pages, continuations that share it, decoding steps replayed as a graph.

    python examples/serve_pruned.py            # needs an MI355X; random inputs
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2601_07667_amd import asl


def run(Hq=32, Hk=8, d=128, N=8192, W=32, budget=2048, continuations=6, steps=16, page_size=64, seed=0):
    """Returns what came out: the window's attention, the scores, the kept tokens, each step's outputs."""
    dev, S, n_keep = torch.device("cuda:0"), 7, min(budget, N)
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)

    def ints(*x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    ctx = asl.Asl(N, Hk + 1, Hq * W)
    ctx.asl_paged_reserve(continuations + 1, max(W, continuations) * Hq, d)

    # an empty cache: row 0 will be the prompt, row 1 what is kept of it, the others its continuations
    n_rows, width = 2 + continuations, -(-N // page_size) + 1
    n_pages = width + -(-n_keep // page_size) + continuations * (2 + steps // page_size) + 1
    k_pages, v_pages = normal(n_pages, Hk, page_size, d), normal(n_pages, Hk, page_size, d)
    table, kv_len = ints(*[0] * (n_rows * width)).view(n_rows, width), ints(*[0] * n_rows)
    refs = ints(*[0] * n_pages)
    pages = asl.make_pages(Hq, Hk, d, page_size, n_pages, n_rows, width)

    # prefill: the layer's keys and values into pages, then attention; here for the window's queries alone
    k, v, q_obs = normal(Hk, N, d), normal(Hk, N, d), normal(Hq, W, d)
    ctx.asl_pages_grow(pages, ints(0), ints(N), 1, table, kv_len, refs)
    ctx.asl_pages_write(pages, k, v, ints(0), ints(0, N), 1, N, table, kv_len, k_pages, v_pages)
    window = asl.make_attn(1, W, W, N)
    q, out = q_obs.transpose(0, 1), torch.empty((W, Hq, d), dtype=torch.bfloat16, device=dev)
    lse = torch.empty((Hq, W), dtype=torch.float32, device=dev)
    ctx.asl_paged_attention(pages, window, q, k_pages, v_pages, table, kv_len, ints(0, W), out, lse=lse)

    # the layer's scores in one pass over the keys, its selection; the kept tokens into pages of their own
    params = asl.make_params(Hq, Hk, d, N, W, S, budget)
    scores = torch.empty((Hk + 1, N - W), dtype=torch.float32, device=dev)
    ring = torch.zeros((8, N - W), dtype=torch.int32, device=dev)
    state, stat = asl.new_state(dev), asl.new_stat(dev)
    idx = torch.empty((Hk + 1, n_keep), dtype=torch.int32, device=dev)
    ctx.asl_layer_step(params, q_obs, k, None, 0, 10, 8, 0.3, scores, ring, state, stat, idx, lse=lse)
    ctx.asl_pages_grow(pages, ints(1), ints(n_keep), 1, table, kv_len, refs)
    ctx.asl_pages_compact(pages, ints(0), ints(1), ints(0, n_keep), 1, n_keep, idx[:Hk], table, kv_len, k_pages, v_pages)
    ctx.asl_pages_free(pages, ints(0), 1, table, kv_len, refs)

    # its continuations, one token a step each; the kept prompt is read once for all of them
    n = continuations
    rows, one, cu = ints(*range(2, 2 + n)), ints(*[1] * n), ints(*range(n + 1))
    group, prefix = ints(0, n), ints(n_keep)
    k_ptrs, v_ptrs = (torch.tensor([x.data_ptr()], dtype=torch.int64, device=dev) for x in (k_pages, v_pages))
    ctx.asl_pages_fork(pages, k_ptrs, v_ptrs, 1, ints(*[1] * n), rows, n, table, kv_len, refs)
    q1, k1, v1, o1 = normal(n, Hq, d), normal(n, Hk, d), normal(n, Hk, d), torch.empty((n, Hq, d), dtype=torch.bfloat16, device=dev)
    batch = asl.make_attn(n, n, 1, n_keep + steps + 1, n_groups=1)

    def step():
        ctx.asl_pages_grow(pages, rows, one, n, table, kv_len, refs)
        ctx.asl_pages_write(pages, k1.transpose(0, 1), v1.transpose(0, 1), rows, cu, n, n, table, kv_len, k_pages, v_pages)
        ctx.asl_paged_attention(pages, batch, q1, k_pages, v_pages, table, kv_len, cu, o1, rows=rows, group_start=group,
                                prefix_len=prefix)

    step()
    history, outputs = [(q1.clone(), k1.clone(), v1.clone())], [o1.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(steps - 1):
        q1.copy_(normal(n, Hq, d)), k1.copy_(normal(n, Hk, d)), v1.copy_(normal(n, Hk, d))
        graph.replay()
        history.append((q1.clone(), k1.clone(), v1.clone()))
        outputs.append(o1.clone())
    lengths = kv_len.tolist()
    ctx.asl_pages_free(pages, ints(*range(1, 2 + n)), 1 + n, table, kv_len, refs)
    left = int(refs.sum())
    fault = ctx.asl_device_fault()
    ctx.close()
    return dict(q=q, k=k, v=v, out=out, lse=lse, scores=scores, idx=idx, history=history, outputs=outputs, lengths=lengths,
                left=left, fault=fault)


if __name__ == "__main__":
    r = run()
    print("kept %d of %d tokens per head; continuations of %s tokens; pages still held: %d; faults: %d"
          % (r["idx"].shape[1], r["k"].shape[1], r["lengths"][2:], r["left"], r["fault"]))
