"""The paged calls on the GPU where their paths part: head sizes that leave a part of a store,
limits that change, work items of every kind."""
import numpy as np
import pytest

import paged_paths
from paper_2601_07667_amd import asl
from test_gpu_paged import Cache, _attend, _check, _dt, _ints, _oracle, _queries, ctx, wide  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wide_heads(gpu_device):
    c = asl.Asl(2, 1, 1)
    c.asl_paged_reserve(4096, 1 << 17, 256)
    yield c
    assert c.asl_device_fault() == 0
    c.close()


@pytest.mark.parametrize("dtype,d", [("f32", 68), ("f32", 100), ("f32", 132), ("f32", 252), ("f32", 4), ("f32", 60),
                                     ("bf16", 72), ("bf16", 136), ("bf16", 248)])
@pytest.mark.parametrize("lens,n_q", [([100, 128, 7, 64], [1, 3, 2, 1]),               # rows written whole
                                      ([1900, 300, 20, 700], [1, 2, 5, 1]),            # pieces joined within the launch
                                      ([3000, 260, 5], [2, 1, 4])])                    # pieces joined by a launch of their own
def test_rows_of_head_sizes_that_leave_a_part_of_a_store(ctx, gpu_device, lens, n_q, dtype, d):
    """Elements behind a row, between the heads and behind the last row of `out`, keep what they hold."""
    import torch
    Hq, Hk, total = 6, 2, sum(n_q)
    c = Cache(gpu_device, lens, Hk, d, 16, dtype, 21)
    q = _queries(total, Hq, d, dtype, gpu_device, 22)
    ref = _oracle(c, q, n_q)
    cu = _ints(np.concatenate([[0], np.cumsum(n_q)]), gpu_device)
    lse = torch.empty((Hq, total), dtype=torch.float32, device=gpu_device)
    a = asl.make_attn(len(lens), total, max(n_q), max(lens))
    for pad in (0, 8):
        room = torch.full((total * Hq * (d + pad) + 64,), 77.0, dtype=_dt(dtype), device=gpu_device)
        rows = room[:total * Hq * (d + pad)].view(total, Hq, d + pad)
        ctx.asl_paged_attention(c.desc(Hq), a, q, c.k, c.v, c.table, c.kv_len, cu, rows[..., :d], lse=lse)
        _check(rows[..., :d], lse, ref, d, max(lens), dtype, "d %d, pad %d" % (d, pad))
        assert bool((rows[..., d:] == 77).all()) and bool((room[total * Hq * (d + pad):] == 77).all())
    assert ctx.asl_device_fault() == 0


def test_a_fault_outlives_new_limits(gpu_device):
    import torch
    x = asl.Asl(2, 1, 1)
    i = lambda *v: _ints(v, gpu_device)
    table, kv, refs = torch.zeros((2, 4), dtype=torch.int32, device=gpu_device), i(0, 0), i(*[0] * 8)
    p = asl.make_pages(1, 1, 64, 16, 8, 2, 4)
    for limits in ((4, 64, 64), (2, 8, 16), (4, 5000, 64), (4, 5000, 256), (4096, 1 << 20, 256), (1, 1, 1)):
        x.asl_paged_reserve(*limits)
        assert x.asl_device_fault() == 0
        x.asl_pages_grow(p, i(9), i(1), 1, table, kv, refs)               # no such row
        x.asl_paged_reserve(4, 20000 if limits[0] == 4 else 1, 256)
        assert x.asl_device_fault() == 2, limits
    x.close()


def test_graphs_captured_before_new_limits_keep_their_workspace(gpu_device):
    """A graph that joins pieces in the launch, one that joins them after it, and one that grows, writes and forks: captured, the limits
    raised and lowered, replayed between calls under the new ones."""
    import torch
    dev = gpu_device
    x = asl.Asl(2, 1, 1)
    x.asl_paged_reserve(8, 64, 64)
    lens = [1900, 300, 20, 700]
    c = Cache(dev, lens, 2, 64, 16, "bf16", 31)
    q, n_q = _queries(4, 4, 64, "bf16", dev, 32), [1] * 4
    cu = _ints(range(5), dev)
    outs = [torch.empty_like(q) for _ in range(2)]
    lses = [torch.empty((4, 4), dtype=torch.float32, device=dev) for _ in range(2)]
    batches = [asl.make_attn(4, 4, 1, most) for most in (2000, 20000)]
    i = lambda *v: _ints(v, dev)
    pages = asl.make_pages(2, 2, 64, 16, 40, 6, 8)
    table, kv, refs = torch.zeros((6, 8), dtype=torch.int32, device=dev), torch.zeros(6, dtype=torch.int32, device=dev), i(*[0] * 40)
    kp, vp = (torch.zeros((40, 2, 16, 64), dtype=torch.bfloat16, device=dev) for _ in range(2))
    kptr, vptr = (torch.tensor([t.data_ptr()], dtype=torch.int64, device=dev) for t in (kp, vp))
    new = _queries(2 * 21, 1, 64, "bf16", dev, 33).reshape(2, 21, 64)
    lists = dict(row=i(0), add=i(21), cu=i(0, 21), parents=i(0, 0, 0), children=i(1, 2, 3), all=i(0, 1, 2, 3))

    def attend():
        for a, out, lse in zip(batches, outs, lses):
            x.asl_paged_attention(c.desc(4), a, q, c.k, c.v, c.table, c.kv_len, cu, out, lse=lse)

    def books():
        x.asl_pages_grow(pages, lists["row"], lists["add"], 1, table, kv, refs)
        x.asl_pages_write(pages, new, new, lists["row"], lists["cu"], 1, 21, table, kv, kp, vp)
        x.asl_pages_fork(pages, kptr, vptr, 1, lists["parents"], lists["children"], 3, table, kv, refs)

    attend()
    books()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs + lses]
    _check(outs[0], lses[0], _oracle(c, q, n_q), 64, max(lens), "bf16", "before")
    want_books = [t.clone() for t in (table, kv, refs, kp, vp)]
    x.asl_pages_free(pages, lists["all"], 4, table, kv, refs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attend()
        books()
    limits = [(8, 64, 64), (8, 100, 64), (8, 60000, 64), (2, 8, 16), (4096, 1 << 18, 256), (8, 16, 64)]
    for limit in limits:
        x.asl_paged_reserve(*limit)
        fill = torch.full((1 << 24,), -1, dtype=torch.int32, device=dev)      # what a freed workspace could be handed out as
        for t in outs + lses:
            t.fill_(float("nan"))
        for t in (kv, refs, kp, vp):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs + lses, want)), limit
        assert all(torch.equal(a, b) for a, b in zip((kv, refs, kp, vp), want_books[1:])), limit
        assert bool((fill == -1).all())
        if limit[0] >= 8 and limit[1] >= 16 and limit[2] >= 64:               # the same calls now
            for t in outs + lses:
                t.fill_(float("nan"))
            attend()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs + lses, want)), limit
    assert x.asl_device_fault() == 0
    x.close()


# ----------------------------------------------------------------------------------- work items of every kind
def _cache(dev, c, seed):
    """The case's rows.  A group's members read its prefix from their first one's pages: their own table entries for the whole tiles of it
    lead to a page of NaN, so that a call that does not read them apart shows."""
    lens, groups, ps = c["lens"], c["groups"] or [], c["ps"]
    x = Cache(dev, lens, c["Hk"], c["d"], ps, c["dtype"], seed)
    at, poison = 0, next((p for p in range(x.n_pages) if x.refs_host[p] == 0))
    table = x.host_table.copy()
    for m, p in groups:
        tokens = min(p, lens[at]) // 64 * 64 if m > 1 else 0
        for r in range(at + 1, at + m):
            n = min(p, lens[r])
            for pages in x.pages_t:                          # the same tokens
                for t in range(0, -(-n // ps)):
                    part = min(ps, n - t * ps)
                    pages[x.host_table[r, t], :, :part] = pages[x.host_table[at, t], :, :part]
            if tokens >= 128:
                table[r, :tokens // ps] = poison
        at += m
    x.table = _ints(table, dev)
    assert bool(x.k[poison].isnan().all())
    return x


def _run(ctx, dev, c, x, q):
    groups = c["groups"]
    return _attend(ctx, x, q, c["n_q"], c["Hq"], c["causal"], groups, max_kv=c["max_kv"])


@pytest.mark.parametrize("c", paged_paths.shared_cases(), ids=lambda c: c["name"])
def test_prefixes_that_are_read_apart(wide, wide_heads, gpu_device, c):
    x = _cache(gpu_device, c, 41)
    q = _queries(sum(c["n_q"]), c["Hq"], c["d"], c["dtype"], gpu_device, 42)
    ctx = wide if c["d"] <= 128 else wide_heads
    out, lse = _run(ctx, gpu_device, c, x, q)
    _check(out, lse, _oracle(x, q, c["n_q"], causal=c["causal"]), c["d"], max(c["lens"]), c["dtype"], c["name"])
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("c", paged_paths.tile_cases(), ids=lambda c: c["name"])
def test_tiles(wide, gpu_device, c):
    x = _cache(gpu_device, c, 43)
    q = _queries(sum(c["n_q"]), c["Hq"], c["d"], c["dtype"], gpu_device, 44)
    out, lse = _run(wide, gpu_device, c, x, q)
    _check(out, lse, _oracle(x, q, c["n_q"], causal=c["causal"]), c["d"], max(c["lens"]), c["dtype"], c["name"])
    assert wide.asl_device_fault() == 0
