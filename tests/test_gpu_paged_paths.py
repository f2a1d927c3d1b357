"""The paged calls on the GPU where their paths part: head sizes that leave a part of a store,
limits that change, work items of every kind."""
import numpy as np
import pytest

import paged_paths
from paper_2601_07667_amd import asl
from test_gpu_paged import Cache, _attend, _bounds, _check, _dt, _ints, _oracle, _queries, ctx, wide  # noqa: F401

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


def _same_where_seen(out, lse, ref, d, n_keys, dtype, what):
    """Like _check, with infinities and NaN where the oracle has them."""
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        tol, tol_lse = _bounds(d, n_keys, dtype, ref)
        finite = np.isfinite(ref[0])
        assert np.array_equal(o[~finite], ref[0][~finite], equal_nan=True), (what, "not finite")
        assert np.all(np.abs(o - ref[0])[finite] <= tol[finite]), (what, "out")
        seen = np.isfinite(ref[1])
        assert np.array_equal(l[~seen], ref[1][~seen], equal_nan=True), (what, "lse of rows without keys")
        assert np.all(np.abs(l - ref[1])[seen] <= tol_lse[seen]), (what, "lse")


ODD = [c for c in paged_paths.tile_cases() if c["causal"] and max(c["n_q"]) >= 17 and c["d"] >= 64] + [
    c for c in paged_paths.shared_cases() if c["name"] in ("members of any length", "drafts", "tiles for both", "tiles beside split prefixes")]


@pytest.mark.filterwarnings("ignore:invalid value encountered")
@pytest.mark.parametrize("c", ODD, ids=lambda c: "%s, %d %d" % ((c["name"],) + c["kinds"]))
def test_values_that_are_no_numbers_reach_those_that_see_them(wide, gpu_device, c):
    """Infinities of either sign and NaN among the values, where some queries of a sequence see them and others do not, and in sight of all:
    each reaches its element of the queries that see it.  NaN, infinite and lowest keys and values behind what any query sees reach nobody."""
    import torch
    x = _cache(gpu_device, c, 45)
    q = _queries(sum(c["n_q"]), c["Hq"], c["d"], c["dtype"], gpu_device, 46, spread=1.0)
    inf, nan, ps = float("inf"), float("nan"), c["ps"]
    lowest = torch.finfo(torch.bfloat16).min
    firsts, at = {}, 0                                       # whose pages hold a member's prefix
    for m, p in c["groups"] or []:
        tokens = min(p, c["lens"][at]) // 64 * 64 if m > 1 else 0
        firsts.update({r: (at, min(tokens, c["lens"][r]) if tokens >= 128 else 0) for r in range(at, at + m)})
        at += m

    def put(r, t, e, value, of=x.v):
        """Token t of row r, in its own pages and, of a prefix, in those of every member that has it."""
        a, shared = firsts.get(r, (r, 0))
        rows = [s for s in firsts if firsts[s][0] == a and t < c["lens"][s]] if t < shared else [r]
        for s in rows:
            of[x.host_table[s, t // ps], 0, t % ps, e] = value

    for r, (L, n) in enumerate(zip(c["lens"], c["n_q"])):
        if L < 3 or n < 3:
            continue
        d, last = c["d"], min(n, L)
        put(r, L - 1, 1, inf)                                # the last query alone sees it
        put(r, L - last // 2 - 1, 5 % d, -inf)
        put(r, L - last // 2 - 1, d - 1, nan)
        put(r, L - 2, 6, inf)
        put(r, L - 1, 6, -inf)                               # the last query: NaN
        put(r, 0, 7, inf)                                    # all
        put(r, L // 2, d // 2, -inf)
    want = _oracle(x, q, c["n_q"], causal=True)
    for r, L in enumerate(c["lens"]):                        # slots behind a row's end
        if L % ps:
            for of, values in ((x.k, (nan, inf, -inf, lowest)), (x.v, (inf, lowest, nan, -inf))):
                for i, value in enumerate(values):
                    of[x.host_table[r, L // ps], :, L % ps + i:L % ps + i + 1] = value
    out, lse = _run(wide, gpu_device, c, x, q)
    _same_where_seen(out, lse, want, c["d"], max(c["lens"]), c["dtype"], c["name"])
    assert not np.isfinite(want[0]).all() and wide.asl_device_fault() == 0


@pytest.mark.parametrize("c", paged_paths.leap_cases(), ids=lambda c: c["name"])
def test_logits_that_rise_from_tile_to_tile(wide, gpu_device, c):
    """For the first KV head the largest logit of some rows grows by tens and hundreds of nats from tile to tile, in sight of all and among
    the last tokens; for the second it falls; for the last the first 80 tokens and one of the last have logits of -Inf in fp32."""
    import torch
    x = _cache(gpu_device, c, 47)
    lens, n_q, d, Hk, ps, P = c["lens"], c["n_q"], c["d"], c["Hk"], c["ps"], paged_paths.LEAP_PREFIX
    G = c["Hq"] // Hk
    lowest = [*range(80), P + 1]
    for r in range(len(lens)):
        for t, size in ((70, 2.0), (130, 4.0), (200, 8.0), (420, 9.0), (P - 1, 12.0), (P + 3, 16.0), (P + 20, 24.0)):
            x.k[x.host_table[r, t // ps], 0, t % ps] = size
            x.k[x.host_table[r, t // ps], 1, t % ps] = -size
        for t in lowest:
            x.k[x.host_table[r, t // ps], Hk - 1, t % ps] = 0
    q = _queries(sum(n_q), c["Hq"], d, "bf16", gpu_device, 48, spread=0.5)
    q[:, :2 * G:3] = q[:, :2 * G:3].abs() * 2 + 1
    q[:, -G:] = q[:, -G:].abs() + 0.5
    reach = _oracle(x, q, n_q)[3]                            # without the keys that count for nothing
    for r in range(len(lens)):
        for t in lowest:
            x.k[x.host_table[r, t // ps], Hk - 1, t % ps] = torch.finfo(torch.bfloat16).min
    want = _oracle(x, q, n_q)
    out, lse = _run(wide, gpu_device, c, x, q)
    _check(out, lse, (want[0], want[1], want[2], reach), d, max(lens), "bf16", c["name"])
    assert wide.asl_device_fault() == 0


@pytest.mark.parametrize("kinds,n_q,max_kv,dtype", [((16, 0), 1, None, "f32"), ((16, 0), 4, None, "bf16"), ((64, 0), 16, paged_paths.WIDE, "bf16"),
                                                   ((128, 0), 33, paged_paths.WIDE, "bf16")])
def test_values_up_to_the_stated_size_do_not_overflow(wide, gpu_device, kinds, n_q, max_kv, dtype):
    """n keys, values just below 2^103 / n, and logits that rise by 23.4 bits behind the first tile, where a reference stays."""
    n = 4096
    c = paged_paths.case("large values", kinds, [n], [n_q], 4, 1, 64, max_kv=max_kv, dtype=dtype)
    x = _cache(gpu_device, c, 51)
    q = _queries(n_q, 4, 64, dtype, gpu_device, 52) * 0 + 1
    for t in range(n):
        x.k[x.host_table[0, t // 16], 0, t % 16] = 0.0 if t < 64 else 2.03125
        x.v[x.host_table[0, t // 16], 0, t % 16] = 0.99 * 2.0 ** 91 * (1 if t % 3 else -1)
    out, lse = _run(wide, gpu_device, c, x, q)
    _check(out, lse, _oracle(x, q, [n_q]), 64, n, dtype, "large values")
    assert wide.asl_device_fault() == 0


@pytest.mark.parametrize("c", paged_paths.large_cases(), ids=lambda c: c["name"])
def test_more_rows_than_the_workspace_grows_with(gpu_device, c):
    ctx = asl.Asl(2, 1, 1)
    ctx.asl_paged_reserve(4096, 1 << 18, 64)
    x = _cache(gpu_device, c, 53)
    q = _queries(sum(c["n_q"]), c["Hq"], c["d"], c["dtype"], gpu_device, 54)
    out, lse = _run(ctx, gpu_device, c, x, q)
    _check(out, lse, _oracle(x, q, c["n_q"], causal=c["causal"]), c["d"], max(c["lens"]), c["dtype"], c["name"])
    assert ctx.asl_device_fault() == 0
    ctx.close()
