"""The paged cache on the GPU against its float64 oracle."""
import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2601_07667_amd import asl

pytestmark = pytest.mark.gpu

NP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}      # a rounding, relative to the value


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = asl.Asl(2, 1, 1)
    c.asl_paged_reserve(300, 1 << 17, 256)
    yield c
    assert c.asl_device_fault() == 0, "a test left the fault word set"
    c.close()


def _torch():
    import torch
    return torch


def _dt(dtype):
    torch = _torch()
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _ints(x, dev):
    torch = _torch()
    return torch.tensor(np.asarray(x, dtype=np.int32), device=dev)


class Cache:
    """Pages with the given rows, page numbers shuffled; what no token fills holds NaN."""

    def __init__(self, dev, lens, Hk, d, ps, dtype, seed=0, shared=(), row_stride=None, spare=3, gap=0, layers=1):
        torch = _torch()
        rng = np.random.default_rng(seed)
        self.lens, self.Hk, self.d, self.ps, self.dtype, self.dev = list(lens), Hk, d, ps, dtype, dev
        need = [-(-x // ps) for x in lens]
        self.width = row_stride or max(need + [0]) + 2
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        table, at = np.full((len(lens), self.width), -1, dtype=np.int64), 0
        for r, n in enumerate(need):
            table[r, :n] = order[at:at + n]
            at += n
        for a, b, prefix in shared:                          # rows a+1 .. b-1 begin like row a, in the same pages
            table[a:b, :prefix // ps] = table[a, :prefix // ps]
        self.host_table = table
        self.refs_host = np.bincount(np.concatenate([table[r, :n] for r, n in enumerate(need)] + [np.zeros(0, dtype=np.int64)]),
                                     minlength=self.n_pages).astype(np.int64)
        self.pages_t = []
        for _ in range(2 * layers):                          # a gap behind each page, NaN too
            x = torch.full((self.n_pages, Hk * ps * d + gap), float("nan"), dtype=_dt(dtype), device=dev)
            view = x[:, :Hk * ps * d].view(self.n_pages, Hk, ps, d)
            val = torch.from_numpy(rng.standard_normal((self.n_pages, Hk, ps, d), dtype=np.float32)).to(dev).to(_dt(dtype))
            used = torch.zeros((self.n_pages, ps), dtype=torch.bool)
            for r, n in enumerate(lens):
                for t in range(need[r]):
                    used[table[r, t], :max(0, min(ps, n - t * ps))] = True
            u = used.to(dev)[:, None, :, None]
            view.copy_(torch.where(u, val, torch.full_like(val, float("nan"))))
            self.pages_t.append(view)
        for a, b, prefix in shared:                          # the last, partly shared page: copies
            part = prefix % ps
            for r in range(a + 1, b):
                for x in self.pages_t:
                    if part:
                        x[table[r, prefix // ps], :, :part] = x[table[a, prefix // ps], :, :part]
        self.k, self.v = self.pages_t[0], self.pages_t[1]
        self.table, self.kv_len, self.refs = _ints(table, dev), _ints(lens, dev), _ints(self.refs_host, dev)
        self.gap = gap

    def desc(self, Hq=None, scale=0.0):
        s = self.Hk * self.ps * self.d
        return asl.make_pages(Hq or self.Hk, self.Hk, self.d, self.ps, self.n_pages, len(self.lens), self.width,
                              dtype=asl.ASL_BF16 if self.dtype == "bf16" else asl.ASL_F32,
                              strides=(s + self.gap, self.ps * self.d, self.d), scale=scale)

    def row(self, x, r):
        """Tokens of row r, float64 [Hk, len, d]."""
        return po.gather(x.double().cpu().numpy(), self.host_table[r], self.lens[r])


def _bounds(d, n_keys, dtype, ref, scale=1.0):
    """How far out and lse may be off.  Logits: d products summed in fp32 (each partial sum rounds, at most `reach` large), and the
    scaling, the change of base and exp2 round too.  Their error e multiplies every p, so it moves out by 2 e spread and lse by
    e.  Sums of n terms in fp32, merged in pieces.  In bf16 p rounds before its product with v, and out rounds at the end."""
    out, lse, spread, reach = ref
    e = reach * (d + 8) * 2.0 ** -24 + 2.0 ** -21
    sums = (n_keys + 64) * 2.0 ** -24
    rel = NP[dtype]
    tol = rel * np.abs(out) + (rel + 2 * e[..., None] + 3 * sums) * spread * 1.01 + 1e-30
    with np.errstate(invalid="ignore"):
        tol_lse = e.T + sums + np.where(np.isfinite(lse), np.abs(lse), 0) * 2.0 ** -22
    return tol, tol_lse


def _check(out, lse, ref, d, n_keys, dtype, what):
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    tol, tol_lse = _bounds(d, n_keys, dtype, ref)
    assert np.all(np.isfinite(o)), what
    bad = np.abs(o - ref[0]) > tol
    assert not bad.any(), (what, "out", int(bad.sum()), float((np.abs(o - ref[0]) / tol).max()), np.argwhere(bad)[:4].tolist())
    gone = ~np.isfinite(ref[1])
    assert np.array_equal(l[gone], ref[1][gone]), what
    off = np.abs(l[~gone] - ref[1][~gone]) > tol_lse[~gone]
    assert not off.any(), (what, "lse", float(np.abs(l[~gone] - ref[1][~gone]).max()))


def _queries(n_tok, Hq, d, dtype, dev, seed, pad=0, spread=2.0):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    x = torch.full((n_tok, Hq, d + pad), float("nan"), dtype=_dt(dtype), device=dev)
    x[..., :d] = (torch.randn((n_tok, Hq, d), generator=g) * spread).to(_dt(dtype)).to(dev)
    return x[..., :d]


def _attend(ctx, c, q, n_q, Hq, causal=True, groups=None, rows=None, scale=0.0, max_q=None, max_kv=None, pad=0):
    torch = _torch()
    dev, total = c.dev, int(sum(n_q))
    cu = _ints(np.concatenate([[0], np.cumsum(n_q)]), dev)
    out = torch.full((max(total, 1), Hq, c.d + pad), float("nan"), dtype=_dt(c.dtype), device=dev)[:total, :, :c.d]
    lse = torch.full((Hq, total), float("nan"), dtype=torch.float32, device=dev)
    a = asl.make_attn(len(n_q), total, max_q if max_q is not None else max(n_q), max_kv if max_kv is not None else max(c.lens),
                      n_groups=len(groups) if groups else 0, causal=causal)
    gs = pl = None
    if groups:
        gs = _ints(np.concatenate([[0], np.cumsum([m for m, _ in groups])]), dev)
        pl = _ints([p for _, p in groups], dev)
    ctx.asl_paged_attention(c.desc(Hq, scale), a, q, c.k, c.v, c.table, c.kv_len, cu, out, lse=lse,
                            rows=None if rows is None else _ints(rows, dev), group_start=gs, prefix_len=pl)
    torch.cuda.synchronize()
    return out, lse


def _oracle(c, q, n_q, scale=0.0, causal=True, rows=None):
    q, k, v = (x.double().cpu().numpy() for x in (q, c.k, c.v))
    row = lambda x, r: po.gather(x, c.host_table[r], c.lens[r])
    parts, at = [], 0
    for b, n in enumerate(n_q):
        r = b if rows is None else rows[b]
        parts.append(po.attention(q[at:at + n], row(k, r), row(v, r), scale or c.d ** -0.5, causal))
        at += n
    return (np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts], axis=1),
            np.concatenate([p[2] for p in parts]), np.concatenate([p[3] for p in parts]))


def _case(ctx, dev, lens, n_q, Hq, Hk, d, ps, dtype, causal=True, groups=None, seed=0, pad=0, gap=0, rows=None, scale=0.0, what="",
          spread=2.0, **bounds):
    shared, at = [], 0
    for m, p in groups or []:
        shared.append((at, at + m, min([p] + list(lens[at:at + m]))))
        at += m
    c = Cache(dev, lens, Hk, d, ps, dtype, seed, shared=shared, gap=gap)
    q = _queries(sum(n_q), Hq, d, dtype, dev, seed + 1, pad, spread)
    out, lse = _attend(ctx, c, q, n_q, Hq, causal, groups, rows, scale, pad=pad, **bounds)
    _check(out, lse, _oracle(c, q, n_q, scale, causal, rows), d, max(lens), dtype, what)
    assert ctx.asl_device_fault() == 0
    return c, q, out, lse


HEADS = [(4, 2, 64), (8, 8, 128), (28, 4, 128), (32, 2, 128), (6, 2, 80), (5, 1, 256), (3, 3, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hk,d", HEADS)
def test_attention_one_token_of_ragged_sequences(ctx, gpu_device, Hq, Hk, d, dtype):
    lens = [1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 300, 0, 517]
    _case(ctx, gpu_device, lens, [1] * len(lens), Hq, Hk, d, 16, dtype, what="ragged")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps", [16, 32, 64, 256, 4096])
def test_attention_page_sizes(ctx, gpu_device, ps, dtype):
    _case(ctx, gpu_device, [700, 3, ps, ps + 1], [1, 3, 2, 1], 8, 2, 128, ps, dtype, what="ps %d" % ps)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hk,d", HEADS)
@pytest.mark.parametrize("causal", [True, False])
def test_attention_many_tokens(ctx, gpu_device, Hq, Hk, d, causal, dtype):
    """Drafts and chunks; sequences with fewer keys than queries, with none, and without queries."""
    _case(ctx, gpu_device, [70, 5, 0, 200, 9, 130, 33], [17, 9, 3, 40, 0, 1, 33], Hq, Hk, d, 32, dtype, causal, what="many")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q", [1, 2, 4, 5, 8, 9, 16, 17, 32, 33, 65, 129])
def test_attention_row_counts(ctx, gpu_device, n_q, dtype):
    """Query rows of one KV head around every tile height (four heads share it)."""
    _case(ctx, gpu_device, [200 + n_q, 260], [n_q, max(1, n_q - 1)], 8, 2, 64, 16, dtype, what="rows %d" % n_q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 500, 4097, 20000, 70001])
def test_attention_long(ctx, gpu_device, n, dtype):
    """A few rows over a long axis: the work is split and joined."""
    _case(ctx, gpu_device, [n], [1], 8, 2, 128, 64, dtype, what="long %d" % n)
    _case(ctx, gpu_device, [n, 1 + n // 3], [2, 1], 14, 2, 64, 16, dtype, seed=5, what="long %d" % n)


def test_attention_long_chunk(ctx, gpu_device):
    _case(ctx, gpu_device, [1100, 700], [300, 257], 8, 2, 128, 64, "bf16", what="chunk")
    _case(ctx, gpu_device, [1000], [1000], 4, 1, 64, 16, "bf16", what="whole prompt")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,G", [(128, 4), (64, 7), (256, 2), (80, 1)])
@pytest.mark.parametrize("groups,own,n_q", [
    ([(5, 300)], [1, 2, 33, 64, 200], [1] * 5),
    ([(3, 129), (1, 70), (4, 512)], [5, 6, 7, 3, 40, 1, 2, 17], [1, 2, 3, 1, 5, 1, 2, 4]),
    ([(2, 0), (3, 31), (2, 700)], [3, 20, 9, 8, 7, 6, 5], [1, 1, 2, 2, 2, 1, 1]),
    ([(40, 200)], [1 + i % 7 for i in range(40)], [1] * 40),
    ([(6, 1500)], [30, 31, 32, 33, 34, 35], [12, 13, 14, 15, 16, 30]),
])
def test_attention_shared_prefix(ctx, gpu_device, groups, own, n_q, d, G, dtype):
    lens = [p for m, p in groups for _ in range(m)]
    lens = [p + x for p, x in zip(lens, own)]
    c, q, out, lse = _case(ctx, gpu_device, lens, n_q, 2 * G, 2, d, 16, dtype, groups=groups, what="shared")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_prefix_longer_than_what_all_queries_see(ctx, gpu_device, dtype):
    """A stated prefix that reaches into the queries' own tokens, or past a sequence's end: only what all see is shared."""
    torch = _torch()
    c = Cache(gpu_device, [200, 200, 200], 2, 64, 16, dtype, 3, shared=[(0, 3, 200)])
    q = _queries(30, 4, 64, dtype, gpu_device, 9)
    for stated in (200, 10 ** 6, -5, 195):
        out, lse = _attend(ctx, c, q, [10, 10, 10], 4, True, groups=[(3, stated)])
        _check(out, lse, _oracle(c, q, [10, 10, 10]), 64, 200, dtype, "stated %d" % stated)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_strides_rows_and_scale(ctx, gpu_device, dtype):
    torch = _torch()
    lens = [90, 40, 17]
    c = Cache(gpu_device, lens, 2, 64, 16, dtype, 2, gap=64)
    q = _queries(10, 8, 64, dtype, gpu_device, 3, pad=24)
    rows, n_q = [2, 0, 2], [3, 2, 5]
    out, lse = _attend(ctx, c, q, n_q, 8, True, None, rows, 0.37, pad=24)
    _check(out, lse, _oracle(c, q, n_q, 0.37, True, rows), 64, 90, dtype, "strides")
    qt = q.transpose(0, 1).contiguous().transpose(0, 1)                  # heads outermost, as the scoring takes its window
    out2, lse2 = _attend(ctx, c, qt, n_q, 8, True, None, rows, 0.37)
    assert torch.equal(out2, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_bounds_only_cut_the_work(ctx, gpu_device, dtype):
    """max_q_len and max_kv_len that are too small or too large change no result beyond rounding."""
    lens, n_q = [300, 40, 7], [9, 2, 5]
    for mq, mk in ((9, 300), (1, 1), (0, 0), (5000, 1 << 24)):
        _case(ctx, gpu_device, lens, n_q, 8, 2, 64, 16, dtype, max_q=mq, max_kv=mk, what="bounds")
    for mq, mk in ((1, 1), (5000, 1 << 24)):
        _case(ctx, gpu_device, [1300, 1340, 1307], n_q, 8, 2, 64, 16, dtype, groups=[(3, 1200)], max_q=mq, max_kv=mk, what="bounds")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_peaks_and_large_logits(ctx, gpu_device, dtype):
    """Logits of hundreds, the largest at the beginning, in the middle and at the end; equal logits."""
    torch = _torch()
    for seed, spread in ((0, 40.0), (1, 0.0), (2, 200.0)):
        _case(ctx, gpu_device, [400, 77], [1, 6], 8, 2, 128, 16, dtype, seed=seed, spread=spread, what="spread %g" % spread)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), "lowest"])
@pytest.mark.parametrize("n_q", [7, 70])
def test_attention_what_is_masked_may_hold_anything(ctx, gpu_device, dtype, bad, n_q):
    """A token that only later queries see: its NaN, infinity or lowest value reaches those and no others."""
    torch = _torch()
    value = torch.finfo(_dt(dtype)).min if bad == "lowest" else bad
    L, at = 150 + n_q, 150 + n_q - 4
    c = Cache(gpu_device, [L, 40], 2, 64, 16, dtype, 4)
    q = _queries(n_q + 2, 8, 64, dtype, gpu_device, 5)
    n = [n_q, 2]
    want = _oracle(c, q, n)
    slot = (c.host_table[0, at // 16], slice(None), at % 16)
    c.v[slot] = value
    c.k[slot] = value
    out, lse = _attend(ctx, c, q, n, 8)
    rows = [i for i in range(n_q + 2) if i < at - (L - n_q) or i >= n_q]    # those that do not see it
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    tol, tol_lse = _bounds(64, L, dtype, want)
    assert np.all(np.abs(o[rows] - want[0][rows]) <= tol[rows])
    assert np.all(np.abs(l[:, rows] - want[1][:, rows]) <= tol_lse[:, rows])
    if isinstance(bad, float) and np.isnan(bad):
        assert np.all(np.isnan(o[at - (L - n_q):n_q]))


def test_attention_infinite_values_in_sight(ctx, gpu_device):
    """An infinite value with a logit like the others' makes the output infinite; a key of -inf logit counts for nothing."""
    torch = _torch()
    for dtype in ("bf16", "f32"):
        c = Cache(gpu_device, [100], 1, 64, 16, dtype, 6)
        q = _queries(2, 4, 64, dtype, gpu_device, 7).abs() + 0.5
        c.v[c.host_table[0, 20 // 16], 0, 20 % 16, 3] = float("inf")
        out, _ = _attend(ctx, c, q, [2], 4)
        o = out.double().cpu().numpy()
        assert np.all(np.isposinf(o[:, :, 3])) and np.all(np.isfinite(np.delete(o, 3, axis=2)))
        c = Cache(gpu_device, [100], 1, 64, 16, dtype, 6)
        c.k[c.host_table[0, 1], 0, 4] = -float("inf")
        keep = [j for j in range(100) if j != 20]
        out, lse = _attend(ctx, c, q, [2], 4, causal=False)
        ref = po.attention(q.double().cpu().numpy(), c.row(c.k, 0)[:, keep], c.row(c.v, 0)[:, keep], 0.125, False)
        _check(out, lse, ref, 64, 100, dtype, "-inf")


def test_attention_repeats_itself_on_other_streams_and_in_graphs(ctx, gpu_device):
    torch = _torch()
    lens, n_q = [900, 33, 1500, 2], [1, 2, 3, 1]
    c = Cache(gpu_device, lens, 2, 128, 16, "bf16", 8)
    q = _queries(sum(n_q), 8, 128, "bf16", gpu_device, 9)
    want, want_l = _attend(ctx, c, q, n_q, 8)
    cu = _ints(np.concatenate([[0], np.cumsum(n_q)]), gpu_device)
    out, lse = torch.empty_like(want), torch.empty_like(want_l)
    a = asl.make_attn(4, sum(n_q), 3, 1500)
    p = c.desc(8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.asl_paged_attention(p, a, q, c.k, c.v, c.table, c.kv_len, cu, out, lse=lse)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_l)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.asl_paged_attention(p, a, q, c.k, c.v, c.table, c.kv_len, cu, out, lse=lse)
    for i in range(4):
        q.copy_(_queries(sum(n_q), 8, 128, "bf16", gpu_device, 20 + i))
        c.kv_len[0] = c.lens[0] = 700 + 50 * i               # lengths that go on between replays
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got, got_l = out.clone(), lse.clone()
        eager, eager_l = _attend(ctx, c, q, n_q, 8)
        assert torch.equal(got, eager) and torch.equal(got_l, eager_l)
        _check(got, got_l, _oracle(c, q, n_q), 128, 1500, "bf16", "replay %d" % i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_numbers_out_of_range_are_left_out(ctx, gpu_device, dtype):
    """Page numbers, rows and lengths out of range: no access, the fault word's bit 1, and every other row as ever."""
    torch = _torch()
    lens, n_q = [200, 100, 60, 300], [1, 1, 2, 40]
    for what in ("page", "row", "length", "negative"):
        c = Cache(gpu_device, lens, 2, 64, 16, dtype, 10)
        q = _queries(sum(n_q), 4, 64, dtype, gpu_device, 11)
        want = _oracle(c, q, n_q)
        rows = [0, 1, 2, 3]
        if what == "page":
            c.table[1, 2] = c.n_pages
            c.table[3, 1] = -7
        elif what == "row":
            rows = [0, 4, 2, -1]
        else:
            c.kv_len[1] = c.kv_len[3] = -1 if what == "negative" else c.width * 16 + 1
        out, lse = _attend(ctx, c, q, n_q, 4, rows=rows)
        assert ctx.asl_device_fault() == 2, what
        ok = [0, 2, 3]                                        # tokens of the sequences 0 and 2
        tol, _ = _bounds(64, 300, dtype, want)
        o = out.double().cpu().numpy()
        assert np.all(np.abs(o[ok] - want[0][ok]) <= tol[ok]), what
        if what == "page":                                    # as if the page's tokens were not there
            keep = [j for j in range(100) if not 32 <= j < 48]
            ref = po.attention(q[1:2].double().cpu().numpy(), _without(c, c.k, 1, keep),
                               _without(c, c.v, 1, keep), 0.125, False)
            _check(out[1:2], lse[:, 1:2], ref, 64, 100, dtype, what)
        else:
            assert np.all(o[1] == 0) and np.all(lse[:, 1].cpu().numpy() == -np.inf)


def _without(c, x, r, keep):
    pages = c.host_table[r].copy()
    return po.gather(x.double().cpu().numpy(), np.where(pages < 0, 0, pages), c.lens[r])[:, keep]


# --------------------------------------------------------------------------------------------------------- pages
def _same_pages(got, want, what):
    assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True), what


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,d,ps,gap", [(1, 8, 16, 0), (2, 64, 16, 16), (8, 128, 64, 0), (3, 80, 32, 8), (2, 256, 128, 0)])
def test_write_appends(ctx, gpu_device, Hk, d, ps, gap, dtype):
    torch = _torch()
    lens, counts = [1, 16, 17, 64, 200, 130, 5], [1, 3, 17, 0, 150, 1, 5]
    c = Cache(gpu_device, lens, Hk, d, ps, dtype, 1, gap=gap)
    total = sum(counts)
    g = torch.Generator().manual_seed(5)
    cu = _ints(np.concatenate([[0], np.cumsum(counts)]), gpu_device)
    rows = _ints(list(range(7)), gpu_device)
    for order in ("tokens first", "heads first"):
        k, v = (torch.randn((total, Hk, d), generator=g).to(_dt(dtype)).to(gpu_device).transpose(0, 1) for _ in range(2))
        if order == "heads first":
            k, v = k.contiguous(), v.contiguous()
        wk, wv = c.k.double().cpu().numpy(), c.v.double().cpu().numpy()
        for want, x in ((wk, k), (wv, v)):
            po.write(want, c.host_table, lens, range(7), counts, np.split(x.double().cpu().numpy(), np.cumsum(counts)[:-1], axis=1))
        ctx.asl_pages_write(c.desc(), k, v, rows, cu, 7, total, c.table, c.kv_len, c.k, c.v)
        _same_pages(c.k, wk, order)
        _same_pages(c.v, wv, order)
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("idx_rows", [1, "Hk"])
@pytest.mark.parametrize("n_src,keep", [(5, 5), (700, 33), (3000, 1000), (9000, 2080)])
def test_write_selected(ctx, gpu_device, n_src, keep, idx_rows, dtype):
    torch = _torch()
    Hk, d, ps = 3, 64, 64
    c = Cache(gpu_device, [keep, 10], Hk, d, ps, dtype, 2)
    rng = np.random.default_rng(n_src)
    idx = np.stack([np.sort(rng.permutation(n_src)[:keep]) for _ in range(1 if idx_rows == 1 else Hk)])
    k, v = (torch.from_numpy(rng.standard_normal((Hk, n_src + 1, d), dtype=np.float32)).to(gpu_device).to(_dt(dtype))[:, 1:] for _ in range(2))
    want = []
    for x, pages in ((k, c.k), (v, c.v)):
        w, full = pages.double().cpu().numpy(), x.double().cpu().numpy()
        po.write(w, c.host_table, c.lens, [0], [keep], [np.stack([full[h, idx[h % len(idx)] if len(idx) > 1 else idx[0]] for h in range(Hk)])])
        want.append(w)
    ctx.asl_pages_write(c.desc(), k, v, _ints([0], gpu_device), _ints([0, keep], gpu_device), 1, keep, c.table, c.kv_len, c.k, c.v,
                        idx=_ints(idx, gpu_device))
    _same_pages(c.k, want[0], "k")
    _same_pages(c.v, want[1], "v")
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,d,ps,idx_rows", [(2, 64, 16, "Hk"), (8, 128, 64, 1), (3, 80, 32, "Hk")])
def test_compact(ctx, gpu_device, Hk, d, ps, idx_rows, dtype):
    lens, counts = [500, 1, 130, 77], [200, 1, 64, 0]
    c = Cache(gpu_device, lens + counts, Hk, d, ps, dtype, 3, gap=16)
    rng = np.random.default_rng(4)
    heads = 1 if idx_rows == 1 else Hk
    idx = np.concatenate([np.stack([np.sort(rng.permutation(n)[:m]) for _ in range(heads)]) for n, m in zip(lens, counts)], axis=1)
    cum = np.concatenate([[0], np.cumsum(counts)])
    want = []
    for pages in (c.k, c.v):
        w = pages.double().cpu().numpy()
        vals = []
        for i, n in enumerate(lens):
            full, sel = po.gather(w, c.host_table[i], n), idx[:, cum[i]:cum[i + 1]]
            vals.append(np.stack([full[h, sel[h if heads > 1 else 0]] for h in range(Hk)]))
        po.write(w, c.host_table, c.lens, [4, 5, 6, 7], counts, vals)
        want.append(w)
    ctx.asl_pages_compact(c.desc(), _ints([0, 1, 2, 3], gpu_device), _ints([4, 5, 6, 7], gpu_device), _ints(cum, gpu_device), 4,
                          sum(counts), _ints(idx, gpu_device), c.table, c.kv_len, c.k, c.v)
    _same_pages(c.k, want[0], "k")
    _same_pages(c.v, want[1], "v")
    assert ctx.asl_device_fault() == 0


def test_write_and_compact_leave_out_what_is_out_of_range(ctx, gpu_device):
    torch = _torch()
    c = Cache(gpu_device, [40, 40, 40], 2, 64, 16, "bf16", 5)
    k = torch.ones((2, 30, 64), dtype=torch.bfloat16, device=gpu_device)
    cu, before = _ints([0, 10, 20, 30], gpu_device), c.k.clone()

    def write(rows=(0, 1, 2), cu=cu, idx=None, table=c.table, kv=c.kv_len):
        c.k.copy_(before)
        ctx.asl_pages_write(c.desc(), k, k, _ints(rows, gpu_device), cu, 3, 30, table, kv, c.k, c.v, idx=idx)
        assert ctx.asl_device_fault() == 2
        return c.k

    got = write(rows=(0, 7, -1))
    changed = (got != before).any(dim=3).any(dim=1) & ~torch.isnan(before).any(dim=3).any(dim=1)
    assert int(changed.sum()) == 10                           # row 0's ten tokens
    write(idx=_ints([[30] * 15 + [-1] * 15], gpu_device))
    write(cu=_ints([0, 50, 50, 50], gpu_device))              # more tokens than the row has
    write(cu=_ints([9, 3, 20, 12], gpu_device))
    write(kv=_ints([-1, 2 ** 30, 40], gpu_device))
    write(table=torch.full_like(c.table, 10 ** 6))
    assert torch.equal(torch.isnan(c.k), torch.isnan(before)) and torch.equal(c.k.nan_to_num(), before.nan_to_num())
    c.k.copy_(before)
    ctx.asl_pages_compact(c.desc(), _ints([0, 9, 1], gpu_device), _ints([2, 2, 2], gpu_device), cu, 3, 30,
                          _ints([[40] * 10 + [0] * 10 + [-3] * 10], gpu_device), c.table, c.kv_len, c.k, c.v)
    assert ctx.asl_device_fault() == 2
    assert torch.equal(c.k.nan_to_num(), before.nan_to_num())


def _books(c):
    return c.host_table.copy(), np.array(c.lens, dtype=np.int64), c.refs_host.copy()


def _same_books(c, table, kv, refs, what):
    got = c.table.cpu().numpy()
    assert np.array_equal(c.kv_len.cpu().numpy(), kv), what
    assert np.array_equal(c.refs.cpu().numpy(), refs), what
    for r, n in enumerate(kv):
        m = -(-int(n) // c.ps)
        assert np.array_equal(got[r, :m], table[r, :m]), (what, r)


@pytest.mark.parametrize("spare,n_rows", [(400, 300), (20, 300), (0, 5), (3000, 40)])
def test_grow(ctx, gpu_device, spare, n_rows):
    rng = np.random.default_rng(spare + n_rows)
    c = Cache(gpu_device, [int(x) for x in rng.integers(0, 70, n_rows)], 1, 8, 16, "bf16", 1, row_stride=40, spare=spare)
    table, kv, refs = _books(c)
    for step in range(3):
        rows = rng.permutation(n_rows)[:rng.integers(1, n_rows + 1)]
        add = rng.integers(0, 60, rows.size)
        po.grow(table, kv, refs, rows, add, 16)
        ctx.asl_pages_grow(c.desc(), _ints(rows, gpu_device), _ints(add, gpu_device), rows.size, c.table, c.kv_len, c.refs)
        _same_books(c, table, kv, refs, "step %d" % step)
    assert ctx.asl_device_fault() == 0


def test_grow_takes_many_pages_of_a_large_pool(ctx, gpu_device):
    torch = _torch()
    n_pages = 100003
    rng = np.random.default_rng(0)
    refs = (rng.random(n_pages) < 0.7).astype(np.int64)
    table, kv = np.full((3, 20000), -1, dtype=np.int64), np.zeros(3, dtype=np.int64)
    p = asl.make_pages(1, 1, 8, 16, n_pages, 3, 20000)
    t, l, f = _ints(table, gpu_device), _ints(kv, gpu_device), _ints(refs, gpu_device)
    add = [16 * 15001 + 1, 16 * 19000, 7]                     # the second does not fit, the third is behind it
    ctx.asl_pages_grow(p, _ints([2, 0, 1], gpu_device), _ints(add, gpu_device), 3, t, l, f)
    po.grow(table, kv, refs, [2, 0, 1], add, 16)
    assert np.array_equal(l.cpu().numpy(), kv) and np.array_equal(f.cpu().numpy(), refs) and kv[0] == 0 and kv[2] > 0
    assert np.array_equal(t.cpu().numpy()[2, :15002], table[2, :15002])
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps,spare,layers", [(16, 60, 2), (64, 60, 1), (16, 4, 3), (32, 0, 1)])
def test_fork_and_free(ctx, gpu_device, ps, spare, layers, dtype):
    torch = _torch()
    rng = np.random.default_rng(ps + spare)
    lens = [200, 1, 64, 0, 130, 33] + [0] * 24
    c = Cache(gpu_device, lens, 2, 40, ps, dtype, 2, row_stride=15, spare=spare, layers=layers, gap=8)
    ks, vs = c.pages_t[0::2], c.pages_t[1::2]
    kp, vp = (torch.tensor([x.data_ptr() for x in t], dtype=torch.int64, device=gpu_device) for t in (ks, vs))
    host = [(k.double().cpu().numpy(), v.double().cpu().numpy()) for k, v in zip(ks, vs)]
    table, kv, refs = _books(c)
    children = 6 + rng.permutation(24)[:17]
    parents = rng.integers(0, 6, 17)
    po.fork(table, kv, refs, host, parents, children)
    ctx.asl_pages_fork(c.desc(), kp, vp, layers, _ints(parents, gpu_device), _ints(children, gpu_device), 17, c.table, c.kv_len, c.refs)
    _same_books(c, table, kv, refs, "fork")
    for (hk, hv), k, v in zip(host, ks, vs):
        _same_pages(k, hk, "k")
        _same_pages(v, hv, "v")
    rows = np.concatenate([children[:9], [0, 4]])             # parents go while continuations still hold their pages
    po.free(table, kv, refs, rows, ps)
    ctx.asl_pages_free(c.desc(), _ints(rows, gpu_device), rows.size, c.table, c.kv_len, c.refs)
    _same_books(c, table, kv, refs, "free")
    rest = np.flatnonzero(kv > 0)
    if rest.size:
        ctx.asl_pages_free(c.desc(), _ints(rest, gpu_device), rest.size, c.table, c.kv_len, c.refs)
    assert int(c.refs.abs().sum()) == 0 and int(c.kv_len.abs().sum()) == 0
    assert ctx.asl_device_fault() == 0


def test_books_refuse_what_is_out_of_range(ctx, gpu_device):
    torch = _torch()

    def fresh():
        return Cache(gpu_device, [40, 20, 0, 0], 1, 8, 16, "bf16", 3, row_stride=5, spare=8)

    def faulted(c):
        assert ctx.asl_device_fault() == 2

    i = lambda *x: _ints(x, gpu_device)
    c = fresh()
    ctx.asl_pages_grow(c.desc(), i(0, 9, -1, 1, 2), i(1, 1, 1, -3, 81), 5, c.table, c.kv_len, c.refs)
    faulted(c)
    assert c.kv_len.tolist() == [41, 20, 0, 0]
    c = fresh()
    ctx.asl_pages_grow(c.desc(), i(2, 2), i(16, 16), 2, c.table, c.kv_len, c.refs)      # a row twice: once
    faulted(c)
    assert c.kv_len.tolist()[2] == 16 and int(c.refs.sum()) == int(c.refs_host.sum()) + 1
    c = fresh()
    ctx.asl_pages_fork(c.desc(), None, None, 0, i(0, 0, 0, 9, 0), i(2, 2, 1, 3, -1), 5, c.table, c.kv_len, c.refs)
    faulted(c)
    assert c.kv_len.tolist() == [40, 20, 40, 0] and int(c.refs.sum()) == int(c.refs_host.sum()) + 3
    c = fresh()
    ctx.asl_pages_free(c.desc(), i(0, 0, 7, -2), 4, c.table, c.kv_len, c.refs)
    faulted(c)
    assert c.kv_len.tolist() == [0, 20, 0, 0] and int(c.refs.sum()) == 2
    c = fresh()
    c.table[0, 1] = 1000
    c.refs[int(c.host_table[1, 0])] = 0                       # a page that nobody holds any more
    ctx.asl_pages_free(c.desc(), i(0, 1), 2, c.table, c.kv_len, c.refs)
    faulted(c)
    assert int(c.refs.min()) == 0 and int(c.refs[int(c.host_table[0, 1])]) == 1


def test_refusals_of_a_context(gpu_device):
    torch = _torch()
    c = Cache(gpu_device, [40, 20], 2, 64, 16, "bf16", 3)
    x = asl.Asl(2, 1, 1)
    q = _queries(2, 4, 64, "bf16", gpu_device, 1)

    def status(f):
        with pytest.raises(asl.AslError) as e:
            f()
        return e.value.status

    def attend(rows=None, **kw):
        _attend(x, c, q, [1, 1], 4, **kw)

    assert status(attend) == asl.ASL_ENOMEM                   # nothing reserved
    for limits, want in (((0, 1, 1), asl.ASL_EINVAL), ((1, 0, 1), asl.ASL_EINVAL), ((1, 1, 0), asl.ASL_EINVAL),
                         ((4097, 1, 1), asl.ASL_EUNSUPPORTED), ((1, 1, 257), asl.ASL_EUNSUPPORTED)):
        assert status(lambda: x.asl_paged_reserve(*limits)) == want
    x.asl_paged_reserve(1, 100, 64)
    assert status(attend) == asl.ASL_ENOMEM                   # two sequences
    x.asl_paged_reserve(2, 7, 64)
    assert status(attend) == asl.ASL_ENOMEM                   # eight query rows
    x.asl_paged_reserve(2, 8, 56)
    assert status(attend) == asl.ASL_ENOMEM                   # d = 64
    x.asl_paged_reserve(2, 8, 64)
    attend()
    k = torch.ones((2, 4, 64), dtype=torch.bfloat16, device=gpu_device)
    i = lambda *v: _ints(v, gpu_device)
    off = torch.ones(2 * 4 * 64 + 4, dtype=torch.bfloat16, device=gpu_device)[4:].view(2, 4, 64)       # 8 bytes off
    assert status(lambda: x.asl_pages_write(c.desc(), off, k, i(0), i(0, 4), 1, 4, c.table, c.kv_len, c.k, c.v)) == asl.ASL_EUNSUPPORTED
    assert status(lambda: x.asl_pages_write(c.desc(), k, k, i(0), i(0, 4), 1, -4, c.table, c.kv_len, c.k, c.v)) == asl.ASL_EINVAL
    assert status(lambda: x.asl_pages_write(c.desc(), k, k, i(0), i(0, 4), -1, 4, c.table, c.kv_len, c.k, c.v)) == asl.ASL_EINVAL
    three = torch.zeros((3, 4), dtype=torch.int32, device=gpu_device)
    assert status(lambda: x.asl_pages_write(c.desc(), k, k, i(0), i(0, 4), 1, 4, c.table, c.kv_len, c.k, c.v, idx=three)) == asl.ASL_EINVAL
    assert status(lambda: x.asl_pages_write(c.desc(), k, k, i(0), i(0, 4), 1, 4, c.table, c.kv_len, None, c.v)) == asl.ASL_EINVAL
    assert status(lambda: x.asl_pages_compact(c.desc(), None, i(0), i(0, 4), 1, 4, three[:1], c.table, c.kv_len, c.k, c.v)) == asl.ASL_EINVAL
    assert status(lambda: x.asl_pages_grow(c.desc(), i(0, 0, 0), i(0, 0, 0), 3, c.table, c.kv_len, c.refs)) == asl.ASL_ENOMEM
    assert status(lambda: x.asl_pages_fork(c.desc(), None, None, 1, i(0), i(1), 1, c.table, c.kv_len, c.refs)) == asl.ASL_EINVAL
    assert status(lambda: x.asl_pages_free(c.desc(), None, 1, c.table, c.kv_len, c.refs)) == asl.ASL_EINVAL
    p = c.desc()
    p.page_size = 24
    assert status(lambda: x.asl_pages_free(p, i(0), 1, c.table, c.kv_len, c.refs)) == asl.ASL_EUNSUPPORTED
    x.asl_pages_grow(c.desc(), i(0), i(0), 0, c.table, c.kv_len, c.refs)          # nothing to do
    assert x.asl_device_fault() == 0
    x.close()


def test_a_prompt_is_pruned_continued_and_decoded(ctx, gpu_device):
    """The calls together: the selected tokens into pages, four continuations, decoding steps in a graph, the end."""
    torch = _torch()
    Hq, Hk, d, ps, N, keep, dev = 8, 2, 64, 16, 600, 100, gpu_device
    g = torch.Generator().manual_seed(1)
    new = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).to(dev)
    k, v = new(Hk, N, d), new(Hk, N, d)
    idx = torch.stack([torch.randperm(N, generator=g)[:keep].sort().values for _ in range(Hk)]).to(torch.int32).to(dev)
    n_pages, n_rows, width = 64, 6, 16
    kp, vp = (torch.full((n_pages, Hk, ps, d), float("nan"), dtype=torch.bfloat16, device=dev) for _ in range(2))
    table, kv, refs = (torch.zeros(s, dtype=torch.int32, device=dev) for s in ((n_rows, width), (n_rows,), (n_pages,)))
    p = asl.make_pages(Hq, Hk, d, ps, n_pages, n_rows, width)
    i = lambda *x: _ints(x, dev)
    ctx.asl_pages_grow(p, i(0), i(keep), 1, table, kv, refs)
    ctx.asl_pages_write(p, k, v, i(0), i(0, keep), 1, keep, table, kv, kp, vp, idx=idx)
    ptr = lambda x: torch.tensor([x.data_ptr()], dtype=torch.int64, device=dev)
    rows = i(1, 2, 3, 4)
    kptr, vptr = ptr(kp), ptr(vp)
    ctx.asl_pages_fork(p, kptr, vptr, 1, i(0, 0, 0, 0), rows, 4, table, kv, refs)
    one, cu = i(1, 1, 1, 1), i(0, 1, 2, 3, 4)
    q, nk, nv = new(4, Hq, d), new(4, Hk, d), new(4, Hk, d)
    out, lse = torch.empty_like(q), torch.empty((Hq, 4), dtype=torch.float32, device=dev)
    a = asl.make_attn(4, 4, 1, 256, n_groups=1)
    gs, pl = i(0, 4), i(keep)

    def step():
        ctx.asl_pages_grow(p, rows, one, 4, table, kv, refs)
        ctx.asl_pages_write(p, nk.transpose(0, 1), nv.transpose(0, 1), rows, cu, 4, 4, table, kv, kp, vp)
        ctx.asl_paged_attention(p, a, q, kp, vp, table, kv, cu, out, lse=lse, rows=rows, group_start=gs, prefix_len=pl)

    step()
    hist_k = [[nk[b].clone()] for b in range(4)]
    hist_v = [[nv[b].clone()] for b in range(4)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    base_k = torch.stack([k[h, idx[h].long()] for h in range(Hk)])
    base_v = torch.stack([v[h, idx[h].long()] for h in range(Hk)])
    for t in range(20):
        q.copy_(new(4, Hq, d)), nk.copy_(new(4, Hk, d)), nv.copy_(new(4, Hk, d))
        graph.replay()
        torch.cuda.synchronize()
        for b in range(4):
            hist_k[b].append(nk[b].clone())
            hist_v[b].append(nv[b].clone())
        if t % 6 == 5:
            refs_ = []
            for b in range(4):
                K = torch.cat([base_k, torch.stack(hist_k[b], dim=1)], dim=1).double().cpu().numpy()
                V = torch.cat([base_v, torch.stack(hist_v[b], dim=1)], dim=1).double().cpu().numpy()
                refs_.append(po.attention(q[b:b + 1].double().cpu().numpy(), K, V, d ** -0.5, True))
            ref = tuple(np.concatenate([r[j] for r in refs_], axis=1 if j == 1 else 0) for j in range(4))
            _check(out, lse, ref, d, keep + t + 2, "bf16", "step %d" % t)
    assert kv.tolist() == [keep] + [keep + 21] * 4 + [0]
    ctx.asl_pages_free(p, i(0, 1, 2, 3, 4), 5, table, kv, refs)
    assert int(refs.abs().sum()) == 0 and int(kv.sum()) == 0
    assert ctx.asl_device_fault() == 0


# ----------------------------------------------------------------------------------------- more sequences, rows, jumps
@pytest.fixture(scope="module")
def wide(gpu_device):
    c = asl.Asl(2, 1, 1)
    c.asl_paged_reserve(4096, 1 << 17, 128)
    yield c
    assert c.asl_device_fault() == 0
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,groups", [(65, None), (130, [(64, 200), (66, 130)]), (700, None), (4096, None), (1500, [(3, 140)] * 500)])
def test_attention_of_many_sequences(wide, gpu_device, n, groups, dtype):
    """More sequences than a wavefront has lanes: each lane plans for several."""
    rng = np.random.default_rng(n)
    own = rng.integers(0 if groups is None else 3, 40, n)
    lens = [int(x) + (0 if groups is None else p) for x, p in
            zip(own, [0] * n if groups is None else [p for m, p in groups for _ in range(m)])]
    n_q = [int(x) for x in rng.integers(0 if groups is None else 1, 3, n)]
    _case(wide, gpu_device, lens, n_q, 4, 2, 64, 16, dtype, groups=groups, what="many sequences")


@pytest.mark.parametrize("n", [1024, 1025, 4096])
def test_pages_of_many_sequences(wide, gpu_device, n):
    """The most rows of a call, grown, written, compacted, continued and freed."""
    torch = _torch()
    rng = np.random.default_rng(n)
    dev, Hk, d, ps, half = gpu_device, 1, 8, 16, n // 2
    lens = [int(x) for x in rng.integers(0, 30, half)] + [0] * (n - half)
    c = Cache(dev, lens, Hk, d, ps, "bf16", 7, row_stride=6, spare=3 * n)
    table, kv, refs = _books(c)
    add = [int(x) for x in rng.integers(0, 20, n)]
    rows = rng.permutation(n)
    po.grow(table, kv, refs, rows, [add[r] for r in rows], ps)
    wide.asl_pages_grow(c.desc(), _ints(rows, dev), _ints([add[r] for r in rows], dev), n, c.table, c.kv_len, c.refs)
    _same_books(c, table, kv, refs, "grow")
    counts = [add[r] for r in rows]
    total = sum(counts)
    k = torch.randn((Hk, total, d)).to(torch.bfloat16).to(dev)
    want = c.k.double().cpu().numpy()
    po.write(want, table, kv, rows, counts, np.split(k.double().cpu().numpy(), np.cumsum(counts)[:-1], axis=1))
    cu = _ints(np.concatenate([[0], np.cumsum(counts)]), dev)
    wide.asl_pages_write(c.desc(), k, k, _ints(rows, dev), cu, n, total, c.table, c.kv_len, c.k, c.v)
    _same_pages(c.k, want, "write")
    wide.asl_pages_free(c.desc(), _ints(rows[:n - half], dev), n - half, c.table, c.kv_len, c.refs)
    po.free(table, kv, refs, rows[:n - half], ps)
    _same_books(c, table, kv, refs, "free")
    held = rows[n - half:]
    parents = held[rng.integers(0, half, n - half)]
    host = [(want, c.v.double().cpu().numpy())]
    po.fork(table, kv, refs, host, parents, rows[:n - half])
    ptr = lambda x: torch.tensor([x.data_ptr()], dtype=torch.int64, device=dev)
    wide.asl_pages_fork(c.desc(), ptr(c.k), ptr(c.v), 1, _ints(parents, dev), _ints(rows[:n - half], dev), n - half, c.table, c.kv_len,
                        c.refs)
    _same_books(c, table, kv, refs, "fork")
    _same_pages(c.k, host[0][0], "fork")
    # the last token of each held row into the last place of another, which is emptied and grown first
    m = min(half, n - half)
    dst = rows[:m]
    po.free(table, kv, refs, dst, ps)
    po.grow(table, kv, refs, dst, [1] * m, ps)
    wide.asl_pages_free(c.desc(), _ints(dst, dev), m, c.table, c.kv_len, c.refs)
    wide.asl_pages_grow(c.desc(), _ints(dst, dev), _ints([1] * m, dev), m, c.table, c.kv_len, c.refs)
    _same_books(c, table, kv, refs, "again")
    src = held[np.argsort(-kv[held], kind="stable")][:m]
    keep = [i for i in range(m) if kv[src[i]] > 0]
    src, dst = src[keep], dst[keep]
    pick = [int(kv[r]) - 1 for r in src]
    want = c.k.double().cpu().numpy()
    vals = [po.gather(want, table[r], int(kv[r]))[:, p:p + 1] for r, p in zip(src, pick)]
    po.write(want, table, kv, dst, [1] * len(dst), vals)
    wide.asl_pages_compact(c.desc(), _ints(src, dev), _ints(dst, dev), _ints(np.arange(len(dst) + 1), dev), len(dst), len(dst),
                           _ints([pick], dev), c.table, c.kv_len, c.k, c.v)
    _same_pages(c.k, want, "compact")
    assert wide.asl_device_fault() == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q", [8, 40])
@pytest.mark.parametrize("shared", [False, True])
def test_attention_logits_that_rise_by_leaps(ctx, gpu_device, shared, n_q, d):
    """The largest logit of a row grows by 100 nats and more from tile to tile, several times over the keys, for some rows."""
    torch = _torch()
    L = 700
    c = Cache(gpu_device, [L, L] if shared else [L], 1, d, 16, "bf16", 3, shared=[(0, 2, 640)] if shared else ())
    for r in range(len(c.lens)):
        for t, size in ((130, 4.0), (200, 8.0), (420, 16.0), (641, 24.0), (690, 32.0)):
            c.k[c.host_table[r, t // 16], 0, t % 16] = size
    G = 4
    q = _queries(n_q * len(c.lens), G, d, "bf16", gpu_device, 5, spread=0.5)
    q[::3] = q[::3].abs() * 2 + 1                             # these rows climb; the others see the same keys with logits of any sign
    n = [n_q] * len(c.lens)
    out, lse = _attend(ctx, c, q, n, G, groups=[(2, 640)] if shared else None)
    _check(out, lse, _oracle(c, q, n), d, L, "bf16", "leaps")
    assert ctx.asl_device_fault() == 0


def test_the_example_from_prefill_to_decoding(gpu_device):
    """examples/serve_pruned.py: its attention and normalisers against the oracle, the scores it got from them against the
    scoring's own, its decoding steps over what it kept."""
    import importlib.util
    import os
    import gpu_util as gu
    from oracle import asl_oracle as orc
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_pruned.py")
    spec = importlib.util.spec_from_file_location("serve_pruned", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    Hq, Hk, d, N, W, n = 8, 2, 64, 1000, 16, 3
    r = example.run(Hq=Hq, Hk=Hk, d=d, N=N, W=W, budget=200, continuations=n, steps=6, page_size=16)
    assert r["fault"] == 0 and r["left"] == 0 and r["lengths"] == [0, 200] + [206] * n
    f = lambda x: x.double().cpu().numpy()
    q, k, v = f(r["q"]), f(r["k"]), f(r["v"])
    _check(r["out"], r["lse"], po.attention(q, k, v, d ** -0.5, True), d, N, "bf16", "window")
    ref = orc.get_ranks(q.transpose(1, 0, 2), k, v, W, 7, 200)
    gu.assert_scores_close(f(r["scores"][:Hk]), ref["P"], "scores by the attention's normalisers")
    idx = r["idx"].cpu().numpy()
    for b in range(n):
        for t, ((q1, _, _), out) in enumerate(zip(r["history"], r["outputs"])):
            K, V = (np.stack([np.concatenate([x[h][idx[h]], np.stack([f(step[1 + j][b])[h] for step in r["history"][:t + 1]])])
                              for h in range(Hk)]) for j, x in enumerate((k, v)))
            ref = po.attention(f(q1[b:b + 1]), K, V, d ** -0.5, True)
            tol, _ = _bounds(d, K.shape[1], "bf16", ref)
            assert np.all(np.abs(f(out[b:b + 1]) - ref[0]) <= tol), (b, t)


@pytest.mark.parametrize("kv", [600, 5000])
def test_lists_that_do_not_ascend_leave_no_trace(ctx, gpu_device, kv):
    """cu_q or group_start out of order: the fault word's bit 1, and the calls behind it (joined in the launch, or apart) as ever."""
    torch = _torch()
    c = Cache(gpu_device, [kv] * 8, 2, 64, 64, "bf16", 12)
    q = _queries(8, 8, 64, "bf16", gpu_device, 13)
    want, want_l = _attend(ctx, c, q, [1] * 8, 8)
    out, lse = torch.empty_like(want), torch.empty_like(want_l)
    for cu in ([0, 8, 0, 8, 0, 8, 0, 8, 8], [0, 5, 1, 7, 2, 8, 3, 8, 8], [-4, 1, 2, 3, 4, 5, 6, 7, 9], [8, 7, 6, 5, 4, 3, 2, 1, 0]):
        a = asl.make_attn(8, 8, 8, kv)
        ctx.asl_paged_attention(c.desc(8), a, q, c.k, c.v, c.table, c.kv_len, _ints(cu, gpu_device), out, lse=lse)
        assert ctx.asl_device_fault() == 2
        got, got_l = _attend(ctx, c, q, [1] * 8, 8)
        assert torch.equal(got, want) and torch.equal(got_l, want_l)
    for gs in ([0, 8, 0, 8], [3, 1, 9, 8], [-1, 2, 4, 8], [0, 2, 5, 100]):
        a = asl.make_attn(8, 8, 1, 10 ** 8, n_groups=3)
        ctx.asl_paged_attention(c.desc(8), a, q, c.k, c.v, c.table, c.kv_len, _ints(range(9), gpu_device), out, lse=lse,
                                group_start=_ints(gs, gpu_device), prefix_len=_ints([kv] * 3, gpu_device))
        ctx.asl_device_fault()
        got, got_l = _attend(ctx, c, q, [1] * 8, 8)
        assert torch.equal(got, want) and torch.equal(got_l, want_l)
    assert ctx.asl_device_fault() == 0


def test_calls_without_work(ctx, gpu_device):
    """No sequences, no tokens: nothing is read, nothing refused."""
    torch = _torch()
    c = Cache(gpu_device, [40, 20], 2, 64, 16, "bf16", 3)
    none, i = torch.empty(0, dtype=torch.int32, device=gpu_device), lambda *x: _ints(x, gpu_device)
    empty = torch.empty((2, 0, 64), dtype=torch.bfloat16, device=gpu_device)
    before, books = c.k.clone(), c.kv_len.clone()
    ctx.asl_pages_grow(c.desc(), none, none, 0, c.table, c.kv_len, c.refs)
    ctx.asl_pages_fork(c.desc(), None, None, 0, none, none, 0, c.table, c.kv_len, c.refs)
    ctx.asl_pages_free(c.desc(), none, 0, c.table, c.kv_len, c.refs)
    ctx.asl_pages_write(c.desc(), empty, empty, i(0), i(0, 0), 1, 0, c.table, c.kv_len, c.k, c.v)
    ctx.asl_pages_compact(c.desc(), i(0), i(1), i(0, 0), 1, 0, none.view(1, 0), c.table, c.kv_len, c.k, c.v)
    out, lse = _attend(ctx, c, _queries(0, 4, 64, "bf16", gpu_device, 1), [0, 0], 4)
    assert out.numel() == 0 and lse.numel() == 0
    assert torch.equal(c.k.nan_to_num(), before.nan_to_num()) and torch.equal(c.kv_len, books)
    assert ctx.asl_device_fault() == 0


def test_offsets_past_32_bits(ctx, gpu_device):
    """Pages beyond 4 GiB: grown, written, continued, compacted, attended to."""
    torch = _torch()
    Hq, Hk, d, ps, dev = 8, 2, 128, 64, gpu_device
    n_pages = (9 << 30) // (Hk * ps * d * 2) // 2 + 7                         # 4.5 GiB each of K and V
    kp, vp = (torch.empty((n_pages, Hk, ps, d), dtype=torch.bfloat16, device=dev) for _ in range(2))
    table, kv = torch.zeros((4, 8), dtype=torch.int32, device=dev), torch.zeros(4, dtype=torch.int32, device=dev)
    refs = torch.ones(n_pages, dtype=torch.int32, device=dev)
    refs[-20:] = 0
    refs[3] = 0                                               # one page at the beginning, the others at the end
    p = asl.make_pages(Hq, Hk, d, ps, n_pages, 4, 8)
    i = lambda *x: _ints(x, dev)
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((Hk, 200, d), generator=g).to(torch.bfloat16).to(dev) for _ in range(2))
    ctx.asl_pages_grow(p, i(0), i(200), 1, table, kv, refs)
    assert table[0, :4].tolist() == [3, n_pages - 20, n_pages - 19, n_pages - 18]
    ctx.asl_pages_write(p, k, v, i(0), i(0, 200), 1, 200, table, kv, kp, vp)
    ptr = lambda x: torch.tensor([x.data_ptr()], dtype=torch.int64, device=dev)
    kptr, vptr = ptr(kp), ptr(vp)
    ctx.asl_pages_fork(p, kptr, vptr, 1, i(0), i(1), 1, table, kv, refs)
    keep = [5, 70, 130, 190, 199]
    ctx.asl_pages_grow(p, i(2), i(5), 1, table, kv, refs)
    ctx.asl_pages_compact(p, i(1), i(2), i(0, 5), 1, 5, i(*keep).view(1, 5), table, kv, kp, vp)
    f = lambda x: x.double().cpu().numpy()
    for n_q in ([1, 1, 1], [40, 40, 3]):
        q = _queries(sum(n_q), Hq, d, "bf16", dev, 3)
        out, lse = torch.empty_like(q.contiguous()), torch.empty((Hq, sum(n_q)), dtype=torch.float32, device=dev)
        cu = np.concatenate([[0], np.cumsum(n_q)])
        for bound in (200, 1 << 20):                          # split items, tiles
            ctx.asl_paged_attention(p, asl.make_attn(3, sum(n_q), max(n_q), bound), q, kp, vp, table, kv, _ints(cu, dev), out, lse=lse)
            parts = [po.attention(f(q)[cu[b]:cu[b + 1]], f(k)[:, s], f(v)[:, s], d ** -0.5, True)
                     for b, s in enumerate((slice(None), slice(None), keep))]
            ref = tuple(np.concatenate([x[j] for x in parts], axis=1 if j == 1 else 0) for j in range(4))
            _check(out, lse, ref, d, 200, "bf16", "past 32 bits")
    assert ctx.asl_device_fault() == 0
