"""Drafting over the paged cache, as cases that can be timed and compared: a step that proposes a tree of tokens for each sequence, attends
over it and keeps one path.

Four operators, each through the calls that a serving program makes:

* ``rotate``: rotary positions of queries and keys, and the same with the keys and values going straight into the pages; rotating back is
  the gradient;
* ``plan``: from the number of new tokens of each request the pages that they need, and of each token its slot and its position;
* ``tree``: attention of drafted tokens, of which each sees its sequence's context and its own ancestors;
* ``accept``: of each sequence's draft the accepted path moves to the first of the draft's places, in every layer, and the rest is given back.

Positions are not places in the cache: pruning takes tokens out of a row, ``pruned[row]`` of them, and those behind keep their positions.
Pages are [n_pages, heads, page_size, d]; a sequence is a row of ``table`` (page numbers) and a length in ``kv_len``; a page with count 0 in
``refs`` is free.  With ``own`` false every operator is computed from its definition with elementary operations.
"""
import functools
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
DTYPE = {BF16: torch.bfloat16, F32: torch.float32}


# ---------------------------------------------------------------------------------------------------------------------
# cases

def listed():
    return [
        # the gradient of a rotation in the small fp32 model (4 query heads, 2 KV heads of 64), one prompt of 512 tokens
        dict(name="rotate back tiny fp32", op="rotate", dtype=F32, Hq=4, Hk=2, d=64, rot=64, pairs="halves", seqs=1, n=512, far=4096,
             scaling="plain", back=True, write=False, ps=16),
        # the prefill of 32768 tokens behind others, positions scaled by parts for a long context
        dict(name="rotate prefill 32K", op="rotate", dtype=BF16, Hq=32, Hk=8, d=128, rot=128, pairs="neighbours", seqs=3, n=32768,
             far=131072, scaling="parts", back=False, write=False, ps=64),
        # one decoding step of 64 requests at far positions, keys and values into their pages: latency
        dict(name="rotate write decode", op="rotate", dtype=BF16, Hq=32, Hk=8, d=128, rot=128, pairs="halves", seqs=64, n=64,
             far=1048576, scaling="linear", back=False, write=True, ps=16),
        # a chunk of two prompts into pages, second head geometry, half of each head rotated
        dict(name="rotate write chunk", op="rotate", dtype=BF16, Hq=28, Hk=4, d=128, rot=64, pairs="halves", seqs=2, n=4085,
             far=262144, scaling="base", back=False, write=True, ps=64),
        # 64 requests with a drafted tree each, behind pruned prompts, pages of 16
        dict(name="plan drafts", op="plan", seqs=64, add_lo=5, add_hi=32, old_lo=2049, old_hi=2548, ps=16, tree=True, spare=300, held=0.3),
        # 24 prompts admitted into a pool that others use too
        dict(name="plan prompts", op="plan", seqs=24, add_lo=500, add_hi=4000, old_lo=0, old_hi=0, ps=64, tree=False, spare=1600, held=0.5),
        # a small model in fp32, five short requests with small trees: latency
        dict(name="tree tiny fp32", op="tree", dtype=F32, Hq=4, Hk=2, d=64, ps=16, groups=5, members=1, prefix=0, ctx_lo=1, ctx_hi=500,
             n_lo=2, n_hi=9),
        # a serving batch whose prompts were pruned to the budget of 2048, trees of 16 to 32 nodes
        dict(name="tree pruned batch", op="tree", dtype=BF16, Hq=32, Hk=8, d=128, ps=64, groups=32, members=1, prefix=0, ctx_lo=2049,
             ctx_hi=2548, n_lo=16, n_hi=32),
        # one request, a tree of 60 nodes over a context that was not pruned, second head geometry
        dict(name="tree 128K", op="tree", dtype=BF16, Hq=28, Hk=4, d=128, ps=64, groups=1, members=1, prefix=0, ctx_lo=131089,
             ctx_hi=131089, n_lo=60, n_hi=60),
        # 8 prompts pruned to 2048 + window, 6 continuations of each that draft trees of 5 to 12 nodes, pages of 16
        dict(name="tree shared prompts", op="tree", dtype=BF16, Hq=28, Hk=4, d=128, ps=16, groups=8, members=6, prefix=2090, ctx_lo=6,
             ctx_hi=200, n_lo=5, n_hi=12),
        # 64 requests keep 1 to 6 of 16 to 32 nodes, 8 layers
        dict(name="accept batch", op="accept", dtype=BF16, Hk=8, d=128, ps=16, layers=8, seqs=64, n_lo=16, n_hi=32, keep_lo=1, keep_hi=6,
             old_lo=40, old_hi=250),
        # the small fp32 model, two layers, three requests: latency
        dict(name="accept tiny fp32", op="accept", dtype=F32, Hk=2, d=64, ps=16, layers=2, seqs=3, n_lo=5, n_hi=9, keep_lo=1, keep_hi=4,
             old_lo=1, old_hi=500),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, its logarithm uniform."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case; none costs more than the largest listed ones (fp32 products run at a sixteenth of bf16's rate)."""
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] <= 6e8 and w["flops"] <= (1.1e11 if c.get("dtype") != F32 else 7e9):
            return c


def _draw(rng):
    op = rng.choice(["rotate", "rotate", "plan", "tree", "tree", "accept"])
    dtype = rng.choice([BF16, BF16, BF16, F32])
    Hk = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 4, 7, 8])
    d = rng.choice([64, 80, 96, 128, 128, 128, 256])
    ps = rng.choice([16, 32, 64, 128, 256])
    if op == "rotate":
        write = rng.random() < 0.5
        n = _log(rng, 1, 20000)
        return dict(op=op, dtype=dtype, Hq=G * Hk, Hk=Hk, d=d, rot=rng.choice([d, d, d // 2, d // 4, d // 4 - 2]),
                    pairs=rng.choice(["halves", "neighbours"]), seqs=_log(rng, 1, min(n, 100)), n=n, far=n + _log(rng, 2000, 8000000),
                    scaling=rng.choice(["plain", "linear", "base", "parts"]), back=not write and rng.random() < 0.4, write=write, ps=ps)
    if op == "plan":
        tree = rng.random() < 0.6
        hi = _log(rng, 1, 64 if tree else 3000)
        return dict(op=op, seqs=_log(rng, 1, 300), add_lo=rng.choice([0, 1, max(1, hi // 2)]) if hi > 1 else 1, add_hi=hi,
                    old_lo=0, old_hi=_log(rng, 1, 3000), ps=ps, tree=tree, spare=_log(rng, 1, 2000), held=rng.choice([0.0, 0.3, 0.8]))
    if op == "tree":
        c = dict(op=op, dtype=dtype, Hq=G * Hk, Hk=Hk, d=d, ps=ps, groups=1, members=1, prefix=0, n_lo=1)
        kind = rng.choice(["batch", "long", "shared", "wide"])
        if kind == "batch":
            hi = _log(rng, 2, 4000)
            c |= dict(groups=_log(rng, 1, 48), ctx_lo=rng.choice([0, hi // 2]), ctx_hi=hi, n_hi=_log(rng, 2, 64))
        elif kind == "long":
            n = _log(rng, 4000, 60000)
            c |= dict(groups=rng.choice([1, 2]), ctx_lo=n - 99, ctx_hi=n, n_hi=_log(rng, 1, 64))
        elif kind == "shared":
            c |= dict(groups=rng.choice([1, 1, 2, 5]), members=_log(rng, 2, 16), prefix=_log(rng, 50, 6000), ctx_lo=0,
                      ctx_hi=_log(rng, 6, 300), n_hi=_log(rng, 1, 30))
        else:
            hi = _log(rng, 60, 400)
            c |= dict(groups=rng.choice([1, 2, 4]), ctx_lo=0, ctx_hi=_log(rng, 20, 4000), n_lo=hi // 2, n_hi=hi)
        return c
    hi = _log(rng, 1, 64)
    keep = _log(rng, 1, min(hi, 12))
    return dict(op=op, dtype=dtype, Hk=Hk, d=d, ps=ps, layers=_log(rng, 1, 8), seqs=_log(rng, 1, 64), n_lo=max(1, hi // 2), n_hi=hi,
                keep_lo=rng.choice([0, 1]), keep_hi=keep, old_lo=0, old_hi=_log(rng, 1, 300))


# ---------------------------------------------------------------------------------------------------------------------
# inputs

class _Lengths:
    """The whole numbers of a case. The lengths are the case's own, so that tensors of any seed have the same shapes; which
    sequence has which is the seed's."""

    def __init__(self, c, seed):
        fixed = torch.Generator().manual_seed(13)
        op = c["op"]
        n = c["groups"] * c["members"] if op == "tree" else c["seqs"]
        order = torch.randperm(n, generator=torch.Generator().manual_seed(7 * int(seed) + 1)).tolist()

        def between(lo, hi):
            x = torch.randint(lo, hi + 1, (n,), generator=fixed).tolist()
            return [x[i] for i in order]

        self.rows = n
        if op == "rotate":                                       # n tokens in `seqs` runs
            cut = sorted(torch.randint(0, c["n"] - n + 1, (n - 1,), generator=fixed).tolist())
            cut = [0] + [x + i + 1 for i, x in enumerate(cut)] + [c["n"]]
            self.n = [b - a for a, b in zip(cut, cut[1:])]
            self.n = [self.n[i] for i in order]
            self.old = between(0, 40)
        elif op == "tree":
            self.n = between(c["n_lo"], c["n_hi"])
            self.old = [c["prefix"] + x for x in between(c["ctx_lo"], c["ctx_hi"])]
        elif op == "accept":
            self.n, self.old = between(c["n_lo"], c["n_hi"]), between(c["old_lo"], c["old_hi"])
            self.keep = [min(a, b) for a, b in zip(between(c["keep_lo"], c["keep_hi"]), self.n)]
        else:
            self.n, self.old = between(c["add_lo"], c["add_hi"]), between(c["old_lo"], c["old_hi"])
        self.kv = [a + b for a, b in zip(self.n, self.old)]
        self.pages = [-(-x // c["ps"]) for x in self.kv]
        self.old_pages = [-(-x // c["ps"]) for x in self.old]


def _cumulative(counts):
    out = [0]
    for x in counts:
        out.append(out[-1] + x)
    return out


def _freqs(c):
    """Radians that a position adds to the angle of each pair, and the factor of cos and sin."""
    r = c["rot"]
    i = torch.arange(r // 2, dtype=torch.float64)
    f = 10000.0 ** (-2.0 * i / r)
    s = 8.0
    if c["scaling"] == "linear":
        return f / s, 1.0
    if c["scaling"] == "base":
        return (10000.0 * s ** (r / max(r - 2.0, 1.0))) ** (-2.0 * i / r), 1.0
    if c["scaling"] == "parts":                                  # pairs of many turns over the first 8192 positions stay as they are
        keep = ((8192.0 * f / (2.0 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return f * (keep + (1.0 - keep) / s), 0.1 * math.log(s) + 1.0
    return f, 1.0


def _draft(n, gen):
    """Each node's parent among the draft's nodes, an earlier one, or -1: some chains, some branches."""
    r = torch.rand((n, 2), generator=gen).tolist()
    return [-1 if i == 0 or a < 0.03 else i - 1 if a < 0.45 else int(b * i) for i, (a, b) in enumerate(r)]


def _inputs(c, seed):
    dev, ps, op = "cuda", c["ps"], c["op"]
    ln = _Lengths(c, seed)
    host = torch.Generator().manual_seed(7 * int(seed) + 2)
    g = torch.Generator(device=dev).manual_seed(7 * int(seed) + 3)

    def ints(v, dtype=torch.int32):
        return torch.tensor(v, dtype=dtype).to(dev)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(DTYPE[c["dtype"]])

    s = dict(c, lens=ln, total=sum(ln.n))
    if op == "rotate":
        n, Hq, Hk, d = c["n"], c["Hq"], c["Hk"], c["d"]
        start = [int(x * (c["far"] - m)) for x, m in zip(torch.rand(len(ln.n), generator=host, dtype=torch.float64).tolist(), ln.n)]
        s["pos"] = torch.cat([torch.arange(a, a + m) for a, m in zip(start, ln.n)]).to(torch.int32).to(dev)
        f, s["magnitude"] = _freqs(c)
        s["freqs"] = f.to(dev)
        x = normal(n, Hq + 2 * Hk, d)                            # what one projection leaves
        s |= dict(q=x[:, :Hq], k=x[:, Hq:Hq + Hk], v=x[:, Hq + Hk:])
        s["q_out"] = torch.empty((n, Hq, d), dtype=x.dtype, device=dev)
        if not c["write"]:
            s["k_out"] = torch.empty((n, Hk, d), dtype=x.dtype, device=dev)
            return s
    # a cache in use: no row's pages are neighbours
    width = max(ln.pages) + 1                                    # entries of a table row
    shared = c["prefix"] // ps if op == "tree" and c["members"] > 1 else 0    # pages that a group's rows have in common
    held = ln.old_pages if op == "plan" else [p - shared for p in ln.pages]
    used = sum(held) + (shared * c["groups"] if shared else 0)
    if op == "plan":
        n_pages = used + int((c["spare"] + 1) / (1.0 - c["held"])) + 1     # others hold a part of the rest
    else:
        n_pages = used + 3
    order = torch.randperm(n_pages, generator=host, dtype=torch.int64).tolist()
    table = torch.full((ln.rows, width), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(held):
        if shared:
            if r % c["members"] == 0:
                first = order[at:at + shared]
                at += shared
            table[r, :shared] = torch.tensor(first, dtype=torch.int32)
        table[r, shared:shared + n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[torch.tensor(order[:used], dtype=torch.int64)] = 1
    if op == "plan":
        refs[torch.tensor(order[used:n_pages - c["spare"]], dtype=torch.int64)] = 1
    # counts and lengths are one buffer, so that a pass begins by putting both back with one copy
    s["book_before"] = torch.cat([refs, torch.tensor(ln.old if op == "plan" else ln.kv, dtype=torch.int32)]).to(dev)
    s["book"] = s["book_before"].clone()
    s |= dict(n_pages=n_pages, width=width, table=table.to(dev), refs=s["book"][:n_pages], kv_len=s["book"][n_pages:],
              cu=ints(_cumulative(ln.n)), rows=ints(list(range(ln.rows))))
    if op == "rotate":
        s["k_pages"], s["v_pages"] = normal(n_pages, Hk, ps, d), normal(n_pages, Hk, ps, d)
        slots = []
        for r, (a, m) in enumerate(zip(ln.old, ln.n)):
            t = torch.arange(a, a + m)
            slots.append(table[r].long()[t // ps] * ps + t % ps)
        s["slot"] = torch.cat(slots).to(dev)
    elif op == "plan":
        s |= dict(add=ints(ln.n), pruned=ints(torch.randint(0, 100000, (ln.rows,), generator=host).tolist()),
                  cu_out=torch.empty(ln.rows + 1, dtype=torch.int32, device=dev), slot=torch.empty(s["total"], dtype=torch.int64, device=dev),
                  pos=torch.empty(s["total"], dtype=torch.int32, device=dev))
        s["parent"] = ints(sum((_draft(m, host) for m in ln.n), [])) if c["tree"] else None
    elif op == "tree":
        s["k_pages"], s["v_pages"] = normal(n_pages, c["Hk"], ps, c["d"]), normal(n_pages, c["Hk"], ps, c["d"])
        s["parent"] = ints(sum((_draft(m, host) for m in ln.n), []))
        s |= dict(group_start=ints(_cumulative([c["members"]] * c["groups"])), prefix_len=ints([shared * ps] * c["groups"]))
        s["q"] = normal(s["total"], c["Hq"], c["d"]) * 2         # logits with a spread of 2: some tokens stand out
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((c["Hq"], s["total"]), dtype=torch.float32, device=dev)
    else:
        s["k_pages"], s["v_pages"] = normal(c["layers"], n_pages, c["Hk"], ps, c["d"]), normal(c["layers"], n_pages, c["Hk"], ps, c["d"])
        s["k_ptrs"] = torch.tensor([x.data_ptr() for x in s["k_pages"]], dtype=torch.int64).to(dev)
        s["v_ptrs"] = torch.tensor([x.data_ptr() for x in s["v_pages"]], dtype=torch.int64).to(dev)
        most = max(ln.keep + [1])
        path = torch.zeros((ln.rows, most), dtype=torch.int32)
        for r, (m, a) in enumerate(zip(ln.n, ln.keep)):
            # a path's nodes: the first as they stand, those behind a branch from behind the accepted places, so that a second pass finds
            # the cache as the first one left it
            stay = int(torch.randint(0, a + 1, (1,), generator=host))
            rest = torch.randperm(m - a, generator=host)[:a - stay].sort().values + a
            stay = a - len(rest)
            path[r, :a] = torch.cat([torch.arange(stay), rest]).to(torch.int32)
        s |= dict(path=path.to(dev), n_path=ints(ln.keep))
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# ---------------------------------------------------------------------------------------------------------------------
# the operators from their definitions

def _plain_turn(s, x):
    """The pairs of x's first elements turned by their positions' angles; angles in 64 bits."""
    r = s["rot"]
    t = s["pos"].double()[:, None] * s["freqs"]
    cos, sin = (t.cos() * s["magnitude"]).float()[:, None], (t.sin() * s["magnitude"]).float()[:, None]
    if s["back"]:
        sin = -sin
    x = x.float()
    if s["pairs"] == "halves":
        a, b = x[..., :r // 2], x[..., r // 2:r]
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
    a, b = a * cos - b * sin, a * sin + b * cos
    y = torch.cat([a, b], dim=-1) if s["pairs"] == "halves" else torch.stack([a, b], dim=-1).flatten(-2)
    return torch.cat([y, x[..., r:]], dim=-1).to(s["q"].dtype)


def _plain_rotate(s):
    q, k = _plain_turn(s, s["q"]), _plain_turn(s, s["k"])
    if not s["write"]:
        return q, k
    page, at = s["slot"] // s["ps"], s["slot"] % s["ps"]
    s["k_pages"][page, :, at] = k
    s["v_pages"][page, :, at] = s["v"]
    return q, s["k_pages"], s["v_pages"]


def _ancestors(s, parent):
    """[sequences, most, most]: whether node j is node i or an ancestor of it; by squaring, since a path has at most `most` steps."""
    cu, dev = s["cu"].long(), parent.device
    most = max(max(s["lens"].n), 1)
    n = cu[1:] - cu[:-1]
    i = torch.arange(most, device=dev)
    there = i < n[:, None]
    p = parent.long()[(cu[:-1, None] + i).clamp(max=max(s["total"] - 1, 0))]
    step = ((i[None, None] == p[:, :, None]) | (i[None, None] == i[None, :, None])) & there[:, :, None]
    a = step.float()
    for _ in range(max(1, (most - 1).bit_length())):
        a = (torch.matmul(a, a) > 0).float()
    return a > 0


def _plain_plan(s):
    s["book"].copy_(s["book_before"])
    table, kv, refs, ps = s["table"], s["kv_len"], s["refs"], s["ps"]
    r, add = s["rows"].long(), s["add"].long()
    old = kv[r].long()
    have, want = (old + ps - 1) // ps, (old + add + ps - 1) // ps
    need = want - have
    upto = need.cumsum(0)
    fits = upto <= (refs == 0).sum()
    free = torch.argsort((refs != 0).int(), stable=True)
    t = torch.arange(table.shape[1], device=table.device)
    new = (t >= have[:, None]) & (t < want[:, None]) & fits[:, None]
    number = (upto - need)[:, None] + t - have[:, None]
    fresh = free[number.clamp(0, free.numel() - 1)]
    table[r] = torch.where(new, fresh.int(), table[r])
    refs.index_add_(0, torch.where(new, fresh, 0).reshape(-1), new.int().reshape(-1))
    kv[r] = torch.where(fits, old + add, old).int()
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device=kv.device), add.cumsum(0)])
    j = torch.arange(s["total"], device=kv.device)
    seq = torch.searchsorted(cu[1:], j, right=True)
    i = j - cu[seq]
    at = old[seq] + i
    slot = table[r[seq], (at // ps).clamp(max=table.shape[1] - 1)].long() * ps + at % ps
    slot = torch.where(fits[seq], slot, -1)
    if s["parent"] is not None:
        i = _ancestors(s, s["parent"]).sum(dim=2)[seq, i] - 1
    pos = old[seq] + i + s["pruned"].long()[r[seq]]
    return table, kv, refs, cu.int(), slot, pos.int()


def _plain_tree(s):
    """softmax(scale q K^T) V over each node's context and ancestors, all sequences padded to the longest; log-sum-exp of each row."""
    Hq, Hk, d, ps = s["Hq"], s["Hk"], s["d"], s["ps"]
    B, G, dev = s["lens"].rows, s["Hq"] // s["Hk"], s["q"].device
    kv, cu = s["kv_len"].long(), s["cu"].long()
    n = cu[1:] - cu[:-1]
    most_q, most_kv = max(max(s["lens"].n), 1), max(s["lens"].kv)
    pages = s["table"].long().clamp(min=0)[:, :-(-most_kv // ps)]
    k = s["k_pages"][pages].float().transpose(1, 2).reshape(B, Hk, -1, d)
    v = s["v_pages"][pages].float().transpose(1, 2).reshape(B, Hk, -1, d)
    i = torch.arange(most_q, device=dev)
    q = s["q"][(cu[:-1, None] + i).clamp(max=s["total"] - 1)].float()                         # [B, i, Hq, d]
    q = q.reshape(B, most_q, Hk, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hk, most_q * G, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(d ** -0.5)                                    # [B, Hk, i * G, keys]
    j = torch.arange(k.shape[2], device=dev) - (kv - n)[:, None]                              # a key's node, if there is one
    anc = _ancestors(s, s["parent"])
    seen = anc.gather(2, j.clamp(0, most_q - 1)[:, None].expand(B, most_q, -1)) & (j < n[:, None])[:, None]
    seen = torch.where((j < 0)[:, None], torch.ones_like(seen), seen)
    x.masked_fill_(~seen.repeat_interleave(G, dim=1)[:, None], -math.inf)
    top = x.amax(dim=3, keepdim=True).clamp(min=-3.0e38)
    p = x.sub_(top).exp_()
    z = p.sum(dim=3, keepdim=True)
    o = torch.matmul(p, v) / z.clamp(min=1e-38)
    lse = (top + z.log()).squeeze(3)
    tok = torch.arange(s["total"], device=dev)
    seq = torch.searchsorted(cu[1:], tok, right=True)
    o = o.reshape(B, Hk, most_q, G, d).permute(0, 2, 1, 3, 4).reshape(B, most_q, Hq, d)
    lse = lse.reshape(B, Hk, most_q, G).permute(0, 2, 1, 3).reshape(B, most_q, Hq)
    at = (seq, tok - cu[seq])
    return o[at].to(s["q"].dtype), lse[at].t().contiguous()


def _plain_accept(s):
    s["book"].copy_(s["book_before"])
    table, kv, refs, ps = s["table"].long(), s["kv_len"], s["refs"], s["ps"]
    r, cu, path = s["rows"].long(), s["cu"].long(), s["path"].long()
    L, a = kv[r].long(), s["n_path"].long()
    base = L - (cu[1:] - cu[:-1])
    t = torch.arange(path.shape[1], device=kv.device)
    kept = t < a[:, None]
    src, dst = base[:, None] + torch.where(kept, path, 0), base[:, None] + torch.where(kept, t, 0)   # (others: node 0 onto itself)
    last = table.shape[1] - 1
    from_page, to_page = table[r[:, None], (src // ps).clamp(max=last)], table[r[:, None], (dst // ps).clamp(max=last)]
    src_at, dst_at = src % ps, dst % ps
    first = path[:, :1] == 0                                     # (node 0 is moved onto: its new value for the others too)
    for x in (s["k_pages"], s["v_pages"]):
        moved = x[:, from_page, :, src_at]                       # [sequences, path, layers, heads, d]
        moved = torch.where((kept | first)[:, :, None, None, None], moved, moved[:, :1])
        x[:, to_page, :, dst_at] = moved
    have, want = (L + ps - 1) // ps, (base + a + ps - 1) // ps
    e = torch.arange(table.shape[1], device=kv.device)
    gone = (e >= want[:, None]) & (e < have[:, None])
    refs.index_add_(0, torch.where(gone, table[r], 0).reshape(-1), -gone.int().reshape(-1))
    kv[r] = (base + a).int()
    return kv, refs, s["k_pages"], s["v_pages"]


# ---------------------------------------------------------------------------------------------------------------------
# the framework's calls

@functools.lru_cache(maxsize=None)
def _handle(seqs, query_rows, d):
    """The program's context, made once for the largest call that it makes."""
    from paper_2601_07667_amd import asl
    ctx = asl.Asl(2, 1, 1)
    ctx.asl_paged_reserve(seqs, query_rows, d)
    return ctx


def _ctx():
    return _handle(512, 1 << 18, 256)


@functools.lru_cache(maxsize=None)
def _layout(*sizes, dtype):
    from paper_2601_07667_amd import asl
    return asl.make_pages(*sizes, dtype=asl.ASL_F32 if dtype == F32 else asl.ASL_BF16)


@functools.lru_cache(maxsize=None)
def _rotation(Hq, Hk, d, rot, pairs, dtype, magnitude, back):
    from paper_2601_07667_amd import asl
    return asl.make_rotation(Hq, Hk, d, rot, pairs=asl.ASL_PAIRS_HALVES if pairs == "halves" else asl.ASL_PAIRS_NEIGHBOURS,
                             dtype=asl.ASL_F32 if dtype == F32 else asl.ASL_BF16, magnitude=magnitude, back=back)


@functools.lru_cache(maxsize=None)
def _batch(n_seqs, total_q, max_q_len, max_kv_len, n_groups):
    from paper_2601_07667_amd import asl
    return asl.make_attn(n_seqs, total_q, max_q_len, max_kv_len, n_groups=n_groups)


def _pages(s):
    """The description of the pages, which a program makes once."""
    Hk = s.get("Hk", 1)
    return _layout(s.get("Hq", Hk), Hk, s.get("d", 64), s["ps"], s["n_pages"], s["lens"].rows, s["width"], dtype=s.get("dtype", BF16))


def _own_rotate(s):
    r = _rotation(s["Hq"], s["Hk"], s["d"], s["rot"], s["pairs"], s["dtype"], s["magnitude"], s["back"])
    if s["write"]:
        _ctx().asl_rotate_write(_pages(s), r, s["q"], s["k"], s["v"], s["pos"], s["slot"], s["freqs"], s["q_out"], s["k_pages"],
                                s["v_pages"])
        return s["q_out"], s["k_pages"], s["v_pages"]
    _ctx().asl_rotate(r, s["q"], s["k"], s["pos"], s["freqs"], s["q_out"], s["k_out"])
    return s["q_out"], s["k_out"]


def _own_plan(s):
    s["book"].copy_(s["book_before"])
    _ctx().asl_pages_plan(_pages(s), s["rows"], s["add"], s["seqs"], s["total"], s["table"], s["kv_len"], s["refs"], s["cu_out"], s["slot"],
                          s["pos"], parent=s["parent"], pruned=s["pruned"])
    return s["table"], s["kv_len"], s["refs"], s["cu_out"], s["slot"], s["pos"]


def _own_tree(s):
    shared = s["members"] > 1
    a = _batch(s["lens"].rows, s["total"], s["n_hi"], s["prefix"] + s["ctx_hi"] + s["n_hi"], s["groups"] if shared else 0)
    _ctx().asl_tree_attention(_pages(s), a, s["q"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], s["cu"], s["parent"], s["out"],
                              lse=s["lse"], group_start=s["group_start"] if shared else None,
                              prefix_len=s["prefix_len"] if shared else None)
    return s["out"], s["lse"]


def _own_accept(s):
    s["book"].copy_(s["book_before"])
    _ctx().asl_pages_accept(_pages(s), s["k_ptrs"], s["v_ptrs"], s["layers"], s["rows"], s["cu"], s["path"], s["n_path"], s["seqs"],
                            s["table"], s["kv_len"], s["refs"])
    return s["kv_len"], s["refs"], s["k_pages"], s["v_pages"]


def run(state):
    op = state["op"]
    if own:
        return {"rotate": _own_rotate, "plan": _own_plan, "tree": _own_tree, "accept": _own_accept}[op](state)
    return {"rotate": _plain_rotate, "plan": _plain_plan, "tree": _plain_tree, "accept": _plain_accept}[op](state)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    c, ln = case, _Lengths(case, 0)
    e = 4 if c.get("dtype") == F32 else 2
    n = sum(ln.n)
    if c["op"] == "rotate":
        heads = c["Hq"] + c["Hk"] * (2 if c["write"] else 1)
        return {"bytes": 2 * n * heads * c["d"] * e + n * (12 if c["write"] else 4), "flops": 3 * n * (c["Hq"] + c["Hk"]) * c["rot"]}
    if c["op"] == "plan":
        fresh = sum(ln.pages) - sum(ln.old_pages)
        return {"bytes": n * (16 if c["tree"] else 12) + 12 * fresh + 24 * ln.rows, "flops": 0}
    if c["op"] == "tree":
        Hk, d = c["Hk"], c["d"]
        shared = c["prefix"] if c["members"] > 1 else 0
        keys = sum(ln.kv) - shared * (c["members"] - 1) * c["groups"]
        # a node's ancestors among the draft are few beside its context: half of the draft at most, half of that counted
        pairs = sum(m * (old + (m + 3) // 4) for m, old in zip(ln.n, ln.old))
        return {"bytes": 2 * keys * Hk * d * e + 2 * n * c["Hq"] * d * e + 4 * n * c["Hq"] + 4 * sum(ln.pages) + 4 * n,
                "flops": 4.0 * pairs * c["Hq"] * d}
    moved = sum(ln.keep) // 2                                    # about half of a path's nodes stand where they belong
    gone = sum(ln.pages) - sum(-(-(o + a) // c["ps"]) for o, a in zip(ln.old, ln.keep))
    return {"bytes": 4 * c["layers"] * moved * c["Hk"] * c["d"] * e + 12 * gone + 8 * sum(ln.keep) + 16 * ln.rows, "flops": 0}


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, written apart

def _chain(parent, i):
    out = []
    while i >= 0:
        out.append(i)
        i = parent[i]
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    op, ps = case["op"], case["ps"]
    if op == "rotate":
        r, h = case["rot"], case["rot"] // 2
        angle = s["pos"].to(torch.float64)[:, None] * s["freqs"][None, :]
        turn = torch.polar(torch.full_like(angle, s["magnitude"]), -angle if case["back"] else angle)[:, None, :]
        first = torch.arange(h, device="cuda") * (1 if case["pairs"] == "halves" else 2)
        second = first + (h if case["pairs"] == "halves" else 1)
        outs = []
        for x in (s["q"], s["k"]):
            y = x.to(torch.float64).clone()
            z = torch.complex(y[..., first], y[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            outs.append(y)
        if not case["write"]:
            return tuple(outs)
        k, v = s["k_pages"].to(torch.float64), s["v_pages"].to(torch.float64)
        slot = s["slot"]
        for head in range(case["Hk"]):
            k[slot // ps, head, slot % ps] = outs[1][:, head]
            v[slot // ps, head, slot % ps] = s["v"][:, head].to(torch.float64)
        return outs[0], k, v
    kv, table = s["kv_len"].tolist(), s["table"].tolist()
    if op == "plan":
        refs, parent, pruned = s["refs"].tolist(), s["parent"].tolist() if s["parent"] is not None else None, s["pruned"].tolist()
        free = [p for p, x in enumerate(refs) if x == 0]
        cu, slot, pos, room = [0], [], [], True
        for b, m in enumerate(s["add"].tolist()):
            old = kv[b]
            have, want = -(-old // ps), -(-(old + m) // ps)
            room = room and want - have <= len(free)
            if room:
                for t in range(have, want):
                    table[b][t] = free.pop(0)
                    refs[table[b][t]] = 1
                kv[b] = old + m
            for i in range(m):
                slot.append(table[b][(old + i) // ps] * ps + (old + i) % ps if room else -1)
                deep = i if parent is None else len(_chain(parent[cu[-1]:cu[-1] + m], i)) - 1
                pos.append(old + deep + pruned[b])
            cu.append(cu[-1] + m)
        i32 = torch.int32
        return (torch.tensor(table, dtype=i32), torch.tensor(kv, dtype=i32), torch.tensor(refs, dtype=i32), torch.tensor(cu, dtype=i32),
                torch.tensor(slot, dtype=torch.int64), torch.tensor(pos, dtype=i32))
    cu = s["cu"].tolist()
    if op == "tree":
        G, parent = case["Hq"] // case["Hk"], s["parent"].tolist()
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
        for b in range(len(kv)):
            m, L = cu[b + 1] - cu[b], kv[b]
            if m == 0:
                continue
            at = torch.arange(L, device="cuda")
            page, slot = s["table"][b].long()[at // ps], at % ps
            seen = torch.zeros((m, L), dtype=torch.bool)
            seen[:, :L - m] = True
            for i in range(m):
                seen[i, [L - m + a for a in _chain(parent[cu[b]:cu[b + 1]], i)]] = True
            hide = ~seen.to("cuda")
            for h in range(case["Hk"]):
                K, V = s["k_pages"][page, h, slot].double(), s["v_pages"][page, h, slot].double()
                for g in range(h * G, (h + 1) * G):
                    x = s["q"][cu[b]:cu[b + 1], g].double() @ K.T / math.sqrt(case["d"])
                    x[hide] = -math.inf
                    lse[g, cu[b]:cu[b + 1]] = torch.logsumexp(x, dim=1)
                    out[cu[b]:cu[b + 1], g] = torch.softmax(x, dim=1) @ V
        return out, lse
    refs = s["refs"].tolist()
    k, v = s["k_pages"].double(), s["v_pages"].double()
    for b, (path, a) in enumerate(zip(s["path"].tolist(), s["n_path"].tolist())):
        L = kv[b]
        base = L - (cu[b + 1] - cu[b])
        for t, node in enumerate(path[:a]):
            p0, p1 = table[b][(base + node) // ps], table[b][(base + t) // ps]
            if node != t:
                k[:, p1, :, (base + t) % ps] = k[:, p0, :, (base + node) % ps]
                v[:, p1, :, (base + t) % ps] = v[:, p0, :, (base + node) % ps]
        for e in range(-(-(base + a) // ps), -(-L // ps)):
            refs[table[b][e]] -= 1
        kv[b] = base + a
    return torch.tensor(kv, dtype=torch.int32), torch.tensor(refs, dtype=torch.int32), k, v
