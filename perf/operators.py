"""The paged cache and the attention that reads it, as cases that can be timed and compared.

Four operators, each through the calls that a serving program makes once the layers' caches have been pruned:

* ``attention``: attention over a cache kept in pages, for batches of one query token or of many, with a prompt that
  several sequences share (its keys and values are then needed once for all of them);
* ``write``: new tokens, or the tokens that the selection kept of a dense cache, into the last positions of table rows;
* ``compact``: the kept tokens of paged sequences into the pages of other rows;
* ``fork``: continuations of a sequence that share its full pages and get a copy of the last, partly filled one; then
  they are freed again, so that a pass leaves the counts as it found them.

A sequence is a row of ``table`` (page numbers) and a length in ``kv_len``; pages are [n_pages, heads, page_size, d].
With ``own`` false every operator is computed from its definition with elementary operations.
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
        # a small model in fp32 (4 query heads, 2 KV heads of 64), five short requests with a draft of up to 4 tokens: latency
        dict(name="attention tiny fp32", op="attention", dtype=F32, Hq=4, Hk=2, d=64, ps=16, groups=5, members=1, prefix=0,
             own_lo=1, own_hi=500, q_lo=1, q_hi=4, causal=True),
        # one request decoding over a context that was not pruned, second head geometry: all keys and values, one token
        dict(name="attention decode 128K", op="attention", dtype=BF16, Hq=28, Hk=4, d=128, ps=64, groups=1, members=1, prefix=0,
             own_lo=131089, own_hi=131089, q_lo=1, q_hi=1, causal=True),
        # a serving batch whose prompts were pruned to the budget of 2048 and that has generated up to 500 tokens since
        dict(name="attention decode pruned batch", op="attention", dtype=BF16, Hq=32, Hk=8, d=128, ps=64, groups=48, members=1,
             prefix=0, own_lo=2049, own_hi=2548, q_lo=1, q_hi=1, causal=True),
        # 64 requests behind one long common prompt, each with a short question and answer of its own
        dict(name="attention shared prompt 32K", op="attention", dtype=BF16, Hq=32, Hk=8, d=128, ps=64, groups=1, members=64,
             prefix=32768, own_lo=1, own_hi=700, q_lo=1, q_hi=1, causal=True),
        # 8 prompts pruned to 2048 + window, 6 continuations of each, a draft of 2 to 5 tokens being verified, pages of 16
        dict(name="attention shared drafts", op="attention", dtype=BF16, Hq=28, Hk=4, d=128, ps=16, groups=8, members=6,
             prefix=2090, own_lo=6, own_hi=200, q_lo=2, q_hi=5, causal=True),
        # a chunk of two prompts being prefilled behind what is cached of them: compute
        dict(name="attention prefill chunk", op="attention", dtype=BF16, Hq=32, Hk=8, d=128, ps=64, groups=2, members=1, prefix=0,
             own_lo=14001, own_hi=16384, q_lo=1537, q_hi=2048, causal=True),
        # one new token of each of 64 requests, one layer: latency
        dict(name="write append", op="write", dtype=BF16, Hk=8, d=128, ps=16, seqs=64, n_lo=1, n_hi=1, old_lo=40, old_hi=250,
             src=0),
        # the tokens that the selection kept of a 128K prompt (budget 8192, window 64), per head, into pages
        dict(name="write selected 128K", op="write", dtype=BF16, Hk=4, d=128, ps=64, seqs=1, n_lo=8192, n_hi=8192, old_lo=0,
             old_hi=0, src=131072),
        # a batch of paged contexts pruned again to the budget, per-head tokens
        dict(name="compact batch", op="compact", dtype=BF16, Hk=8, d=128, ps=64, seqs=12, src_lo=5001, src_hi=8192, keep=2048,
             per_head=True),
        # the small fp32 model's budget of 128 from 512 tokens, tokens shared by the heads
        dict(name="compact tiny fp32", op="compact", dtype=F32, Hk=2, d=64, ps=16, seqs=3, src_lo=300, src_hi=512, keep=128,
             per_head=False),
        # a prompt continued four times, two layers: latency
        dict(name="fork one", op="fork", dtype=BF16, Hk=8, d=128, ps=64, layers=2, parents=1, times=4, len_lo=2071, len_hi=2071),
        # a batch of 24 continued 8 times each over 16 layers
        dict(name="fork batch", op="fork", dtype=BF16, Hk=8, d=128, ps=64, layers=16, parents=24, times=8, len_lo=100, len_hi=700),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, its logarithm uniform."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case; none costs more than the largest listed ones (fp32 products run at a sixteenth of bf16's rate)."""
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] <= 4.5e8 and w["flops"] <= (8e11 if c["dtype"] == BF16 else 5e10):
            return c


def _draw(rng):
    op = rng.choice(["attention", "attention", "attention", "write", "compact", "fork"])
    dtype = rng.choice([BF16, BF16, BF16, F32])
    Hk = rng.choice([1, 2, 4, 8])
    d = rng.choice([64, 80, 96, 128, 128, 128, 256])
    ps = rng.choice([16, 32, 64, 128, 256])
    if op == "attention":
        G = rng.choice([1, 2, 4, 7, 8])
        kind = rng.choice(["decode", "long", "shared", "chunk", "cross"])
        c = dict(op=op, dtype=dtype, Hq=G * Hk, Hk=Hk, d=d, ps=ps, groups=1, members=1, prefix=0, q_lo=1, q_hi=1, causal=True)
        if kind == "decode":
            hi = _log(rng, 2, 4000)
            c |= dict(groups=_log(rng, 1, 64), own_lo=_log(rng, 1, hi), own_hi=hi, q_hi=rng.choice([1, 1, 2, 5]))
        elif kind == "long":
            n = _log(rng, 4000, 100000)
            c |= dict(groups=rng.choice([1, 2]), own_lo=n - 99, own_hi=n)
        elif kind == "shared":
            c |= dict(groups=rng.choice([1, 1, 2, 5]), members=_log(rng, 2, 24), prefix=_log(rng, 50, 8000), own_lo=5,
                      own_hi=_log(rng, 6, 500), q_hi=rng.choice([1, 1, 3, 5]))
        elif kind == "chunk":
            n = _log(rng, 8, 1500)
            c |= dict(groups=rng.choice([1, 2, 3]), own_lo=n, own_hi=n + _log(rng, 1, 6000), q_lo=max(1, n // 2), q_hi=n)
        else:                      # every query sees every key: an encoder's states, of another length than the queries
            n = _log(rng, 1, 3000)
            c |= dict(groups=_log(rng, 1, 8), own_lo=max(1, n // 2), own_hi=n, q_hi=_log(rng, 1, 300), causal=False)
        return c
    if op == "write":
        if rng.random() < 0.5:
            n = _log(rng, 1, 200)
            return dict(op=op, dtype=dtype, Hk=Hk, d=d, ps=ps, seqs=_log(rng, 1, 100), n_lo=1, n_hi=n, old_lo=0, old_hi=200, src=0)
        n = _log(rng, 17, 4096)
        return dict(op=op, dtype=dtype, Hk=Hk, d=d, ps=ps, seqs=1, n_lo=n, n_hi=n, old_lo=0, old_hi=0, src=n * _log(rng, 1, 16) + 1)
    if op == "compact":
        hi = _log(rng, 20, 6000)
        return dict(op=op, dtype=dtype, Hk=Hk, d=d, ps=ps, seqs=_log(rng, 1, 8), src_lo=hi // 2 + 1, src_hi=hi,
                    keep=_log(rng, 1, hi // 2), per_head=rng.random() < 0.5)
    return dict(op=op, dtype=dtype, Hk=Hk, d=d, ps=ps, layers=rng.choice([1, 2, 4]), parents=_log(rng, 1, 24),
                times=_log(rng, 1, 8), len_lo=1, len_hi=_log(rng, 2, 700))


# ---------------------------------------------------------------------------------------------------------------------
# inputs

class _Lengths:
    """The whole numbers of a case. The lengths are the case's own, so that tensors of any seed have the same shapes; which
    sequence has which is the seed's."""

    def __init__(self, c, seed):
        fixed = torch.Generator().manual_seed(11)
        op = c["op"]
        n = c["groups"] * c["members"] if op == "attention" else c["parents"] if op == "fork" else c["seqs"]
        order = torch.randperm(n, generator=torch.Generator().manual_seed(7 * int(seed) + 1)).tolist()

        def between(lo, hi):
            x = torch.randint(lo, hi + 1, (n,), generator=fixed).tolist()
            return [x[i] for i in order]

        self.rows = n
        if op == "attention":
            own_len, self.q = between(c["own_lo"], c["own_hi"]), between(c["q_lo"], c["q_hi"])
            if c["causal"]:                                      # the queries are the last of a sequence's own tokens
                self.q = [min(a, b) for a, b in zip(self.q, own_len)]
            self.kv = [c["prefix"] + x for x in own_len]
        elif op == "write":
            self.n, self.old = between(c["n_lo"], c["n_hi"]), between(c["old_lo"], c["old_hi"])
            self.kv = [a + b for a, b in zip(self.n, self.old)]
        elif op == "compact":
            self.kv = between(c["src_lo"], c["src_hi"])
            self.n = [min(c["keep"], x) for x in self.kv]
            self.rows = 2 * n
        else:
            self.kv = between(c["len_lo"], c["len_hi"])
            self.rows = n * (1 + c["times"])
        self.pages = [-(-x // c["ps"]) for x in self.kv]


def _cumulative(counts):
    out = [0]
    for x in counts:
        out.append(out[-1] + x)
    return out


def _inputs(c, seed):
    dev, dt, ps, Hk, d, op = "cuda", DTYPE[c["dtype"]], c["ps"], c["Hk"], c["d"], c["op"]
    ln = _Lengths(c, seed)
    host = torch.Generator().manual_seed(7 * int(seed) + 2)
    g = torch.Generator(device=dev).manual_seed(7 * int(seed) + 3)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32).to(dev)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(dt)

    s = dict(c, lens=ln)
    width = max(ln.pages) + 1                                    # entries of a table row
    shared = c["prefix"] // ps if op == "attention" and c["members"] > 1 else 0
    owned = [p - shared for p in ln.pages]
    dst = [-(-n // ps) for n in ln.n] if op == "compact" else []
    used = sum(owned) + (shared * c["groups"] if shared else 0) + sum(dst)
    spare = c["parents"] * c["times"] + 3 if op == "fork" else 3  # pages that nobody holds
    n_pages = used + spare
    order = torch.randperm(n_pages, generator=host, dtype=torch.int64).tolist()  # a cache in use: no row's pages are neighbours
    table = torch.full((ln.rows, width), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(owned):
        if shared:
            if r % c["members"] == 0:
                first = order[at:at + shared]
                at += shared
            table[r, :shared] = torch.tensor(first, dtype=torch.int32)
        table[r, shared:shared + n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    for i, n in enumerate(dst):
        table[c["seqs"] + i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    lens = ln.kv + (ln.n if op == "compact" else [0] * (ln.rows - len(ln.kv)))
    s |= dict(n_pages=n_pages, width=width, table=table.to(dev), kv_len=ints(lens))
    layers = c["layers"] if op == "fork" else 1
    s["k_pages"] = normal(layers, n_pages, Hk, ps, d)
    s["v_pages"] = normal(layers, n_pages, Hk, ps, d)
    if op != "fork":
        s["k_pages"], s["v_pages"] = s["k_pages"][0], s["v_pages"][0]
    if op == "attention":
        total = sum(ln.q)
        s |= dict(total_q=total, cu_q=ints(_cumulative(ln.q)), group_start=ints(_cumulative([c["members"]] * c["groups"])),
                  prefix_len=ints([c["prefix"]] * c["groups"]))
        s["q"] = normal(total, c["Hq"], d) * 2                   # logits with a spread of 2: some tokens stand out
        s["out"] = torch.empty((total, c["Hq"], d), dtype=dt, device=dev)
        s["lse"] = torch.empty((c["Hq"], total), dtype=torch.float32, device=dev)
    elif op == "write":
        total = sum(ln.n)
        n_src = c["src"] or total
        s |= dict(total=total, n_src=n_src, cu=ints(_cumulative(ln.n)), rows=ints(list(range(c["seqs"]))), idx=None)
        if c["src"]:                                             # what a selection leaves: ascending tokens of each head
            pick = torch.rand((Hk, n_src), generator=g, device=dev).topk(total, dim=1).indices
            s["idx"] = pick.sort(dim=1).values.to(torch.int32).contiguous()
            s["k"], s["v"] = normal(Hk, n_src, d), normal(Hk, n_src, d)
        else:                                                    # what a projection leaves: tokens, then heads
            s["k"], s["v"] = normal(n_src, Hk, d).transpose(0, 1), normal(n_src, Hk, d).transpose(0, 1)
    elif op == "compact":
        total, heads = sum(ln.n), Hk if c["per_head"] else 1
        picks = [torch.rand((heads, L), generator=host).topk(n, dim=1).indices.sort(dim=1).values for L, n in zip(ln.kv, ln.n)]
        s |= dict(total=total, cu=ints(_cumulative(ln.n)), idx=torch.cat(picks, dim=1).to(torch.int32).contiguous().to(dev),
                  src_rows=ints(list(range(c["seqs"]))), dst_rows=ints(list(range(c["seqs"], 2 * c["seqs"]))))
    else:
        refs = torch.zeros(n_pages, dtype=torch.int32)
        refs[torch.tensor(order[:used], dtype=torch.int64)] = 1
        P, t = c["parents"], c["times"]
        s |= dict(refs=refs.to(dev), parents=ints([i // t for i in range(P * t)]), children=ints(list(range(P, P * (1 + t)))))
        s["k_ptrs"] = torch.tensor([x.data_ptr() for x in s["k_pages"]], dtype=torch.int64).to(dev)
        s["v_ptrs"] = torch.tensor([x.data_ptr() for x in s["v_pages"]], dtype=torch.int64).to(dev)
    return s


def prepare(case, seed):
    return _inputs(case, seed)


# ---------------------------------------------------------------------------------------------------------------------
# the operators from their definitions

def _plain_attention(s):
    """softmax(scale q K^T) V over each sequence's pages, all sequences padded to the longest; log-sum-exp of each row."""
    Hq, Hk, d, ps = s["Hq"], s["Hk"], s["d"], s["ps"]
    B, G, dev = s["lens"].rows, s["Hq"] // s["Hk"], s["q"].device
    kv, cu = s["kv_len"].long(), s["cu_q"].long()
    n_q = cu[1:] - cu[:-1]
    most_q, most_kv = max(s["lens"].q), max(s["lens"].kv)
    pages = s["table"].long().clamp(min=0)[:, :-(-most_kv // ps)]
    k = s["k_pages"][pages].float().transpose(1, 2).reshape(B, Hk, -1, d)
    v = s["v_pages"][pages].float().transpose(1, 2).reshape(B, Hk, -1, d)
    i = torch.arange(most_q, device=dev)
    q = s["q"][(cu[:-1, None] + i).clamp(max=s["total_q"] - 1)].float()                       # [B, i, Hq, d]
    q = q.reshape(B, most_q, Hk, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hk, most_q * G, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(d ** -0.5)                                    # [B, Hk, i * G, keys]
    last = kv[:, None] - n_q[:, None] + i + 1 if s["causal"] else kv[:, None].expand(B, most_q)
    seen = torch.arange(k.shape[2], device=dev) < last[:, :, None]
    x.masked_fill_(~seen.repeat_interleave(G, dim=1)[:, None], -math.inf)
    top = x.amax(dim=3, keepdim=True).clamp(min=-3.0e38)
    p = x.sub_(top).exp_()
    z = p.sum(dim=3, keepdim=True)
    o = torch.matmul(p, v) / z.clamp(min=1e-38)
    lse = (top + z.log()).squeeze(3)
    tok = torch.arange(s["total_q"], device=dev)
    seq = torch.searchsorted(cu[1:], tok, right=True)
    o = o.reshape(B, Hk, most_q, G, d).permute(0, 2, 1, 3, 4).reshape(B, most_q, Hq, d)
    lse = lse.reshape(B, Hk, most_q, G).permute(0, 2, 1, 3).reshape(B, most_q, Hq)
    at = (seq, tok - cu[seq])
    return o[at].to(s["q"].dtype), lse[at].t().contiguous()


def _plain_places(s, rows):
    """Of each new token: its sequence, and the page and slot of its place, the last ones of its row."""
    cu, kv = s["cu"].long(), s["kv_len"].long()
    j = torch.arange(s["total"], device=cu.device)
    seq = torch.searchsorted(cu[1:], j, right=True)
    r = rows.long()[seq]
    pos = kv[r] - (cu[seq + 1] - j)
    return seq, s["table"].long()[r, pos // s["ps"]], pos % s["ps"]


def _plain_write(s):
    _, page, slot = _plain_places(s, s["rows"])
    h = torch.arange(s["Hk"], device=page.device)[:, None]
    src = torch.arange(s["total"], device=page.device)[None] if s["idx"] is None else s["idx"].long()
    s["k_pages"][page[None], h, slot[None]] = s["k"][h, src]
    s["v_pages"][page[None], h, slot[None]] = s["v"][h, src]
    return s["k_pages"], s["v_pages"]


def _plain_compact(s):
    seq, page, slot = _plain_places(s, s["dst_rows"])
    h = torch.arange(s["Hk"], device=page.device)[:, None]
    src = s["idx"].long()
    from_page = s["table"].long()[s["src_rows"].long()[seq][None], src // s["ps"]]
    s["k_pages"][page[None], h, slot[None]] = s["k_pages"][from_page, h, src % s["ps"]]
    s["v_pages"][page[None], h, slot[None]] = s["v_pages"][from_page, h, src % s["ps"]]
    return s["k_pages"], s["v_pages"]


def _plain_fork(s):
    """Forks take the lowest free pages in the order of the list, while there are enough; then all are freed."""
    table, kv, refs, ps = s["table"], s["kv_len"], s["refs"], s["ps"]
    pa, ch = s["parents"].long(), s["children"].long()
    n = kv[pa].long()
    full, part = n // ps, n % ps
    need = (part > 0).long()
    upto = need.cumsum(0)
    fits = upto <= (refs == 0).sum()
    free = torch.argsort((refs != 0).int(), stable=True)
    new = free[(upto - 1).clamp(min=0)]
    t = torch.arange(table.shape[1], device=table.device)
    held = (t < full[:, None]) & fits[:, None]
    rows = table[pa]
    at_part = (t == full[:, None]) & ((need > 0) & fits)[:, None]
    old = rows.long().gather(1, full[:, None].clamp(max=table.shape[1] - 1))[:, 0].clamp(min=0)
    table[ch] = torch.where(held, rows, torch.where(at_part, new[:, None].int(), table[ch]))
    kv[ch] = torch.where(fits, n, kv[ch].long()).int()
    refs.index_add_(0, rows.clamp(min=0).reshape(-1).long(), held.reshape(-1).int())
    takes = (need > 0) & fits
    refs.index_add_(0, new, takes.int())
    to = torch.where(takes, new, old)
    filled = (torch.arange(ps, device=table.device) < part[:, None])[None, :, None, :, None]
    for_k = torch.where(filled, s["k_pages"][:, old], s["k_pages"][:, to])
    for_v = torch.where(filled, s["v_pages"][:, old], s["v_pages"][:, to])
    s["k_pages"][:, to] = for_k
    s["v_pages"][:, to] = for_v
    # the continuations end
    gone = t < (-(-kv[ch].long() // ps))[:, None]
    refs.index_add_(0, table[ch].clamp(min=0).reshape(-1).long(), -gone.reshape(-1).int())
    kv[ch] = 0
    return table, kv, refs, s["k_pages"], s["v_pages"]


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
    return _handle(256, 1 << 19, 256)


@functools.lru_cache(maxsize=None)
def _layout(*sizes, dtype):
    from paper_2601_07667_amd import asl
    return asl.make_pages(*sizes, dtype=asl.ASL_BF16 if dtype == BF16 else asl.ASL_F32)


@functools.lru_cache(maxsize=None)
def _batch(n_seqs, total_q, max_q_len, max_kv_len, n_groups, causal):
    from paper_2601_07667_amd import asl
    return asl.make_attn(n_seqs, total_q, max_q_len, max_kv_len, n_groups=n_groups, causal=causal)


def _pages(s):
    """The description of the pages, which a program makes once."""
    return _layout(s.get("Hq", s["Hk"]), s["Hk"], s["d"], s["ps"], s["n_pages"], s["lens"].rows, s["width"], dtype=s["dtype"])


def _own_attention(s):
    shared = s["members"] > 1
    a = _batch(s["lens"].rows, s["total_q"], s["q_hi"], s["prefix"] + s["own_hi"], s["groups"] if shared else 0, s["causal"])
    _ctx().asl_paged_attention(_pages(s), a, s["q"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], s["cu_q"], s["out"],
                               lse=s["lse"], group_start=s["group_start"] if shared else None,
                               prefix_len=s["prefix_len"] if shared else None)
    return s["out"], s["lse"]


def _own_write(s):
    _ctx().asl_pages_write(_pages(s), s["k"], s["v"], s["rows"], s["cu"], s["seqs"], s["total"], s["table"], s["kv_len"],
                           s["k_pages"], s["v_pages"], idx=s["idx"])
    return s["k_pages"], s["v_pages"]


def _own_compact(s):
    _ctx().asl_pages_compact(_pages(s), s["src_rows"], s["dst_rows"], s["cu"], s["seqs"], s["total"], s["idx"], s["table"],
                             s["kv_len"], s["k_pages"], s["v_pages"])
    return s["k_pages"], s["v_pages"]


def _own_fork(s):
    n, p = s["parents"].numel(), _pages(s)
    _ctx().asl_pages_fork(p, s["k_ptrs"], s["v_ptrs"], s["layers"], s["parents"], s["children"], n, s["table"], s["kv_len"],
                          s["refs"])
    _ctx().asl_pages_free(p, s["children"], n, s["table"], s["kv_len"], s["refs"])
    return s["table"], s["kv_len"], s["refs"], s["k_pages"], s["v_pages"]


def run(state):
    op = state["op"]
    if own:
        return {"attention": _own_attention, "write": _own_write, "compact": _own_compact, "fork": _own_fork}[op](state)
    return {"attention": _plain_attention, "write": _plain_write, "compact": _plain_compact, "fork": _plain_fork}[op](state)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    c, ln = case, _Lengths(case, 0)
    e = 2 if c["dtype"] == BF16 else 4
    Hk, d = c["Hk"], c["d"]
    if c["op"] == "attention":
        shared = c["prefix"] if c["members"] > 1 else 0
        keys = sum(ln.kv) - shared * (c["members"] - 1) * c["groups"]
        pairs = sum(n * kv - (n * (n - 1) // 2 if c["causal"] else 0) for n, kv in zip(ln.q, ln.kv))
        q = sum(ln.q)
        return {"bytes": 2 * keys * Hk * d * e + 2 * q * c["Hq"] * d * e + 4 * q * c["Hq"] + 4 * sum(ln.pages),
                "flops": 4.0 * pairs * c["Hq"] * d}
    if c["op"] in ("write", "compact"):
        n = sum(ln.n)
        idx = (n * Hk if c.get("per_head") or c.get("src") else n if c["op"] == "compact" else 0)
        return {"bytes": 4 * n * Hk * d * e + 4 * idx, "flops": 0}
    copied = sum(x % c["ps"] for x in ln.kv) * c["times"]
    entries = sum(ln.pages) * c["times"]
    once = sum(x % c["ps"] for x in ln.kv)
    return {"bytes": 2 * c["layers"] * (copied + once) * Hk * d * e + 4 * (5 * entries), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, written apart

def exact(case, seed):
    s = _inputs(case, seed)
    kv = s["kv_len"].tolist()
    table = s["table"].long()
    if case["op"] == "attention":
        cu, G = s["cu_q"].tolist(), case["Hq"] // case["Hk"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
        for b in range(len(kv)):
            n, L = cu[b + 1] - cu[b], kv[b]
            if n == 0 or L == 0:
                continue
            at = torch.arange(L, device="cuda")
            page, slot = table[b][at // case["ps"]], at % case["ps"]
            limit = torch.arange(L - n, L, device="cuda") if case["causal"] else torch.full((n,), L - 1, device="cuda")
            hide = at[None, :] > limit[:, None]
            for h in range(case["Hk"]):
                K, V = s["k_pages"][page, h, slot].double(), s["v_pages"][page, h, slot].double()
                for g in range(h * G, (h + 1) * G):
                    x = s["q"][cu[b]:cu[b + 1], g].double() @ K.T / math.sqrt(case["d"])
                    x[hide] = -math.inf
                    lse[g, cu[b]:cu[b + 1]] = torch.logsumexp(x, dim=1)
                    out[cu[b]:cu[b + 1], g] = torch.softmax(x, dim=1) @ V
        return out, lse
    if case["op"] in ("write", "compact"):
        cu, total = s["cu"].tolist(), s["total"]
        rows = (s["rows"] if case["op"] == "write" else s["dst_rows"]).tolist()
        k, v = s["k_pages"].double(), s["v_pages"].double()
        for i, r in enumerate(rows):
            for h in range(case["Hk"]):
                n = cu[i + 1] - cu[i]
                if case["op"] == "write":
                    src = s["idx"][h, cu[i]:cu[i + 1]].long() if s["idx"] is not None else torch.arange(cu[i], cu[i + 1], device="cuda")
                    new_k, new_v = s["k"][h][src], s["v"][h][src]
                else:
                    src = s["idx"][h if case["per_head"] else 0, cu[i]:cu[i + 1]].long()
                    page = table[s["src_rows"][i]][src // case["ps"]]
                    new_k, new_v = s["k_pages"][page, h, src % case["ps"]], s["v_pages"][page, h, src % case["ps"]]
                pos = torch.arange(kv[r] - n, kv[r], device="cuda")
                k[table[r][pos // case["ps"]], h, pos % case["ps"]] = new_k.double()
                v[table[r][pos // case["ps"]], h, pos % case["ps"]] = new_v.double()
        return k, v
    rows, refs, ps = s["table"].tolist(), s["refs"].tolist(), case["ps"]
    k, v = s["k_pages"].double(), s["v_pages"].double()
    for a, b in zip(s["parents"].tolist(), s["children"].tolist()):
        full, part = divmod(kv[a], ps)
        for t in range(full):
            rows[b][t] = rows[a][t]
            refs[rows[a][t]] += 1
        if part:
            page = refs.index(0)
            refs[page] = 1
            k[:, page, :, :part] = k[:, rows[a][full], :, :part]
            v[:, page, :, :part] = v[:, rows[a][full], :, :part]
            rows[b][full] = page
        kv[b] = kv[a]
    for b in s["children"].tolist():
        for t in range(-(-kv[b] // ps)):
            refs[rows[b][t]] -= 1
        kv[b] = 0
    return torch.tensor(rows, dtype=torch.int32), torch.tensor(kv, dtype=torch.int32), torch.tensor(refs, dtype=torch.int32), k, v
