"""Drafting over the paged cache on the GPU against its float64 oracle."""
import random

import numpy as np
import pytest

from oracle import draft_oracle as do
from oracle import paged_oracle as po
from paper_2601_07667_amd import asl
from test_gpu_paged import NP, Cache, _attend, _bounds, _check, _dt, _ints, _queries, _torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = asl.Asl(2, 1, 1)
    c.asl_paged_reserve(4096, 1 << 17, 256)
    yield c
    assert c.asl_device_fault() == 0, "a test left the fault word set"
    c.close()


def _longs(x, dev):
    torch = _torch()
    return torch.tensor(np.asarray(x, dtype=np.int64), device=dev)


def _random_parents(n, seed, chain=0.45, root=0.05):
    r = random.Random(seed)
    return [-1 if i == 0 or r.random() < root else i - 1 if r.random() < chain else r.randrange(i) for i in range(n)]


# ---------------------------------------------------------------------------------------------------------------- rotate
def _turn_bound(y, reach, angle, dtype):
    """How far a rotated element may be off.  |x| <= pi / 4 rounds once (half an ulp: 0.79 x 2^-24), its series and their last additions round
    (together under 1.3 x 2^-24 for either of sine and cosine, at most 1 in size), the magnitude rounds (2^-24), a product and a sum each
    (2^-24 of magnitude (|a| + |b|)): under 6 x 2^-24 of that in all.  The angle: three roundings of 64 bits here and two in the oracle.
    The result rounds once."""
    return NP[dtype] * np.abs(y) * 1.01 + reach * (6 * 2.0 ** -24 + 5 * 2.0 ** -53 * angle) + 1e-38


def _layout(torch, n, H, d, kind, dtype, dev, fill=None):
    """A [n, H, d] tensor: dense, heads first, a slice of a wider projection, or off every alignment but an element's."""
    def empty(*s):
        x = torch.empty(s, dtype=_dt(dtype), device=dev)
        x.fill_(float("nan"))
        return x
    x = {"dense": lambda: empty(n, H, d), "heads": lambda: empty(H, n, d).transpose(0, 1), "wide": lambda: empty(n, H + 3, d + 8)[:, 1:H + 1, :d],
         "odd": lambda: empty(n * H * (d + 1) + 5)[3:3 + n * H * (d + 1)].view(n, H, d + 1)[..., :d]}[kind]()
    if fill is not None:
        x.copy_(fill)
    return x


def _rotated(ctx, dev, n, Hq, Hk, d, rot, halves, dtype, kinds=("dense", "dense"), back=False, magnitude=0.0, far=5000, seed=0, pos=None,
             in_place=False):
    torch = _torch()
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    pos = rng.integers(-far, far + 1, n) if pos is None else np.asarray(pos)
    f = do.freqs(rot)
    r = asl.make_rotation(Hq, Hk, d, rot, pairs=asl.ASL_PAIRS_HALVES if halves else asl.ASL_PAIRS_NEIGHBOURS,
                          dtype=asl.ASL_BF16 if dtype == "bf16" else asl.ASL_F32, magnitude=magnitude, back=back)
    ins, outs = [], []
    for H in (Hq, Hk):
        x = torch.randn((n, H, d), generator=g).to(_dt(dtype)).to(dev)
        ins.append(_layout(torch, n, H, d, kinds[0], dtype, dev, x) if H else None)
        outs.append((ins[-1] if in_place else _layout(torch, n, H, d, kinds[1], dtype, dev)) if H else None)
    kept = [x.double().cpu().numpy() if x is not None else None for x in ins]
    ctx.asl_rotate(r, ins[0], ins[1], _ints(pos, dev), torch.from_numpy(f).to(dev), outs[0], outs[1])
    torch.cuda.synchronize()
    for x, y in zip(kept, outs):
        if x is None:
            continue
        ref, reach = do.rotate(x, pos, f, halves, magnitude if magnitude > 0 else 1.0, back)
        tol = _turn_bound(ref, reach, np.abs(pos.astype(np.float64))[:, None, None] * f[0], dtype)
        got = y.double().cpu().numpy()
        bad = ~(np.abs(got - ref) <= tol)
        assert not bad.any(), (float(np.nanmax(np.abs(got - ref) / tol)), np.argwhere(bad)[:4].tolist())
        np.testing.assert_array_equal(got[..., rot:], x[..., rot:])
    return ins, outs


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 64), (128, 64), (80, 20), (96, 24), (64, 14), (256, 256), (100, 100), (8, 2), (2, 2), (512, 512),
                                   (2048, 2046)])
def test_rotate(ctx, gpu_device, d, rot, halves, dtype):
    _rotated(ctx, gpu_device, 13, 5, 2, d, rot, halves, dtype, magnitude=1.21, seed=d + rot)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("kinds", [("wide", "heads"), ("heads", "wide"), ("odd", "dense"), ("dense", "odd"), ("odd", "odd")])
def test_rotate_strides(ctx, gpu_device, kinds, halves, dtype):
    ins, outs = _rotated(ctx, gpu_device, 9, 7, 3, 80, 48, halves, dtype, kinds, seed=4)
    _rotated(ctx, gpu_device, 9, 7, 3, 34, 30, halves, dtype, kinds, seed=5)
    for x in outs:                                           # what lies between the rows is not written to
        wide = x.as_strided(x.shape[:2] + (x.shape[2] + 1,), x.stride()) if "odd" == kinds[1] else None
        if wide is not None:
            assert bool(wide[..., -1].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,Hq,Hk", [(0, 4, 2), (1, 32, 8), (1, 1, 1), (1, 1, 0), (3, 0, 5), (64, 28, 4), (511, 8, 8), (2500, 3, 1), (5, 200, 7)])
def test_rotate_sizes(ctx, gpu_device, n, Hq, Hk, dtype):
    for halves in (True, False):
        _rotated(ctx, gpu_device, n, Hq, Hk, 64, 64, halves, dtype, seed=n)


@pytest.mark.parametrize("halves", [True, False])
def test_rotations_too_large_for_the_caches(ctx, gpu_device, halves):
    """Calls of more than 100 MB take kernels of their own: the same bits as in two smaller calls, in place, and into pages."""
    torch = _torch()
    dev, n, Hq, Hk, d, ps = gpu_device, 4100, 40, 8, 128, 64
    g = torch.Generator(device=dev).manual_seed(1)
    x = torch.randn((n, Hq + 2 * Hk, d), generator=g, device=dev).to(torch.bfloat16)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    pos, f = _ints(np.arange(n) * 7, dev), torch.from_numpy(do.freqs(d)).to(dev)
    r = asl.make_rotation(Hq, Hk, d, pairs=0 if halves else 1)
    parts = [torch.empty((n, H, d), dtype=torch.bfloat16, device=dev) for H in (Hq, Hk)]
    for a, b in ((0, 2000), (2000, n)):
        ctx.asl_rotate(r, q[a:b], k[a:b], pos[a:b], f, parts[0][a:b], parts[1][a:b])
    whole = [torch.empty_like(t) for t in parts]
    ctx.asl_rotate(r, q, k, pos, f, *whole)
    assert torch.equal(whole[0], parts[0]) and torch.equal(whole[1], parts[1])
    pages = [torch.zeros((n // ps + 1, Hk, ps, d), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    out = torch.empty_like(parts[0])
    ctx.asl_rotate_write(asl.make_pages(Hq, Hk, d, ps, n // ps + 1, 1, 1), r, q, k, v, pos, _longs(np.arange(n), dev), f, out, *pages)
    assert torch.equal(out, parts[0])
    for t, want in zip(pages, (parts[1], v)):
        assert torch.equal(t.transpose(1, 2).reshape(-1, Hk, d)[:n], want)
    ctx.asl_rotate(r, q, k, pos, f, q, k)
    assert torch.equal(q, parts[0]) and torch.equal(k, parts[1]) and ctx.asl_device_fault() == 0


@pytest.mark.parametrize("halves", [True, False])
def test_rotate_far_positions(ctx, gpu_device, halves):
    """Angles of millions of turns, to the last bit of fp32."""
    pos = [0, 1, -1, 131071, 1048575, 10 ** 7 + 1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345]
    _rotated(ctx, gpu_device, len(pos), 4, 2, 128, 128, halves, "f32", pos=pos)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("d,rot,kind", [(128, 128, "dense"), (128, 32, "wide"), (34, 30, "odd")])
def test_rotate_in_place(ctx, gpu_device, d, rot, kind, halves, dtype):
    _rotated(ctx, gpu_device, 33, 6, 2, d, rot, halves, dtype, (kind, kind), in_place=True, seed=7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("halves", [True, False])
def test_rotating_back_is_the_gradient(ctx, gpu_device, halves, dtype):
    """Against the formula's, and against differences: the map is linear, so <R x, g> changes by <dx, R^T g>."""
    torch = _torch()
    dev, n, H, d, rot, mu = gpu_device, 21, 3, 64, 48, 1.3
    _rotated(ctx, dev, n, H, 2, d, rot, halves, dtype, back=True, magnitude=mu, seed=11)
    pos, f = _ints(np.arange(n) * 1000 - 7, dev), torch.from_numpy(do.freqs(rot)).to(dev)
    make = lambda back: asl.make_rotation(H, 0, d, rot, pairs=0 if halves else 1, dtype=asl.ASL_F32, magnitude=mu, back=back)
    x, dx, g = (torch.randn((n, H, d), generator=torch.Generator().manual_seed(s)).to(dev) for s in (1, 2, 3))

    def through(v, back=False):
        out = torch.empty_like(v)
        ctx.asl_rotate(make(back), v, None, pos, f, out, None)
        return out.double()
    grad = through(g, back=True)
    left, right = float(((through(x + dx) - through(x)) * g.double()).sum()), float((dx.double() * grad).sum())
    # each of the n H d products is off by at most (6 + 2) 2^-24 of |values| up to 2 x mu x 6
    assert abs(left - right) <= n * H * d * 16 * 2.0 ** -24 * 2 * mu * 6 * 6


def test_rotate_leaves_numbers_that_are_none_where_they_are(ctx, gpu_device):
    torch = _torch()
    for halves in (True, False):
        for rot in (16, 6):
            x = torch.ones((2, 2, 32), device=gpu_device)
            x[0, 0, rot:] = float("inf")
            x[0, 1, 1] = float("nan")
            out = torch.empty_like(x)
            r = asl.make_rotation(2, 0, 32, rot, pairs=0 if halves else 1, dtype=asl.ASL_F32)
            ctx.asl_rotate(r, x, None, _ints([3, 4], gpu_device), torch.from_numpy(do.freqs(rot)).to(gpu_device), out, None)
            other = rot // 2 + 1 if halves else 0
            want = torch.zeros_like(x, dtype=torch.bool)
            want[0, 1, 1] = want[0, 1, other] = True
            assert torch.equal(out.isnan(), want) and bool((out[0, 0, rot:] == float("inf")).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("halves", [True, False])
@pytest.mark.parametrize("d,rot,ps,n,kind", [(128, 128, 16, 37, "dense"), (128, 64, 64, 5, "wide"), (80, 20, 32, 70, "odd"), (64, 14, 16, 1, "heads"),
                                             (256, 256, 16, 9, "wide"), (8, 6, 16, 3, "odd")])
def test_rotate_write(ctx, gpu_device, d, rot, ps, n, kind, halves, dtype):
    """The pages get what asl_rotate gives, bit for bit, at the slots; all else stays."""
    torch = _torch()
    dev, Hq, Hk = gpu_device, 6, 3
    rng = np.random.default_rng(n)
    n_pages = -(-n // ps) + 3
    slot = rng.permutation(n_pages * ps)[:n]
    slot[n // 2] = -1
    pos, f = _ints(rng.integers(0, 100000, n), dev), torch.from_numpy(do.freqs(rot)).to(dev)
    g = torch.Generator().manual_seed(n)
    q, k, v = (_layout(torch, n, H, d, kind, dtype, dev, torch.randn((n, H, d), generator=g).to(_dt(dtype)).to(dev)) for H in (Hq, Hk, Hk))
    pages = [torch.randn((n_pages, Hk, ps, d), generator=g).to(_dt(dtype)).to(dev) for _ in range(2)]
    want = [x.clone() for x in pages]
    e = asl.ASL_BF16 if dtype == "bf16" else asl.ASL_F32
    r = asl.make_rotation(Hq, Hk, d, rot, pairs=0 if halves else 1, dtype=e, magnitude=0.9)
    q_out, q_two, k_two = (torch.empty((n, H, d), dtype=_dt(dtype), device=dev) for H in (Hq, Hq, Hk))
    desc = asl.make_pages(Hq, Hk, d, ps, n_pages, 1, 1, dtype=e)
    ctx.asl_rotate_write(desc, r, q, k, v, pos, _longs(slot, dev), f, q_out, pages[0], pages[1])
    ctx.asl_rotate(r, q, k, pos, f, q_two, k_two)
    assert torch.equal(q_out, q_two)
    for j, s in enumerate(slot):
        if s >= 0:
            want[0][s // ps, :, s % ps] = k_two[j]
            want[1][s // ps, :, s % ps] = v[j]
    assert torch.equal(pages[0], want[0]) and torch.equal(pages[1], want[1])
    assert ctx.asl_device_fault() == 0


def test_slots_out_of_range_are_left_out(ctx, gpu_device):
    torch = _torch()
    dev, d, ps = gpu_device, 64, 16
    slot = [-2, 2 * ps, 5, -2 ** 63, 2 ** 63 - 1, 3 * ps * 2 ** 32]
    n = len(slot)
    q, k = torch.ones((n, 2, d), dtype=torch.bfloat16, device=dev), torch.ones((n, 1, d), dtype=torch.bfloat16, device=dev)
    pages = torch.zeros((4, 1, ps, d), dtype=torch.bfloat16, device=dev)
    desc = asl.make_pages(2, 1, d, ps, 2, 1, 1)              # two of the four pages
    out = torch.zeros_like(q)
    vp = pages.clone()
    ctx.asl_rotate_write(desc, asl.make_rotation(2, 1, d), q, k, k, _ints([0] * n, dev), _longs(slot, dev),
                         torch.from_numpy(do.freqs(d)).to(dev), out, pages, vp)
    assert ctx.asl_device_fault() == 2
    assert bool((out == 1).all())
    for x in (pages, vp):
        assert float(x.sum()) == d and bool((x[0, 0, 5] == 1).all())


def test_rotations_of_broadcast_heads(ctx, gpu_device):
    """Inputs may share one place; outputs of several heads or tokens may not."""
    torch = _torch()
    r, pos, f = asl.make_rotation(4, 2, 64), _ints([5, 6, 7], gpu_device), asl.rotation_freqs(64).to(gpu_device)
    one = torch.randn(3, 1, 64, device=gpu_device).to(torch.bfloat16)
    q, k = one.expand(3, 4, 64), one[:1].expand(3, 2, 64)
    qo, ko = torch.empty(3, 4, 64, dtype=torch.bfloat16, device=gpu_device), torch.empty(3, 2, 64, dtype=torch.bfloat16, device=gpu_device)
    ctx.asl_rotate(r, q, k, pos, f, qo, ko)
    want_q, want_k = torch.empty_like(qo), torch.empty_like(ko)
    ctx.asl_rotate(r, q.contiguous(), k.contiguous(), pos, f, want_q, want_k)
    assert torch.equal(qo, want_q) and torch.equal(ko, want_k)
    for outs in ((qo[:, :1].expand(3, 4, 64), ko), (qo[:1].expand(3, 4, 64), ko), (qo, ko[:, :1].expand(3, 2, 64)), (qo, ko[:1].expand(3, 2, 64))):
        with pytest.raises(asl.AslError, match="one place") as e:
            ctx.asl_rotate(r, q, k, pos, f, *outs)
        assert e.value.status == asl.ASL_EINVAL
    ctx.asl_rotate(asl.make_rotation(1, 0, 64), one[:1], None, pos[:1], f, qo[:1, :1].as_strided((1, 1, 64), (0, 0, 1)), None)
    assert torch.equal(qo[0, 0], want_q[0, 0])


def test_rotate_refusals(ctx, gpu_device):
    torch = _torch()
    dev = gpu_device
    q, k = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device=dev), torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=dev)
    pos, f, slot = _ints([0] * 3, dev), torch.from_numpy(do.freqs(64)).to(dev), _longs([0] * 3, dev)
    pages = torch.zeros((1, 2, 16, 64), dtype=torch.bfloat16, device=dev)
    for r, word in ((asl.make_rotation(4, 2, 64, 63), "rot_dim"), (asl.make_rotation(4, 2, 64, dtype=7), "dtype")):
        with pytest.raises(asl.AslError, match=word):
            ctx.asl_rotate(r, q, k, pos, f, q, k)
    for desc in (asl.make_pages(4, 1, 64, 16, 1, 1, 1), asl.make_pages(4, 2, 128, 16, 1, 1, 1), asl.make_pages(4, 2, 64, 16, 1, 1, 1, dtype=asl.ASL_F32)):
        with pytest.raises(asl.AslError, match="differ"):
            ctx.asl_rotate_write(desc, asl.make_rotation(4, 2, 64), q, k, k, pos, slot, f, q, pages, pages)
    bare = asl.Asl(2, 1, 1)
    with pytest.raises(asl.AslError, match="reserve"):
        bare.asl_rotate_write(asl.make_pages(4, 2, 64, 16, 1, 1, 1), asl.make_rotation(4, 2, 64), q, k, k, pos, slot, f, q, pages, pages)
    bare.asl_rotate(asl.make_rotation(4, 2, 64), q, k, pos, f, q, k)     # (needs no workspace)
    torch.cuda.synchronize()
    bare.close()


# ------------------------------------------------------------------------------------------------------------------ plan
class _Book:
    def __init__(self, dev, n_rows, width, ps, n_pages, lens=(), held=(), seed=0):
        rng = np.random.default_rng(seed)
        self.ps, self.n_pages, self.width, self.dev = ps, n_pages, width, dev
        self.table, self.kv, self.refs = np.full((n_rows, width), -1, dtype=np.int64), np.zeros(n_rows, dtype=np.int64), np.zeros(n_pages, dtype=np.int64)
        order, at = rng.permutation(n_pages), 0
        for r, x in enumerate(lens):
            need = -(-x // ps)
            self.table[r, :need] = order[at:at + need]
            self.kv[r] = x
            at += need
        self.refs[order[:at]] = 1
        self.refs[[p for p in held if self.refs[p] == 0]] = 3
        self.up()

    def up(self):
        self.d_table, self.d_kv, self.d_refs = _ints(self.table, self.dev), _ints(self.kv, self.dev), _ints(self.refs, self.dev)

    def desc(self, Hq=1, Hk=1, d=64, dtype=asl.ASL_BF16):
        return asl.make_pages(Hq, Hk, d, self.ps, self.n_pages, len(self.kv), self.width, dtype=dtype)

    def plan(self, ctx, rows, add, total, parent=None, pruned=None, guard=7):
        torch = _torch()
        n = len(rows)
        cu, slot = torch.full((n + 1 + guard,), 99, dtype=torch.int32, device=self.dev), torch.full((total + guard,), 99, dtype=torch.int64, device=self.dev)
        pos = torch.full((total + guard,), 99, dtype=torch.int32, device=self.dev)
        ctx.asl_pages_plan(self.desc(), _ints(rows, self.dev), _ints(add, self.dev), n, total, self.d_table, self.d_kv, self.d_refs, cu, slot, pos,
                           parent=None if parent is None else _ints(parent, self.dev), pruned=None if pruned is None else _ints(pruned, self.dev))
        for x, m in ((cu, n + 1), (slot, total), (pos, total)):
            assert bool((x[m:] == 99).all())
        return cu[:n + 1].cpu().numpy(), slot[:total].cpu().numpy(), pos[:total].cpu().numpy()

    def check(self, ctx, rows, add, total=None, parent=None, pruned=None):
        total = sum(add) if total is None else total
        got = self.plan(ctx, rows, add, total, parent, pruned)
        want = do.plan(self.table, self.kv, self.refs, rows, add, self.ps, total, parent, pruned)
        for a, b, what in zip(got, want, ("cu", "slot", "pos")):
            np.testing.assert_array_equal(a, b, err_msg=what)
        np.testing.assert_array_equal(self.d_kv.cpu().numpy(), self.kv)
        np.testing.assert_array_equal(self.d_refs.cpu().numpy(), self.refs)
        for r, x in enumerate(self.kv):
            np.testing.assert_array_equal(self.d_table[r, :-(-int(x) // self.ps)].cpu().numpy(), self.table[r, :-(-int(x) // self.ps)])
        return got


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("ps", [16, 64, 4096])
def test_plan_batches(ctx, gpu_device, ps, tree):
    lens = [0, 1, 15, 16, 17, 300, 64, 0, 5]
    b = _Book(gpu_device, 12, 600 // ps + 30, ps, 300, lens, held=range(0, 60, 3), seed=1)
    rows, add = [5, 0, 11, 3, 4, 8, 1], [33, 1, 0, 16, 70, 2, 250]
    parent = sum((_random_parents(m, m) for m in add), []) if tree else None
    b.check(ctx, rows, add, parent=parent, pruned=np.arange(12) * 1000)
    b.check(ctx, rows, add, total=sum(add) + 9, parent=None if parent is None else parent + [77] * 9)
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("n,add", [(1, [0]), (1, [1]), (1, [8191]), (1, [8192]), (1, [8193]), (3, [9000, 0, 7000]), (300, None), (4096, None), (1025, None)])
def test_plan_sizes(ctx, gpu_device, n, add):
    """Around the sizes at which the work is divided otherwise: requests of a thread, tokens of the one workgroup."""
    rng = np.random.default_rng(n)
    add = add if add is not None else rng.integers(0, 5, n).tolist()
    for tree in (False, True):
        b = _Book(gpu_device, n + 1, 9000 // 16 + 2, 16, sum(add) // 16 + n + 50, [3] * n, held=range(0, 40, 7), seed=n)
        parent = sum((_random_parents(m, m, root=0.01) for m in add), []) if tree else None
        b.check(ctx, rng.permutation(n).tolist(), add, parent=parent, pruned=rng.integers(0, 1000, n + 1) if tree else None)
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("total", [0, 5, 8192, 9000])
@pytest.mark.parametrize("tree", [False, True])
def test_plan_of_no_requests(ctx, gpu_device, total, tree):
    """No token has a slot or a position, whatever the lists held before."""
    torch = _torch()
    b = _Book(gpu_device, 3, 5, 16, 20, [30, 0, 7])
    slot, pos, cu = _longs(np.full(total, 3), gpu_device), _ints(np.full(total, 3), gpu_device), _ints([9], gpu_device)
    none = _ints([], gpu_device)
    ctx.asl_pages_plan(b.desc(), none, none, 0, total, b.d_table, b.d_kv, b.d_refs, cu, slot, pos, parent=_ints(np.zeros(total), gpu_device) if tree else None)
    assert cu.tolist() == [0] and torch.all(slot == -1) and torch.all(pos == -1)
    assert b.d_kv.tolist() == [30, 0, 7] and ctx.asl_device_fault() == 0


def test_plan_without_enough_pages(ctx, gpu_device):
    """The first request that does not get its pages, and all behind it, stay as they were: no slots, but positions."""
    b = _Book(gpu_device, 5, 20, 16, 12, [10, 20, 0, 5, 16], seed=2)
    _, slot, pos = b.check(ctx, [0, 1, 2, 3, 4], [10, 40, 100, 1, 3])
    assert np.all(slot[50:] == -1) and np.all(slot[:50] >= 0) and np.all(pos >= 0)
    assert ctx.asl_device_fault() == 0                       # no number was out of range
    b = _Book(gpu_device, 3, 2000, 16, 2000, [10, 20, 0], held=range(2000), seed=3)
    _, slot, _ = b.check(ctx, [2, 0, 1], [0, 6, 7])          # a full pool: what the last pages still hold room for
    assert list(slot >= 0) == [True] * 13
    _, slot, _ = b.check(ctx, [1, 0, 2], [1, 1, 0])          # and not a token more
    assert list(slot >= 0) == [True, False]
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("total", [0, 5, 12, 9000])
def test_plan_of_more_tokens_than_there_is_room_for(ctx, gpu_device, total):
    add = [5, 7, 1, 0, 9000, 2]
    b = _Book(gpu_device, 6, 700, 16, 1000, [3] * 6, seed=4)
    b.check(ctx, list(range(6)), add, total=total, parent=_random_parents(total, 1) if total == 12 else None)
    assert ctx.asl_device_fault() == 2
    b = _Book(gpu_device, 3, 700, 16, 100, [3] * 3, seed=4)
    got = b.plan(ctx, [0, 1, 2], [2 ** 31 - 1] * 3, 10)      # sums past 32 bits
    assert list(got[0]) == [0, 0, 0, 0] and np.all(got[1] == -1) and ctx.asl_device_fault() == 2
    np.testing.assert_array_equal(b.d_kv.cpu().numpy(), b.kv)


def test_plan_of_numbers_out_of_range(ctx, gpu_device):
    """Rows, lengths and parents that are none: their tokens get no slot, the others theirs."""
    for big, width in ((0, 20), (8300, 600)):                # in the one workgroup, and by the launch of its own
        b = _Book(gpu_device, 6, width, 16, 800, [3, 4, 5, 6, 7, 0], seed=5)
        b.kv[3] = -4
        b.kv[4] = width * 16 + 1
        b.up()
        add = [2, 3, 4, 5, 6, -7, 1, width * 16, big]
        rows = [0, 9, -1, 3, 4, 1, 6, 2, 5]
        b.check(ctx, rows, add, total=sum(max(x, 0) for x in add))
        assert ctx.asl_device_fault() == 2
    b = _Book(gpu_device, 2, 20, 16, 30, [3, 4], seed=5)     # a row twice: one of the requests has it
    got = b.plan(ctx, [0, 1, 0], [20, 20, 20], 60)
    assert ctx.asl_device_fault() == 2
    assert b.d_kv.tolist() == [23, 24] and int((b.d_refs > 0).sum()) == 4
    assert sorted([int((got[1][:20] >= 0).sum()), int((got[1][40:] >= 0).sum())]) == [0, 20]
    for big in (0, 8300):
        b = _Book(gpu_device, 2, 600, 16, 800, [3, 4], seed=6)
        parent = [-1, 0, 2, 1, 99, -5, 3] + [-1] + list(range(big - 1)) if big else [-1, 0, 2, 1, 99, -5, 3]
        b.check(ctx, [1, 0], [7, big], parent=parent)
        assert ctx.asl_device_fault() == 2


def test_plan_refusals(ctx, gpu_device):
    b = _Book(gpu_device, 2, 4, 16, 8, [1, 1])
    i = _ints([0, 1, 0], gpu_device)
    s = _longs([0] * 4, gpu_device)
    call = lambda n, total, refs=b.d_refs: ctx.asl_pages_plan(b.desc(), i, i, n, total, b.d_table, b.d_kv, refs, _ints([0] * 5000, gpu_device), s, i)
    for args, status in (((-1, 1), asl.ASL_EINVAL), ((4097, 1), asl.ASL_ENOMEM), ((1, -1), asl.ASL_EINVAL), ((1, 1, None), asl.ASL_EINVAL)):
        with pytest.raises(asl.AslError) as e:
            call(*args)
        assert e.value.status == status
    call(0, 3)
    assert ctx.asl_device_fault() == 0


# ------------------------------------------------------------------------------------------------------------------ tree
def _cu(n_q):
    return np.concatenate([[0], np.cumsum(n_q)])


def _tree(ctx, c, q, n_q, parent, Hq, groups=None, rows=None, scale=0.0, max_q=None, max_kv=None, pad=0):
    torch = _torch()
    dev, total = c.dev, int(sum(n_q))
    out = torch.full((max(total, 1), Hq, c.d + pad), float("nan"), dtype=_dt(c.dtype), device=dev)[:total, :, :c.d]
    lse = torch.full((Hq, total), float("nan"), dtype=torch.float32, device=dev)
    a = asl.make_attn(len(n_q), total, max_q if max_q is not None else max(n_q), max_kv if max_kv is not None else max(c.lens),
                      n_groups=len(groups) if groups else 0)
    gs = pl = None
    if groups:
        gs, pl = _ints(_cu([m for m, _ in groups]), dev), _ints([p for _, p in groups], dev)
    ctx.asl_tree_attention(c.desc(Hq, scale), a, q, c.k, c.v, c.table, c.kv_len, _ints(_cu(n_q), dev), _ints(parent, dev), out, lse=lse,
                           rows=None if rows is None else _ints(rows, dev), group_start=gs, prefix_len=pl)
    torch.cuda.synchronize()
    return out, lse


def _tree_oracle(c, q, n_q, parent, scale=0.0, rows=None):
    q, k, v = (x.double().cpu().numpy() for x in (q, c.k, c.v))
    parts, at = [], 0
    for b, n in enumerate(n_q):
        r = b if rows is None else rows[b]
        parts.append(do.attention(q[at:at + n], po.gather(k, c.host_table[r], c.lens[r]), po.gather(v, c.host_table[r], c.lens[r]),
                                  scale or c.d ** -0.5, parent[at:at + n]))
        at += n
    return (np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts], axis=1),
            np.concatenate([p[2] for p in parts]), np.concatenate([p[3] for p in parts]))


def _tree_case(ctx, dev, lens, n_q, Hq, Hk, d, ps, dtype, groups=None, seed=0, pad=0, gap=0, rows=None, scale=0.0, what="", chain=0.45, **bounds):
    shared, at = [], 0
    for m, p in groups or []:
        shared.append((at, at + m, min([p] + list(lens[at:at + m]))))
        at += m
    c = Cache(dev, lens, Hk, d, ps, dtype, seed, shared=shared, gap=gap)
    q = _queries(sum(n_q), Hq, d, dtype, dev, seed + 1, pad)
    parent = sum((_random_parents(n, seed + 10 * b, chain) for b, n in enumerate(n_q)), [])
    out, lse = _tree(ctx, c, q, n_q, parent, Hq, groups, rows, scale, pad=pad, **bounds)
    _check(out, lse, _tree_oracle(c, q, n_q, parent, scale, rows), d, max(lens), dtype, what)
    assert ctx.asl_device_fault() == 0
    return c, q, parent, out, lse


HEADS = [(4, 2, 64), (8, 8, 128), (28, 4, 128), (32, 2, 128), (6, 2, 80), (5, 1, 256), (3, 3, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hk,d", HEADS)
def test_tree_ragged_sequences(ctx, gpu_device, Hq, Hk, d, dtype):
    """Contexts of any length beside drafts of any size; sequences with fewer keys than nodes, with none, and without nodes."""
    _tree_case(ctx, gpu_device, [70, 5, 0, 200, 9, 130, 33, 1, 95], [17, 9, 3, 40, 0, 1, 33, 1, 31], Hq, Hk, d, 32, dtype, what="ragged")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 129, 300, 511, 512])
def test_tree_sizes(ctx, gpu_device, n, dtype):
    """Nodes around every tile height and word of bits, behind contexts around the tiles' borders."""
    for context in (0, 1, 31, 64, 100):
        _tree_case(ctx, gpu_device, [n + context, max(1, n // 2) + 130], [n, max(1, n // 2)], 8, 2, 64, 16, dtype, seed=n + context,
                   what="n %d context %d" % (n, context))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", ["chain", "star", "roots"])
def test_tree_shapes(ctx, gpu_device, shape, dtype):
    n, lens = 90, [90 + 77, 90 + 64, 90]
    parent = {"chain": list(range(-1, n - 1)), "star": [-1] + [0] * (n - 1), "roots": [-1] * n}[shape]
    c = Cache(gpu_device, lens, 2, 64, 16, dtype, 3)
    q = _queries(3 * n, 8, 64, dtype, gpu_device, 4)
    out, lse = _tree(ctx, c, q, [n] * 3, parent * 3, 8)
    _check(out, lse, _tree_oracle(c, q, [n] * 3, parent * 3), 64, max(lens), dtype, shape)
    if shape == "chain":                                     # what causal attention gives, up to rounding
        two, lse2 = _attend(ctx, c, q, [n] * 3, 8)
        _check(two, lse2, _tree_oracle(c, q, [n] * 3, parent * 3), 64, max(lens), dtype, shape)
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps", [16, 32, 64, 256, 4096])
def test_tree_page_sizes(ctx, gpu_device, ps, dtype):
    _tree_case(ctx, gpu_device, [700, 31, ps, ps + 1], [21, 30, 12, 1], 8, 2, 128, ps, dtype, what="ps %d" % ps)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [4097, 20000, 70001])
def test_tree_long_contexts(ctx, gpu_device, n, dtype):
    _tree_case(ctx, gpu_device, [n], [9], 8, 2, 128, 64, dtype, what="long %d" % n)
    _tree_case(ctx, gpu_device, [n // 4, 1 + n // 9], [20, 2], 14, 2, 64, 16, dtype, seed=5, what="long %d" % n)


@pytest.mark.parametrize("d,Hq,Hk", [(128, 32, 8), (64, 16, 8), (128, 28, 4), (72, 8, 8), (128, 8, 8)])
@pytest.mark.parametrize("lo,hi", [(3, 8), (16, 33), (60, 61), (100, 180)])
def test_tree_tiles(ctx, gpu_device, lo, hi, d, Hq, Hk):
    """Batches that take the tiles of 64 and of 128 rows, drafts that end inside and across them."""
    n_q = [lo + (7 * i) % (hi - lo) for i in range(9)]
    lens = [900 + 61 * i + n for i, n in enumerate(n_q)]
    _tree_case(ctx, gpu_device, lens, n_q, Hq, Hk, d, 16, "bf16", seed=lo, what="tiles", max_kv=1 << 20)


def test_tree_sequences_longer_than_stated(ctx, gpu_device):
    """max_kv_len decides how items are cut, not what is computed: without pieces to join too."""
    n_q, lens = [32] * 24, [9000, 8500] + [40 + 9 * i for i in range(22)]
    rng = random.Random(5)
    c = Cache(gpu_device, lens, 8, 64, 64, "bf16", 5)
    parent = sum([_random_parents(n, rng.randrange(99)) for n in n_q], [])
    q = _queries(sum(n_q), 32, 64, "bf16", gpu_device, 6)
    ref = _tree_oracle(c, q, n_q, parent)
    for stated in (2048, 9000):
        out, lse = _tree(ctx, c, q, n_q, parent, 32, max_kv=stated)
        _check(out, lse, ref, 64, max(lens), "bf16", "stated %d" % stated)
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,G", [(128, 4), (64, 7), (256, 2), (80, 1)])
@pytest.mark.parametrize("groups,own,n_q", [
    ([(5, 300)], [4, 2, 33, 64, 200], [4, 1, 7, 10, 12]),
    ([(3, 129), (1, 70), (4, 512)], [5, 6, 7, 3, 40, 1, 2, 17], [1, 2, 3, 1, 5, 1, 2, 4]),
    ([(17, 2112)], [20 + i for i in range(17)], [1 + i for i in range(17)]),
    ([(6, 1500)], [30, 31, 32, 33, 34, 35], [12, 13, 14, 15, 16, 30]),
])
def test_tree_shared_prefix(ctx, gpu_device, groups, own, n_q, d, G, dtype):
    lens = [p for m, p in groups for _ in range(m)]
    lens = [p + x for p, x in zip(lens, own)]
    for max_kv in (max(lens), 1 << 20):
        _tree_case(ctx, gpu_device, lens, n_q, 8 * G if d == 128 else 2 * G, 8 if d == 128 else 2, d, 16, dtype, groups=groups, what="shared",
                   max_kv=max_kv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_prefix_longer_than_the_contexts(ctx, gpu_device, dtype):
    """A stated prefix that reaches into the drafts, or past a sequence's end, members that end before it: only what all nodes see is shared."""
    P = 2112
    lens = [P + 3 * i for i in range(17)] + [2000, 700, 63, 64, 0, 1]
    n_q = [1 + 13 * (i % 4) for i in range(23)]
    for kv in (max(lens), 1 << 20):
        c = Cache(gpu_device, lens, 8, 128, 16, dtype, 3, shared=[(0, 17, P)])
        for r in range(17, 23):                              # the short ones hold copies of the prefix
            for x in c.pages_t:
                for t in range(-(-lens[r] // 16)):
                    m = min(16, lens[r] - 16 * t)
                    x[c.host_table[r, t], :, :m] = x[c.host_table[0, t], :, :m]
        q = _queries(sum(n_q), 8, 128, dtype, gpu_device, 9)
        parent = sum((_random_parents(n, n) for n in n_q), [])
        for stated in (P, 10 ** 6, -5):
            out, lse = _tree(ctx, c, q, n_q, parent, 8, groups=[(23, stated)], max_kv=kv)
            _check(out, lse, _tree_oracle(c, q, n_q, parent), 128, max(lens), dtype, "stated %d" % stated)
    assert ctx.asl_device_fault() == 0


def test_tree_token_strides_past_32_bits(ctx, gpu_device):
    """Tokens of one page a megabyte apart, all heads of a token beside each other: places past 2^31 bytes inside the page."""
    torch = _torch()
    dev, L, n, ps, Hk, d, tok = gpu_device, 3000, 40, 4096, 8, 64, 1 << 19
    k, v = (torch.empty(ps * tok, dtype=torch.bfloat16, device=dev) for _ in range(2))      # whole pages: slots behind the end are read too
    g = torch.Generator().manual_seed(3)
    kv = [torch.randn((L, Hk, d), generator=g).to(torch.bfloat16) for _ in range(2)]
    for x, y in zip((k, v), kv):
        x.as_strided((L, Hk, d), (tok, d, 1)).copy_(y.to(dev))
    q = _queries(n, 32, d, "bf16", dev, 4)
    parent = _random_parents(n, 5)
    out = torch.empty((n, 32, d), dtype=torch.bfloat16, device=dev)
    lse = torch.empty((32, n), dtype=torch.float32, device=dev)
    desc = asl.make_pages(32, Hk, d, ps, 1, 1, 1, strides=(0, d, tok))
    for max_kv in (L, 1 << 20):
        ctx.asl_tree_attention(desc, asl.make_attn(1, n, n, max_kv), q, k, v, _ints([0], dev), _ints([L], dev), _ints([0, n], dev), _ints(parent, dev),
                               out, lse=lse)
        ref = do.attention(q.double().cpu().numpy(), *(x.double().numpy().transpose(1, 0, 2) for x in kv), d ** -0.5, parent)
        _check(out, lse, ref, d, L, "bf16", "strides")
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_strides_rows_and_scale(ctx, gpu_device, dtype):
    torch = _torch()
    lens = [90, 40, 17]
    c = Cache(gpu_device, lens, 2, 64, 16, dtype, 2, gap=64)
    q = _queries(20, 8, 64, dtype, gpu_device, 3, pad=24)
    rows, n_q, parent = [2, 0, 2], [9, 6, 5], _random_parents(9, 1) + _random_parents(6, 2) + _random_parents(5, 3)
    out, lse = _tree(ctx, c, q, n_q, parent, 8, None, rows, 0.37, pad=24)
    _check(out, lse, _tree_oracle(c, q, n_q, parent, 0.37, rows), 64, 90, dtype, "strides")
    qt = q.transpose(0, 1).contiguous().transpose(0, 1)
    out2, lse2 = _tree(ctx, c, qt, n_q, parent, 8, None, rows, 0.37)
    assert torch.equal(out2, out) and torch.equal(lse2, lse)
    for mq, mk in ((1, 1), (0, 0), (512, 1 << 24)):          # bounds only cut the work
        out, lse = _tree(ctx, c, q, n_q, parent, 8, None, rows, 0.37, max_q=mq, max_kv=mk)
        _check(out, lse, _tree_oracle(c, q, n_q, parent, 0.37, rows), 64, 90, dtype, "bounds")
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("odd", ["nan", "inf", "both"])
def test_tree_numbers_that_are_none_reach_only_what_sees_them(ctx, gpu_device, odd, dtype):
    """An infinite or NaN key or value of a node changes that node and its descendants, and nobody else."""
    torch = _torch()
    n, bad = 40, 5
    for Hq, Hk, lens, mk in ((8, 2, [n + 70, n + 33, n], None), (32, 8, [n + 900] * 9, 1 << 20)):
        c = Cache(gpu_device, lens, Hk, 64, 16, dtype, 3)
        q = _queries(n * len(lens), Hq, 64, dtype, gpu_device, 4)
        parent = _random_parents(n, 8)
        parent[bad + 1] = bad
        clean, lse0 = _tree(ctx, c, q, [n] * len(lens), parent * len(lens), Hq, max_kv=mk)
        below = [bad in do.path_to(parent, i) for i in range(n)]
        assert 2 <= sum(below) < n - 5
        for r, L in enumerate(lens):
            at = L - n + bad
            page, slot = c.host_table[r, at // 16], at % 16
            if odd != "inf":
                c.v[page, :, slot, 3] = float("nan")
            if odd != "nan":
                c.v[page, :, slot, 9] = float("inf")
                c.v[page, :, slot, 11] = float("-inf")
            if odd == "both":
                c.k[page, :, slot, 2] = float("nan")
        out, lse = _tree(ctx, c, q, [n] * len(lens), parent * len(lens), Hq, max_kv=mk)
        sees = torch.tensor(below * len(lens), device=gpu_device)
        assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse[:, ~sees], lse0[:, ~sees])
        hit = out[sees]
        if odd == "both":
            assert bool(hit.isnan().all()) and bool(lse[:, sees].isnan().all())
        else:
            if odd == "nan":
                assert bool(hit[..., 3].isnan().all())
                rest = [e for e in range(64) if e != 3]
            else:
                assert bool((hit[..., 9] == float("inf")).all()) and bool((hit[..., 11] == float("-inf")).all())
                rest = [e for e in range(64) if e not in (9, 11)]
            assert torch.equal(hit[..., rest], clean[sees][..., rest]) and torch.equal(lse[:, sees], lse0[:, sees])
    assert ctx.asl_device_fault() == 0


def test_tree_parents_out_of_range_stand_for_none(ctx, gpu_device):
    for kv in (None, 1 << 20):
        c = Cache(gpu_device, [80, 300], 8, 64, 16, "bf16", 5)
        q = _queries(40, 32, 64, "bf16", gpu_device, 6)
        parent = _random_parents(20, 1) + _random_parents(20, 2)
        parent[3], parent[7], parent[25], parent[30], parent[0] = 3, 2 ** 31 - 1, -2, -2 ** 31, 19
        out, lse = _tree(ctx, c, q, [20, 20], parent, 32, max_kv=kv)
        _check(out, lse, _tree_oracle(c, q, [20, 20], parent), 64, 300, "bf16", "parents")
        assert ctx.asl_device_fault() == 2


def test_tree_drafts_that_are_too_long_are_left_out(ctx, gpu_device):
    torch = _torch()
    c = Cache(gpu_device, [600, 300], 2, 64, 16, "bf16", 5)
    n_q, parent = [513, 20], list(range(-1, 512)) + _random_parents(20, 2)
    q = _queries(533, 8, 64, "bf16", gpu_device, 6)
    with pytest.raises(asl.AslError, match="512") as e:
        _tree(ctx, c, q, n_q, parent, 8)
    assert e.value.status == asl.ASL_EUNSUPPORTED
    out, lse = _tree(ctx, c, q, n_q, parent, 8, max_q=20)    # what cu_q says is more than what was stated
    assert ctx.asl_device_fault() == 2
    assert bool(out[:513].isnan().all()) and bool(lse[:, :513].isnan().all())
    ref = _tree_oracle(c, q, n_q, parent)
    _check(out[513:], lse[:, 513:], [ref[0][513:], ref[1][:, 513:], ref[2][513:], ref[3][513:]], 64, 600, "bf16", "the other one")
    with pytest.raises(asl.AslError, match="CAUSAL"):
        ctx.asl_tree_attention(c.desc(8), asl.make_attn(1, 5, 5, 9, causal=False), q, c.k, c.v, c.table, c.kv_len, _ints([0, 5], gpu_device),
                               _ints(parent, gpu_device), q)


# ---------------------------------------------------------------------------------------------------------------- accept
def _accept(ctx, c, layers, rows, counts, path, n_path, table=None):
    torch = _torch()
    dev = c.dev
    k_ptrs, v_ptrs = (torch.tensor([x.data_ptr() for x in c.pages_t[i::2][:layers]] + [0], dtype=torch.int64, device=dev) for i in (0, 1))
    ctx.asl_pages_accept(c.desc(), k_ptrs, v_ptrs, layers, _ints(rows, dev), _ints(_cu(counts), dev), _ints(path, dev), _ints(n_path, dev), len(rows),
                         c.table, c.kv_len, c.refs)
    torch.cuda.synchronize()


def _accepted(c, layers, rows, counts, paths):
    """The oracle's pages, lengths and counts."""
    kv, refs = np.array(c.lens, dtype=np.int64), c.refs_host.copy()
    pages = [x.float().cpu().numpy().copy() for x in c.pages_t]
    do.accept(c.host_table, kv, refs, [(pages[2 * i], pages[2 * i + 1]) for i in range(layers)], rows, counts, paths, c.ps)
    return pages, kv, refs


def _same_pages(c, pages):
    for x, y in zip(c.pages_t, pages):
        np.testing.assert_array_equal(x.float().cpu().numpy(), y)


def _padded(paths, width):
    return np.array([list(p) + [-9] * (width - len(p)) for p in paths], dtype=np.int64).reshape(len(paths), width)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,d,ps,layers", [(2, 64, 16, 1), (8, 128, 16, 3), (1, 80, 64, 2), (3, 8, 32, 2), (4, 256, 4096, 1), (40, 256, 16, 1)])
def test_accept(ctx, gpu_device, Hk, d, ps, layers, dtype):
    rng = random.Random(d)
    counts = [1, 5, 16, 17, 40, 64, 9, 3]
    lens = [1, 5 + 11, 16 + 16, 17 + 100, 40 + 3, 64 + 15, 9, 3 + 33, 50]
    paths = [do.path_to(p, rng.randrange(len(p))) for p in ([_random_parents(n, n) for n in counts])]
    paths[1], paths[6] = [], list(range(9))                  # nothing is kept, everything is
    paths[4] = sorted(rng.sample(range(40), 30))
    c = Cache(gpu_device, lens, Hk, d, ps, dtype, 1, layers=layers)
    rows = [3, 1, 0, 2, 5, 4, 7, 6]
    perm = lambda x: [x[r] for r in rows]
    want = _accepted(c, layers, rows, perm(counts), perm(paths))
    _accept(ctx, c, layers, rows, perm(counts), _padded(perm(paths), 41), [len(p) for p in perm(paths)])
    _same_pages(c, want[0])
    np.testing.assert_array_equal(c.kv_len.cpu().numpy(), want[1])
    np.testing.assert_array_equal(c.refs.cpu().numpy(), want[2])
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("stay", [0, 1, 100, 511])
def test_accept_long_paths(ctx, gpu_device, stay):
    """Paths of up to 512 nodes whose places overlap their nodes', over many rounds of the workgroup."""
    rng = random.Random(stay)
    m = 700
    path = list(range(stay)) + sorted(rng.sample(range(stay, m), 512 - stay))
    c = Cache(gpu_device, [m + 21], 8, 128, 16, "bf16", 2)
    want = _accepted(c, 1, [0], [m], [path])
    _accept(ctx, c, 1, [0], [m], _padded([path], 512), [512])
    _same_pages(c, want[0])
    assert c.kv_len.tolist() == [512 + 21] and np.array_equal(c.refs.cpu().numpy(), want[2])
    assert ctx.asl_device_fault() == 0


def test_accept_without_layers(ctx, gpu_device):
    """The lengths and the pages alone: a draft that is dropped."""
    c = Cache(gpu_device, [100, 40], 1, 64, 16, "bf16", 2)
    _, kv, refs = _accepted(c, 0, [1, 0], [40, 37], [[], []])
    _accept(ctx, c, 0, [1, 0], [40, 37], np.zeros((2, 0)), [0, 0])
    assert np.array_equal(c.kv_len.cpu().numpy(), kv) and np.array_equal(c.refs.cpu().numpy(), refs)
    assert list(kv) == [63, 0] and ctx.asl_device_fault() == 0


def test_accept_numbers_out_of_range(ctx, gpu_device):
    """Lists that are none leave their row as it was; a path ends where it does not ascend."""
    torch = _torch()
    lens = [50, 50, 50, 50, 50, 50, 50]
    c = Cache(gpu_device, lens, 2, 64, 16, "bf16", 2)
    counts = [10, 10, 10, 10, 51, 10, 10]
    rows = [0, 1, 9, 3, 4, 5, 6]
    path = _padded([[0, 2, 1, 5], [3, 10, 11], [0, 1], [0, 2], [0, 1], [-1, 3], [4, 4, 9]], 4)
    n_path = [4, 3, 2, 5, 2, 2, 3]
    kept = {0: [0, 2], 1: [3], 5: [], 6: [4]}
    want = _accepted(c, 1, list(kept), [10] * 4, list(kept.values()))
    _accept(ctx, c, 1, rows, counts, path, n_path)
    assert ctx.asl_device_fault() == 2
    _same_pages(c, want[0])
    assert np.array_equal(c.kv_len.cpu().numpy(), want[1]) and np.array_equal(c.refs.cpu().numpy(), want[2])
    c.kv_len.copy_(_ints(lens, gpu_device))
    c2 = Cache(gpu_device, lens, 2, 64, 16, "bf16", 2)       # the counts of pieces that are there are zero again: the next call is right
    want = _accepted(c2, 1, range(7), [10] * 7, [[1, 7]] * 7)
    _accept(ctx, c2, 1, range(7), [10] * 7, _padded([[1, 7]] * 7, 2), [2] * 7)
    _same_pages(c2, want[0])
    assert np.array_equal(c2.kv_len.cpu().numpy(), want[1]) and ctx.asl_device_fault() == 0


def test_accept_leaves_rows_without_pages_alone(ctx, gpu_device):
    """A row that the pool had no page for has no draft: with the plan's slots its own tokens stay."""
    torch = _torch()
    c = Cache(gpu_device, [40, 90, 33], 2, 64, 16, "bf16", 2)
    slot = torch.arange(30, device=gpu_device)
    slot[10:20] = -1
    want = _accepted(c, 1, [0, 2], [10, 10], [[0, 3], [5]])
    k_ptrs, v_ptrs = (torch.tensor([x.data_ptr()], dtype=torch.int64, device=gpu_device) for x in (c.k, c.v))
    cu, path, n_path = _ints([0, 10, 20, 30], gpu_device), _ints([[0, 3], [1, 2], [5, 0]], gpu_device), _ints([2, 2, 1], gpu_device)
    call = lambda slot: ctx.asl_pages_accept(c.desc(), k_ptrs, v_ptrs, 1, _ints([0, 1, 2], gpu_device), cu, path, n_path, 3, c.table, c.kv_len,
                                             c.refs, slot=slot)
    call(slot)
    torch.cuda.synchronize()
    _same_pages(c, want[0])
    assert np.array_equal(c.kv_len.cpu().numpy(), want[1]) and np.array_equal(c.refs.cpu().numpy(), want[2])
    assert ctx.asl_device_fault() == 0
    call(slot[:25])                                          # cu goes past the list: the last row is left out
    assert ctx.asl_device_fault() == 2 and c.kv_len.tolist() == [24, 90, 24 + 0]


def test_accept_refusals(ctx, gpu_device):
    c = Cache(gpu_device, [50], 2, 64, 16, "bf16", 2)
    for width, n_path, status in ((513, 1, asl.ASL_EUNSUPPORTED),):
        with pytest.raises(asl.AslError) as e:
            _accept(ctx, c, 1, [0], [10], np.zeros((1, width)), [n_path])
        assert e.value.status == status
    with pytest.raises(asl.AslError) as e:
        _accept(ctx, c, -1, [0], [10], np.zeros((1, 1)), [1])
    assert e.value.status == asl.ASL_EINVAL
    _accept(ctx, c, 1, [], [], np.zeros((0, 1)), [])
    assert ctx.asl_device_fault() == 0


# --------------------------------------------------------------------------------------------------------------- together
def _steps(ctx, dev, dtype, graph, steps=5, seed=3):
    """Drafting steps over a batch as a program makes them, the trees and the paths given: plan, rotation into the pages, attention, accept.
    Returns each step's positions, rotated queries and outputs, and what the cache holds."""
    torch = _torch()
    Hq, Hk, d, ps, n, most, layers = 8, 2, 64, 16, 3, 12, 2
    e = asl.ASL_BF16 if dtype == "bf16" else asl.ASL_F32
    rng, rnd = np.random.default_rng(seed), random.Random(seed)
    b = _Book(dev, n + 1, 40, ps, 60, [100, 37, 0, 5], held=range(0, 20, 4), seed=seed)
    total = n * most
    g = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g).to(_dt(dtype)).to(dev)
    kp, vp = normal(layers, b.n_pages, Hk, ps, d), normal(layers, b.n_pages, Hk, ps, d)
    k_ptrs, v_ptrs = (torch.tensor([x.data_ptr() for x in p], dtype=torch.int64, device=dev) for p in (kp, vp))
    f = asl.rotation_freqs(d, kind=asl.ASL_FREQS_PARTS, factor=4.0, context=64.0, low=1.0, high=4.0).to(dev)
    rot, pages, attn = asl.make_rotation(Hq, Hk, d, dtype=e), b.desc(Hq, Hk, d, e), asl.make_attn(n, total, most, 400)
    rows, pruned = _ints([3, 0, 1], dev), _ints([500, 3, 0, 70], dev)
    add, parent, path, n_path = (_ints(np.zeros(s), dev) for s in ((n,), (total,), (n, most), (n,)))
    cu, slot, pos = _ints(np.zeros(n + 1), dev), _longs(np.zeros(total), dev), _ints(np.zeros(total), dev)
    x = torch.zeros((layers, total, Hq + 2 * Hk, d), dtype=_dt(dtype), device=dev)
    q, out = torch.zeros((layers, total, Hq, d), dtype=_dt(dtype), device=dev), torch.zeros((layers, total, Hq, d), dtype=_dt(dtype), device=dev)

    def step():
        ctx.asl_pages_plan(pages, rows, add, n, total, b.d_table, b.d_kv, b.d_refs, cu, slot, pos, parent=parent, pruned=pruned)
        for l in range(layers):
            ctx.asl_rotate_write(pages, rot, x[l, :, :Hq], x[l, :, Hq:Hq + Hk], x[l, :, Hq + Hk:], pos, slot, f, q[l], kp[l], vp[l])
            ctx.asl_tree_attention(pages, attn, q[l], kp[l], vp[l], b.d_table, b.d_kv, cu, parent, out[l], rows=rows)
        ctx.asl_pages_accept(pages, k_ptrs, v_ptrs, layers, rows, cu, path, n_path, n, b.d_table, b.d_kv, b.d_refs, slot=slot)

    recorded = None
    results = []
    for s in range(steps):
        sizes = [rnd.randint(1, most) for _ in range(n)]
        trees = [_random_parents(m, rnd.randrange(1000)) for m in sizes]
        paths = [do.path_to(t, rnd.randrange(len(t)))[:rnd.randint(0, 5)] for t in trees]
        flat = sum(trees, [])
        add.copy_(_ints(sizes, dev)), parent.copy_(_ints(flat + [-7] * (total - len(flat)), dev))
        path.copy_(_ints(_padded(paths, most), dev)), n_path.copy_(_ints([len(p) for p in paths], dev))
        x.copy_(normal(*x.shape)), out.zero_()
        lens_before, table_before = b.d_kv.cpu().numpy(), None
        if not graph:
            step()
        else:
            if recorded is None:
                recorded = torch.cuda.CUDAGraph()
                with torch.cuda.graph(recorded):
                    step()
            recorded.replay()
        torch.cuda.synchronize()
        used = sum(sizes)
        results.append(dict(sizes=sizes, trees=trees, paths=paths, before=lens_before, pos=pos[:used].cpu().numpy(), slot=slot.cpu().numpy(),
                            q=q[:, :used].double().cpu().numpy(), x=x[:, :used].double().cpu().numpy(), out=out.double().cpu().numpy()))
    assert ctx.asl_device_fault() == 0
    cache = dict(k=kp.float().cpu().numpy(), v=vp.float().cpu().numpy(), kv=b.d_kv.cpu().numpy(), refs=b.d_refs.cpu().numpy(), book=b, f=f.cpu().numpy())
    return results, cache


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_of_a_batch(ctx, gpu_device, dtype):
    """Positions, rotated queries, attention and the cache's content against a program that keeps each sequence as a list of tokens."""
    results, cache = _steps(ctx, gpu_device, dtype, graph=False)
    Hq, Hk, d, b, layers = 8, 2, 64, cache["book"], 2
    rows, pruned = [3, 0, 1], [500, 3, 0, 70]
    np.testing.assert_array_equal(cache["refs"][b.refs == 3], 3)
    table = b.d_table.cpu().numpy()
    grown = {r: [] for r in rows}                            # each row's kept tokens: (rotated k, v) of each layer
    for s in results:
        at = 0
        for i, r in enumerate(rows):
            m, tree = s["sizes"][i], s["trees"][i]
            L = 0 + int(b.kv[r]) + len(grown[r])
            assert s["before"][r] == L
            pos = [L + len(do.path_to(tree, j)) - 1 + pruned[r] for j in range(m)]
            np.testing.assert_array_equal(s["pos"][at:at + m], pos)
            for l in range(layers):
                x = s["x"][l, at:at + m]
                y, reach = do.rotate(x[:, :Hq + Hk], pos, cache["f"])
                tol = _turn_bound(y, reach, np.array(pos)[:, None, None], dtype)
                assert np.all(np.abs(s["q"][l, at:at + m] - y[:, :Hq]) <= tol[:, :Hq])
            grown[r] += [(s["x"][:, at + j], pos[j]) for j in s["paths"][i]]
            at += m
    for r in rows:
        L = int(b.kv[r]) + len(grown[r])
        assert cache["kv"][r] == L
        for l in range(layers):
            k, v = (po.gather(cache[x][l].astype(np.float64), table[r], L)[:, int(b.kv[r]):] for x in ("k", "v"))
            for t, (x, p) in enumerate(grown[r]):
                np.testing.assert_array_equal(v[:, t], x[l, Hq + Hk:])
                y, reach = do.rotate(x[l, None, Hq:Hq + Hk], [p], cache["f"])
                assert np.all(np.abs(k[:, t] - y[0]) <= _turn_bound(y, reach, p, dtype)[0])


def test_steps_replayed_as_a_graph(ctx, gpu_device):
    """The captured step, replayed while lists and lengths go on, gives what the single calls give, bit for bit."""
    eager, cache = _steps(ctx, gpu_device, "bf16", graph=False, steps=8)
    replayed, cache2 = _steps(ctx, gpu_device, "bf16", graph=True, steps=8)
    for a, b in zip(eager, replayed):
        for key in ("pos", "slot", "q", "out", "before"):
            np.testing.assert_array_equal(a[key], b[key], err_msg=key)
    for key in ("k", "v", "kv", "refs"):
        np.testing.assert_array_equal(cache[key], cache2[key], err_msg=key)


def test_calls_on_another_stream_and_without_work(ctx, gpu_device):
    torch = _torch()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _tree_case(ctx, gpu_device, [300, 70], [20, 9], 8, 2, 64, 16, "bf16", what="stream")
        _rotated(ctx, gpu_device, 5, 2, 1, 64, 64, True, "bf16")
    side.synchronize()
    c = Cache(gpu_device, [10], 1, 64, 16, "bf16")
    e = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=gpu_device)
    i = _ints([0, 0], gpu_device)
    ctx.asl_tree_attention(c.desc(2), asl.make_attn(1, 0, 0, 10), e, c.k, c.v, c.table, c.kv_len, i, i[:0], e)
    ctx.asl_tree_attention(c.desc(2), asl.make_attn(0, 0, 0, 0), e, c.k, c.v, c.table, c.kv_len, i, i[:0], e)
    assert ctx.asl_device_fault() == 0


def test_tree_is_reproducible(ctx, gpu_device):
    torch = _torch()
    c, q, parent, out, lse = _tree_case(ctx, gpu_device, [2000 + 40 * i for i in range(12)], [17 + i for i in range(12)], 32, 8, 128, 64, "bf16", what="again")
    n_q = [17 + i for i in range(12)]
    for _ in range(50):
        o, l = _tree(ctx, c, q, n_q, parent, 32)
        assert torch.equal(o, out) and torch.equal(l, lse)


def test_rows_behind_the_last_sequence_stay(ctx, gpu_device):
    """out and lse have room for more nodes than the lists have, as where the lists are a replayed step's."""
    torch = _torch()
    for n_q, d, lens in (([20, 9, 40], 128, [3000, 70, 900]), ([3, 2, 1], 64, [30, 7, 90])):
        total, used = 96, sum(n_q)
        c = Cache(gpu_device, lens, 2, d, 64, "bf16", 5)
        parent = sum([_random_parents(n, n) for n in n_q], []) + [-1] * (total - used)
        q = _queries(total, 8, d, "bf16", gpu_device, 6)
        out, lse = torch.full((total, 8, d), 7.0, dtype=torch.bfloat16, device=gpu_device), torch.full((8, total), 7.0, device=gpu_device)
        ctx.asl_tree_attention(c.desc(8), asl.make_attn(3, total, 64, 4096), q, c.k, c.v, c.table, c.kv_len, _ints(_cu(n_q), gpu_device),
                               _ints(parent, gpu_device), out, lse=lse)
        assert torch.all(out[used:] == 7.0) and torch.all(lse[:, used:] == 7.0)
        ref = _tree_oracle(c, q[:used], n_q, parent[:used])
        _check(out[:used], lse[:, :used], ref, d, max(lens), "bf16", "room")
    assert ctx.asl_device_fault() == 0


@pytest.mark.parametrize("nodes,page_size", [(5, 16), (40, 64)])
def test_the_drafting_example(ctx, gpu_device, nodes, page_size):
    """examples/draft_pruned.py: positions and lengths, and every step's attention over what was kept so far against the oracle."""
    import importlib.util
    import os
    torch = _torch()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "draft_pruned.py")
    spec = importlib.util.spec_from_file_location("draft_pruned", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    Hq, Hk, d, N, keep, n = 8, 2, 64, 1000, 200, 3
    r = example.run(Hq=Hq, Hk=Hk, d=d, N=N, W=16, budget=keep, sequences=n, nodes=nodes, steps=6, page_size=page_size)
    assert r["fault"] == 0 and r["left"] == 0
    f = lambda x: x.double().cpu().numpy()
    idx, k, v = r["idx"].cpu().numpy(), f(r["k"]), f(r["v"])
    have = [[np.stack([x[h][idx[h]] for h in range(Hk)]) for x in (k, v)] for _ in range(n)]      # each row's K and V [Hk, tokens, d]
    for s, step in enumerate(r["history"]):
        at = 0
        rotated = torch.empty_like(step["x"][:, Hq:Hq + Hk])
        ctx.asl_rotate(asl.make_rotation(0, Hk, d), None, step["x"][:, Hq:Hq + Hk], step["pos"], r["freqs"], None, rotated)
        for b, (tree, kept) in enumerate(zip(step["trees"], step["paths"])):
            m = len(tree)
            pos = [N - keep + have[b][0].shape[1] + len(do.path_to(tree, i)) - 1 for i in range(m)]
            np.testing.assert_array_equal(step["pos"][at:at + m].cpu().numpy(), pos)
            new = [f(x[at:at + m]).transpose(1, 0, 2) for x in (rotated, step["x"][:, Hq + Hk:])]
            K, V = (np.concatenate([x, y], axis=1) for x, y in zip(have[b], new))
            ref = do.attention(f(step["q"][at:at + m]), K, V, d ** -0.5, tree)
            tol, _ = _bounds(d, K.shape[1], "bf16", ref)
            assert np.all(np.abs(f(step["out"][at:at + m]) - ref[0]) <= tol), (s, b)
            have[b] = [np.concatenate([x, y[:, kept]], axis=1) for x, y in zip(have[b], new)]
            at += m
    assert r["lengths"] == [keep] + [x[0].shape[1] for x in have]
