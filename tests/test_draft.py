"""Drafting over the paged cache without a GPU: refusals, the pieces of a rotation, frequencies, the binding, the oracle's own pins."""
import ctypes
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

from oracle import draft_oracle as do
from oracle import paged_oracle as po
from paper_2601_07667_amd import asl as libasl
from test_bound import ROOT


@pytest.fixture(scope="module")
def client(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("draft") / "draft_client")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2601_07667_amd", "csrc"), os.path.join(ROOT, "tests", "draft_client.cpp"),
                    "-o", exe], check=True)

    def ask(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", check=True, capture_output=True, text=True).stdout
        return out.splitlines()
    return ask


GOOD = dict(Hq=8, Hk=2, d=128, dtype=0, rot=128, pairs=0, flags=0, qt=1024, qh=128, kt=256, kh=128, vt=256, vh=128, qot=1024, qoh=128,
            kot=256, koh=128)


@pytest.mark.parametrize("change,status,word", [
    ({}, 0, ""), (dict(dtype=1, pairs=1, flags=1), 0, ""), (dict(rot=2), 0, ""), (dict(rot=66), 0, ""), (dict(Hq=0), 0, ""),
    (dict(Hk=0), 0, ""), (dict(qt=0, qh=0), 0, ""), (dict(qt=1023, kh=3), 0, ""), (dict(d=2, rot=2), 0, ""), (dict(d=2048, rot=2048), 0, ""),
    (dict(Hq=-1), -1, "heads"), (dict(Hk=-1), -1, "heads"), (dict(d=0), -1, "rot_dim"), (dict(rot=0), -1, "rot_dim"),
    (dict(rot=130), -1, "rot_dim"), (dict(rot=63), -1, "rot_dim"), (dict(pairs=2), -1, "pairs"), (dict(flags=2), -1, "flags"),
    (dict(dtype=2), -4, "dtype"), (dict(d=129, rot=128), -4, "even"), (dict(d=2050), -4, "2048"), (dict(Hq=65536), -4, "65535"),
    (dict(Hk=65536), -4, "65535"), (dict(qh=-1), -1, "stride"), (dict(koh=-128), -1, "stride"), (dict(vt=-2), -1, "stride"),
])
def test_rotations_are_checked(client, change, status, word):
    got = client(["rotation " + " ".join(str(x) for x in {**GOOD, **change}.values())])[0]
    assert int(got.split()[0]) == status and word in got


def test_batches_of_trees_are_checked(client):
    assert [int(x.split()[0]) for x in client(["tree 1 512", "tree 1 0", "tree 0 5", "tree 1 513"])] == [0, 0, -1, -4]
    assert client(["null"]) == ["-1 -1 -1"]


def test_the_items_that_trees_take(client):
    """Few rows or little work: split items, joined in the launch where there are few keys; else tiles of 128 rows, never of 64, with nothing to
    join where there are many tiles of few keys; prefixes apart where that saves enough and a sequence's own rows fit a tile; pieces never
    more than the workspace has room for."""
    # total_q, heads of a group, KV heads, sequences, groups, nodes, keys, bytes of a key
    want = {(5 * 9, 2, 2, 5, 0, 9, 500, 256): (16, 0, 1, 0), (64, 4, 8, 64, 0, 1, 2100, 4096): (16, 0, 0, 0), (5, 4, 8, 1, 0, 5, 2048, 4096): (16, 0, 1, 0),
            (32 * 32, 4, 8, 32, 0, 32, 2580, 4096): (128, 0, 0, 1), (32 * 32, 4, 8, 32, 0, 32, 8193, 4096): (128, 0, 0, 0), (60, 7, 4, 1, 0, 60, 131149, 2048): (128, 0, 0, 0),
            (48 * 12, 7, 4, 48, 8, 12, 2302, 2048): (128, 128, 0, 0), (16 * 12, 4, 8, 16, 0, 12, 8192, 4096): (128, 0, 0, 0),
            (48 * 12, 7, 4, 48, 8, 12, 1000, 2048): (128, 0, 0, 1), (48 * 20, 7, 4, 48, 8, 20, 2302, 2048): (128, 0, 0, 1),
            (4096 * 512, 8, 8, 4096, 0, 512, 1 << 20, 4096): (128, 0, 0, 0), (1, 1, 1, 1, 0, 1, 1, 256): (16, 0, 1, 0)}
    for got, (case, rule) in zip(client(["rule " + " ".join(map(str, c)) for c in want]), want.items()):
        assert tuple(map(int, got.split())) == rule + (1, 1), case


def test_the_pieces_of_a_rotation_take_every_element_once(client):
    lines = ["width %d %d %d %d %d" % (t, d, rot, p, align) for t in (0, 1) for p in (0, 1) for align in (2, 4, 8, 16) if align >= 2 * (t + 1)
             for d in (2, 8, 14, 64, 72, 80, 100, 128) for rot in (2, 4, 6, 14, 16, 20, 30, 32, 48, 64, 80, 100, 128) if rot <= d]
    widths = set()
    for line, got in zip(lines, client(lines)):
        ok, w = map(int, got.split())
        assert ok == 1, line
        widths.add((line.split()[1], line.split()[4], w))
    assert widths == {("0", "0", 16), ("0", "0", 4), ("0", "0", 2), ("0", "1", 16), ("0", "1", 4), ("1", "0", 16), ("1", "0", 4),
                      ("1", "1", 16), ("1", "1", 8)}


@pytest.mark.parametrize("rot", [2, 4, 64, 96, 128])
def test_frequencies(rot):
    for kind, name in ((libasl.ASL_FREQS_PLAIN, "plain"), (libasl.ASL_FREQS_LINEAR, "linear"), (libasl.ASL_FREQS_BASE, "base"),
                       (libasl.ASL_FREQS_PARTS, "parts")):
        for factor in (1.0, 4.0, 32.0):
            more = dict(context=8192.0, low=1.0, high=32.0)
            got = libasl.rotation_freqs(rot, 500000.0, kind, factor, **more).numpy()
            np.testing.assert_allclose(got, do.freqs(rot, 500000.0, name, factor, **more), rtol=1e-13)
            if factor == 1.0:
                np.testing.assert_allclose(got, 500000.0 ** (-2 * np.arange(rot // 2) / rot), rtol=1e-13)
    if rot > 2:                                              # what each scaling is for: the last pair is slowed by the factor, the first by linear alone
        plain = libasl.rotation_freqs(rot).numpy()
        base = libasl.rotation_freqs(rot, kind=libasl.ASL_FREQS_BASE, factor=8.0).numpy()
        parts = libasl.rotation_freqs(rot, kind=libasl.ASL_FREQS_PARTS, factor=8.0, context=4096.0).numpy()
        assert base[0] == plain[0] == parts[0]
        np.testing.assert_allclose(base[-1], plain[-1] / 8, rtol=1e-12)
        if rot >= 64:
            np.testing.assert_allclose(parts[-1], plain[-1] / 8, rtol=1e-12)


def test_frequencies_are_checked():
    bad = [(0, 1e4, 0, 1, 0, 0, 0), (63, 1e4, 0, 1, 0, 0, 0), (64, 0.0, 0, 1, 0, 0, 0), (64, float("nan"), 0, 1, 0, 0, 0), (64, 1e4, 4, 1, 0, 0, 0),
           (64, 1e4, -1, 1, 0, 0, 0), (64, 1e4, 1, 0.0, 0, 0, 0), (64, 1e4, 2, -1.0, 0, 0, 0), (64, 1e4, 3, 2.0, 0.0, 1, 32),
           (64, 1e4, 3, 2.0, 100.0, 32, 32)]
    for rot, base, kind, factor, context, low, high in bad:
        with pytest.raises(libasl.AslError) as e:
            libasl.rotation_freqs(rot, base, kind, factor, context, low, high)
        assert e.value.status == libasl.ASL_EINVAL


def test_calls_without_a_context_are_refused():
    lib = libasl.load()
    none = [None] * 20
    assert lib.asl_rotate(None, None, None, None, None, None, 1, None, None, None) == libasl.ASL_EINVAL
    assert lib.asl_rotate_write(None, None, None, *none[:6], 1, *none[:4]) == libasl.ASL_EINVAL
    assert lib.asl_pages_plan(None, None, None, None, 1, 1, *none[:9]) == libasl.ASL_EINVAL
    assert lib.asl_tree_attention(None, None, None, *none[:13]) == libasl.ASL_EINVAL
    assert lib.asl_pages_accept(None, None, None, None, 0, None, None, None, 1, None, 1, None, 0, *none[:4]) == libasl.ASL_EINVAL
    assert lib.asl_rotation_freqs(None, None) == libasl.ASL_EINVAL


def test_struct_sizes():
    assert ctypes.sizeof(libasl.AslRotation) == 112 and ctypes.sizeof(libasl.AslFreqs) == 48


# ------------------------------------------------------------------------------------------------- the binding
class _Recorder:
    """Stands in for the library: keeps the descriptions that the calls are given."""

    def __init__(self):
        self.seen = []

    def asl_rotate(self, h, r, *rest):
        self.seen.append((libasl.AslRotation.from_buffer_copy(r._obj), rest))
        return libasl.ASL_OK

    def asl_rotate_write(self, h, p, r, *rest):
        self.seen.append((libasl.AslRotation.from_buffer_copy(r._obj), rest))
        return libasl.ASL_OK

    def asl_tree_attention(self, h, p, a, *rest):
        self.seen.append((libasl.AslAttn.from_buffer_copy(a._obj), rest))
        return libasl.ASL_OK

    def _any(self, *args):
        self.seen.append(args)
        return libasl.ASL_OK
    asl_pages_plan = asl_pages_accept = _any

    def asl_destroy(self, h):
        return libasl.ASL_OK


@pytest.fixture
def recorded(monkeypatch):
    monkeypatch.setattr(libasl, "_stream", lambda: 0)
    x = libasl.Asl.__new__(libasl.Asl)
    x.lib, x.h, x.device = _Recorder(), ctypes.c_void_p(1), 0
    return x


def test_rotations_take_the_strides_of_their_tensors(recorded):
    import torch
    r = libasl.make_rotation(4, 2, 8, 6, back=True)
    before = bytes(r)
    x = torch.zeros(3, 8, 8)
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    out = torch.zeros(4, 3, 8).transpose(0, 1)
    pos, f, slot = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.float64), torch.zeros(3, dtype=torch.int64)
    recorded.asl_rotate(r, q, k, pos, f, out, k)
    recorded.asl_rotate_write(libasl.make_pages(4, 2, 8, 16, 1, 1, 1), r, q, k, v, pos, slot, f, q, x, x)
    assert bytes(r) == before
    a, b = recorded.lib.seen[0][0], recorded.lib.seen[1][0]
    assert (a.q_stride_tok, a.q_stride_head, a.k_stride_tok, a.q_out_stride_tok, a.q_out_stride_head, a.k_out_stride_tok) == (64, 8, 64, 8, 24, 64)
    assert (b.v_stride_tok, b.v_stride_head, b.q_out_stride_tok, b.flags, b.rot_dim) == (64, 8, 64, 1, 6)
    recorded.asl_rotate(libasl.make_rotation(4, 0, 8), q, None, pos, torch.zeros(4, dtype=torch.float64), out, None)
    recorded.asl_rotate(libasl.make_rotation(0, 2, 8), None, k, pos, torch.zeros(4, dtype=torch.float64), None, k)


def test_tensors_that_do_not_fit_are_refused(recorded):
    import torch
    r, pages = libasl.make_rotation(4, 2, 8, 6), libasl.make_pages(4, 2, 8, 16, 1, 1, 1)
    q, k = torch.zeros(3, 4, 8), torch.zeros(3, 2, 8)
    pos, f, slot = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.float64), torch.zeros(3, dtype=torch.int64)
    good = dict(q=q, k=k, pos=pos, freqs=f, q_out=q, k_out=k)
    bad = [dict(q=q[:2]), dict(q=k), dict(k=None), dict(k_out=k[..., :4]), dict(q_out=None), dict(pos=pos.long()), dict(pos=torch.zeros(6, dtype=torch.int32)[::2]),
           dict(freqs=f.float()), dict(freqs=f[:2]), dict(freqs=None), dict(q=torch.zeros(3, 8, 4).transpose(1, 2))]
    for change in bad:
        with pytest.raises(libasl.AslError):
            recorded.asl_rotate(r, **{**good, **change})
    good = dict(q=q, k=k, v=k, pos=pos, slot=slot, freqs=f, q_out=q, k_pages=k, v_pages=k)
    for change in (dict(v=None), dict(v=k[:2]), dict(slot=slot.int()), dict(slot=None), dict(slot=slot[:2]), dict(v=torch.zeros(3, 8, 2).transpose(1, 2))):
        with pytest.raises(libasl.AslError):
            recorded.asl_rotate_write(pages, r, **{**good, **change})
    i = torch.zeros(4, dtype=torch.int32)
    plan = lambda slot, pos, cu: recorded.asl_pages_plan(pages, i, i, 2, 3, i, i, i, cu, slot, pos)
    for args in ((slot.int(), pos, i), (slot, pos.long(), i), (slot, pos, i[:2]), (slot[:2], pos, i), (slot, None, i)):
        with pytest.raises(libasl.AslError):
            plan(*args)
    for more in (dict(parent=i[:2]), dict(parent=slot), dict(pruned=i[:0]), dict(pruned=torch.zeros(2))):
        with pytest.raises(libasl.AslError):
            recorded.asl_pages_plan(pages, i, i, 2, 3, i, i, i, i, slot, pos, **more)
    attn = libasl.make_attn(1, 3, 3, 10)
    for parent in (None, i[:2], i.long(), torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(libasl.AslError):
            recorded.asl_tree_attention(pages, attn, q, k, k, i, i, i, parent, q)
    accept = lambda path: recorded.asl_pages_accept(pages, i, i, 1, i, i, path, i, 2, i, i, i)
    for path in (i, torch.zeros(1, 4, dtype=torch.int32), torch.zeros(2, 8, dtype=torch.int32)[:, :4], torch.zeros(2, 4, dtype=torch.int64)):
        with pytest.raises(libasl.AslError, match="path"):
            accept(path)
    assert not recorded.lib.seen
    plan(slot, pos, i), recorded.asl_tree_attention(pages, attn, q, k, k, i, i, i, i[:3], q), accept(torch.zeros(2, 4, dtype=torch.int32))
    assert len(recorded.lib.seen) == 3


# ------------------------------------------------------------------------------------------------- the oracle's pins
@pytest.mark.parametrize("halves", [True, False])
def test_oracle_rotation_closed_forms(halves):
    rng = np.random.default_rng(0)
    x, f = rng.standard_normal((3, 2, 12)), do.freqs(8)
    a, b = do.pairs_of(8, halves)
    y, reach = do.rotate(x, [0, 5, -5], f, halves)
    np.testing.assert_array_equal(y[0], x[0])
    np.testing.assert_array_equal(y[..., 8:], x[..., 8:])
    assert np.all(reach[..., 8:] == 0)
    z = (x[1][:, a] + 1j * x[1][:, b]) * np.exp(5j * f)      # a product of complex numbers
    np.testing.assert_allclose(y[1][:, a] + 1j * y[1][:, b], z, rtol=1e-13)
    back, _ = do.rotate(y, [0, 5, -5], f, halves, back=True)
    np.testing.assert_allclose(back, x, atol=1e-14)
    # scores depend on the distance alone
    q, k = rng.standard_normal((1, 1, 12)), rng.standard_normal((1, 1, 12))
    dots = [float((do.rotate(q, [t + 7], f, halves)[0] * do.rotate(k, [t], f, halves)[0]).sum()) for t in (0, 100, 99999)]
    np.testing.assert_allclose(dots, dots[0], rtol=1e-9)


def test_oracle_tree_attention_closed_forms():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((6, 4, 8)), rng.standard_normal((2, 20, 8)), rng.standard_normal((2, 20, 8))
    chain = do.attention(q, k, v, 0.4, [-1, 0, 1, 2, 3, 4])  # a chain is what causal attention sees
    for x, y in zip(chain, po.attention(q, k, v, 0.4, causal=True)):
        np.testing.assert_allclose(x, y, rtol=1e-13)
    tree = do.attention(q, k, v, 0.4, [-1, 0, 0, -1, 2, 1])
    for i, path in enumerate([[0], [0, 1], [0, 2], [3], [0, 2, 4], [0, 1, 5]]):
        keys = list(range(14)) + [14 + a for a in path]      # each path is a sequence of its own
        one = po.attention(q[i:i + 1], k[:, keys], v[:, keys], 0.4, causal=True)
        np.testing.assert_allclose(tree[0][i], one[0][0], rtol=1e-13)
        np.testing.assert_allclose(tree[1][:, i], one[1][:, 0], rtol=1e-13)
    short = do.attention(q, k[:, :4], v[:, :4], 0.4, [-1, 0, 1, 2, 3, 4])
    assert np.all(short[0][:2] == 0) and np.all(short[1][:, :2] == -np.inf) and np.all(np.isfinite(short[1][:, 2:]))


def test_oracle_plans_and_accepted_paths_keep_the_counts():
    """Over random steps: a page's count is the number of rows that hold it; slots are the table's; what is kept is what was at the path's nodes."""
    rng, rnd = np.random.default_rng(2), random.Random(2)
    ps, n_pages, n_rows = 16, 12, 6
    table, kv_len, refs = np.full((n_rows, 12), -1, dtype=np.int64), np.zeros(n_rows, dtype=np.int64), np.zeros(n_pages, dtype=np.int64)
    pages = np.zeros((n_pages, 1, ps, 1))
    held = [[] for _ in range(n_rows)]                       # the values that each row should hold
    full = 0
    for step in range(200):
        rows = rng.permutation(n_rows)[:4]
        add = [int(min(rng.integers(0, 25), 12 * ps - kv_len[r])) for r in rows]
        parent = [rnd.randint(-1, i - 1) for m in add for i in range(m)]
        before = kv_len.copy()
        cu, slot, pos = do.plan(table, kv_len, refs, rows, add, ps, sum(add), parent, np.arange(n_rows) * 1000)
        new = rng.standard_normal(sum(add))
        got = slot >= 0
        pages[slot[got] // ps, 0, slot[got] % ps, 0] = new[got]
        paths = []
        for i, (r, m) in enumerate(zip(rows, add)):
            if m and kv_len[r] == before[r]:
                full += 1
                assert np.all(slot[cu[i]:cu[i + 1]] == -1)
                m = 0
            path = do.path_to(parent[cu[i]:cu[i + 1]], rnd.randrange(m)) if m else []
            assert all(pos[cu[i] + x] == before[r] + t + 1000 * r for t, x in enumerate(path))
            held[r] += [new[cu[i] + x] for x in path]
            paths.append((r, m, path))
        do.accept(table, kv_len, refs, [(pages, pages.copy())], *zip(*paths), ps)
        for r in range(n_rows):
            assert kv_len[r] == len(held[r])
            np.testing.assert_array_equal(po.gather(pages, table[r], len(held[r]))[0, :, 0], held[r])
            if len(held[r]) > 100 or rnd.random() < 0.05:
                po.free(table, kv_len, refs, [r], ps)
                held[r] = []
        held_pages = np.zeros(n_pages, dtype=np.int64)
        for r in range(n_rows):
            np.add.at(held_pages, table[r, :-(-int(kv_len[r]) // ps)], 1)
        assert np.array_equal(held_pages, refs)
    assert full > 3
