"""The paged cache without a GPU: refusals of its calls, index arithmetic on numbers out of range, the oracle's own pins."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

from oracle import paged_oracle as po
from paper_2601_07667_amd import asl as libasl
from test_bound import ROOT
import shutil


@pytest.fixture(scope="module")
def client(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("paged") / "paged_client")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2601_07667_amd", "csrc"), os.path.join(ROOT, "tests", "paged_client.cpp"),
                    "-o", exe], check=True)

    def ask(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", check=True, capture_output=True, text=True).stdout
        return out.splitlines()
    return ask


GOOD = dict(Hq=8, Hk=2, d=128, dtype=0, ps=64, n_pages=10, n_rows=4, row_stride=6, sp=2 * 64 * 128, sh=64 * 128, st=128, flags=0)


def _fields(**change):
    return " ".join(str(x) for x in {**GOOD, **change}.values())


@pytest.mark.parametrize("change,status,word", [
    ({}, 0, ""), (dict(dtype=1), 0, ""), (dict(ps=16), 0, ""), (dict(ps=4096), 0, ""), (dict(d=80, st=80), 0, ""),
    (dict(Hq=0), -1, "Hk"), (dict(Hk=3), -1, "Hk"), (dict(d=0), -1, "head_dim"), (dict(ps=0), -1, "page_size"),
    (dict(n_pages=0), -1, "n_pages"), (dict(n_rows=0), -1, "n_rows"), (dict(row_stride=0), -1, "row_stride"),
    (dict(flags=1), -1, "flags"), (dict(dtype=2), -4, "dtype"), (dict(ps=8), -4, "power of two"), (dict(ps=48), -4, "power of two"),
    (dict(ps=8192), -4, "power of two"), (dict(row_stride=1 << 25), -4, "2^30"), (dict(row_stride=1 << 24), 0, ""),
    (dict(st=120), -1, "stride"), (dict(sh=-128), -1, "stride"), (dict(sp=-8), -1, "stride"), (dict(d=100, st=104), -4, "16 bytes"),
    (dict(st=132), -4, "16 bytes"), (dict(sh=8195), -4, "16 bytes"), (dict(sp=16385), -4, "16 bytes"),
    (dict(Hq=131072, Hk=1), -4, "heads"), (dict(d=65544, st=65544), -4, "head_dim"),
])
def test_pages_are_checked(client, change, status, word):
    got = client(["pages " + _fields(**change)])[0]
    assert int(got.split()[0]) == status and word in got


@pytest.mark.parametrize("fields,status", [
    ((100, 12800, 128, 12800, 128), 0), ((0, 0, 128, 0, 128), 0), ((-1, 12800, 128, 12800, 128), -1),
    ((100, 12800, 64, 12800, 128), -1), ((100, 12800, 128, 12800, 127), -1), ((100, -8, 128, 12800, 128), -1),
    ((100, 12800, 132, 12800, 128), -4), ((100, 12800, 128, 12801, 128), -4),
])
def test_sources_are_checked(client, fields, status):
    assert int(client(["rows " + _fields() + " " + " ".join(map(str, fields))])[0].split()[0]) == status


@pytest.mark.parametrize("fields,status", [
    ((4, 4, 1, 100, 0, 1, 1024, 128, 1024, 128), 0), ((0, 0, 0, 0, 0, 0, 0, 0, 0, 0), 0), ((4, 4, 1, 100, 4, 1, 1024, 128, 1024, 128), 0),
    ((4, 4, 1, 100, 5, 1, 1024, 128, 1024, 128), -1), ((-1, 4, 1, 100, 0, 1, 1024, 128, 1024, 128), -1),
    ((4, -4, 1, 100, 0, 1, 1024, 128, 1024, 128), -1), ((4, 4, -1, 100, 0, 1, 1024, 128, 1024, 128), -1),
    ((4, 4, 1, -100, 0, 1, 1024, 128, 1024, 128), -1), ((4, 4, 1, 100, -1, 1, 1024, 128, 1024, 128), -1),
    ((4, 4, 1, 100, 0, 2, 1024, 128, 1024, 128), -1), ((4, 4, 1, 100, 0, 1, -8, 128, 1024, 128), -1),
    ((4, 4, 1, 100, 0, 1, 1024, 132, 1024, 128), -4), ((4, 4, 1, 100, 0, 1, 1024, 128, 1025, 128), -4),
])
def test_batches_are_checked(client, fields, status):
    assert int(client(["attn " + _fields() + " " + " ".join(map(str, fields))])[0].split()[0]) == status


def test_null_structs_and_contexts_are_refused(client):
    assert client(["null"]) == ["-1 -1 -1"]
    lib = libasl.load()
    none = [None] * 20
    assert lib.asl_paged_reserve(None, 1, 1, 1) == libasl.ASL_EINVAL
    assert lib.asl_pages_grow(None, None, None, None, 1, *none[:4]) == libasl.ASL_EINVAL
    assert lib.asl_pages_fork(None, None, None, None, 0, None, None, 1, *none[:4]) == libasl.ASL_EINVAL
    assert lib.asl_pages_free(None, None, None, 1, *none[:4]) == libasl.ASL_EINVAL
    assert lib.asl_pages_write(None, None, None, None, None, None, None, 1, 1, *none[:6]) == libasl.ASL_EINVAL
    assert lib.asl_pages_compact(None, None, None, None, None, 1, 1, None, 1, *none[:5]) == libasl.ASL_EINVAL
    assert lib.asl_paged_attention(None, None, None, *none[:12]) == libasl.ASL_EINVAL


def test_struct_sizes():
    assert ctypes.sizeof(libasl.AslPages) == 64 and ctypes.sizeof(libasl.AslRows) == 40 and ctypes.sizeof(libasl.AslAttn) == 56


def test_offsets_of_any_numbers_stay_inside_the_pages(client):
    """Whatever stands in table and kv_len, an offset is that of a slot of one of the n_pages pages, or -1."""
    rng = random.Random(3)
    wild = [-2 ** 31, -1, 0, 1, 2, 3, 5, 6, 7, 100, 2 ** 31 - 1]
    lines, want = [], []
    for _ in range(600):
        n_pages, n_rows, stride, ps = rng.randint(1, 6), rng.randint(1, 4), rng.randint(1, 5), rng.choice([16, 64])
        table = [rng.choice(wild) for _ in range(n_rows * stride)]
        lens = [rng.choice(wild) for _ in range(n_rows)]
        r, pos = rng.choice([-5, -1, 0, 1, 2, 3, 4, 2 ** 31 - 1]), rng.choice([-2 ** 31, -1, 0, 1, 15, 16, 63, 64, 200, 319, 320, 2 ** 31 - 1])
        lines.append("index %d %d %d %d %s %s %d %d" % (n_pages, n_rows, stride, ps, " ".join(map(str, table)),
                                                        " ".join(map(str, lens)), r, pos))
        ok = 0 <= r < n_rows and 0 <= lens[r] <= stride * ps
        off = -1
        if 0 <= r < n_rows and 0 <= pos < stride * ps and 0 <= table[r * stride + pos // ps] < n_pages:
            off = (table[r * stride + pos // ps] * ps + pos % ps) * 16
        want.append("%d %d %d" % (ok, lens[r] if ok else 0, off))
    assert client(lines) == want


def test_the_sequence_of_a_token(client):
    rng = random.Random(4)
    lines, want = [], []
    for _ in range(300):
        n = rng.randint(1, 12)
        counts = [rng.choice([0, 0, 1, 2, 9]) for _ in range(n)]
        cu = [sum(counts[:i]) for i in range(n + 1)]
        if cu[n] == 0:
            continue
        j = rng.randrange(cu[n])
        lines.append("seq %d %s %d" % (n, " ".join(map(str, cu)), j))
        want.append(str(max(i for i in range(n) if cu[i] <= j)))
        lines.append("seq %d %s %d" % (n, " ".join(str(rng.randint(-9, 9)) for _ in range(n + 1)), j))
        want.append(None)
    for (got, w), line in zip(zip(client(lines), want), lines):
        assert 0 <= int(got) < int(line.split()[1])
        assert w is None or got == w


def test_the_cut_of_an_attention_call(client):
    """Every key tile of a segment falls to one item, and no cut gives more items or partial rows than a launch makes room for."""
    rng = random.Random(5)
    lines = []
    for _ in range(400):
        n, Hk = rng.choice([1, 2, 5, 64, 300]), rng.choice([1, 2, 4, 8])
        longest = rng.choice([1, 3, 40, 2000, 16384])
        segments = [(rng.choice([0, 1, 4, 7, 16, 17, 128, 129, 1000]), rng.randint(0, longest)) for _ in range(n)]
        lines.append("cut %d %d %d %d %d %s" % (rng.choice([16, 64, 128]), rng.choice([1, 384, 512]), rng.choice([1, 2, 8]), Hk, n,
                                                " ".join("%d %d" % s for s in segments)))
    for line, got in zip(lines, client(lines)):
        ok, items, most_items, partial, most_partial = map(int, got.split())
        assert ok and items <= most_items and partial <= most_partial, (line, got)


def test_shared_tokens(client):
    for (stated, first, members), want in {(1000, 1000, 2): 960, (1000, 500, 2): 448, (10 ** 9, 191, 3): 128, (127, 1000, 9): 0,
                                           (1000, 1000, 1): 0, (-5, 1000, 4): 0, (1000, 0, 4): 0, (128, 128, 2): 128}.items():
        assert client(["shared %d %d %d" % (stated, first, members)]) == [str(want)]


# ------------------------------------------------------------------------------------------------- the oracle's pins
def test_oracle_attention_closed_forms():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 4, 8)), np.zeros((2, 5, 8)), rng.standard_normal((2, 5, 8))
    out, lse, _, _ = po.attention(q, k, v, 1.0, causal=True)          # equal logits: the mean of the keys seen
    for i in range(3):
        np.testing.assert_allclose(out[i, 3], v[1, :3 + i].mean(axis=0), rtol=1e-14)
        np.testing.assert_allclose(lse[:, i], np.log(3 + i), rtol=1e-14)
    out, lse, _, _ = po.attention(q, k, v, 1.0, causal=False)
    np.testing.assert_allclose(out[0, 0], v[0].mean(axis=0), rtol=1e-14)
    out, lse, _, _ = po.attention(rng.standard_normal((5, 4, 8)), k[:, :2], v[:, :2], 1.0, causal=True)
    assert np.all(out[:3] == 0) and np.all(lse[:, :3] == -np.inf) and np.all(lse[:, 3] == 0)
    k = rng.standard_normal((2, 5, 8))
    out, lse, _, _ = po.attention(q, k, v, 0.5, causal=False)
    x = 0.5 * k[1] @ q[2, 3]
    np.testing.assert_allclose(out[2, 3], (np.exp(x) / np.exp(x).sum()) @ v[1], rtol=1e-12)
    np.testing.assert_allclose(lse[3, 2], np.log(np.exp(x).sum()), rtol=1e-12)


def test_oracle_pages_keep_their_counts():
    """Over random calls: a page's count is the number of rows that hold it, and rows hold no page twice."""
    rng = np.random.default_rng(1)
    ps, n_pages, n_rows = 16, 40, 9
    table, kv_len, refs = np.full((n_rows, 12), -1, dtype=np.int64), np.zeros(n_rows, dtype=np.int64), np.zeros(n_pages, dtype=np.int64)
    full = 0
    for step in range(400):
        kind = rng.integers(3)
        empty, used = np.flatnonzero(kv_len == 0), np.flatnonzero(kv_len > 0)
        if kind == 0:
            rows = rng.permutation(n_rows)[:3]
            add = [int(min(rng.integers(0, 60), 12 * ps - kv_len[r])) for r in rows]
            before = kv_len.copy()
            po.grow(table, kv_len, refs, rows, add, ps)
            full += any(kv_len[r] != before[r] + a for r, a in zip(rows, add))
        elif kind == 1 and empty.size and used.size:
            po.fork_tables(table, kv_len, refs, rng.choice(used, empty.size), empty, ps)
        elif kind == 2 and used.size:
            po.free(table, kv_len, refs, rng.permutation(used)[:2], ps)
        held = np.zeros(n_pages, dtype=np.int64)
        for r in range(n_rows):
            pages = table[r, :-(-int(kv_len[r]) // ps)]
            assert len(set(pages.tolist())) == pages.size
            np.add.at(held, pages, 1)
        assert np.array_equal(held, refs)
    assert full > 10
