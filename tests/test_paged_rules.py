"""The rules of the paged calls without a GPU."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

import paged_paths
from paper_2601_07667_amd import asl as libasl
from test_bound import ROOT


@pytest.fixture(scope="module")
def client(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("rules") / "paged_rules_client")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2601_07667_amd", "csrc"), os.path.join(ROOT, "tests", "paged_rules_client.cpp"),
                    "-o", exe], check=True)

    def ask(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", check=True, capture_output=True, text=True).stdout
        return out.splitlines()
    return ask


@pytest.mark.parametrize("bytes_", [2, 4])
def test_every_store_of_a_row_ends_within_it(client, bytes_):
    """Every head size that the attention accepts, every number of elements that a thread holds."""
    lines = ["stores %d %d %d %d" % (bytes_, held, D, d) for D in (64, 128, 256) for held in (4, 8)
             for d in range(16 // bytes_, D + 1, 16 // bytes_)]
    for line, got in zip(lines, client(lines)):
        ok, w = map(int, got.split())
        assert ok == 1 and w * bytes_ <= 16, line


def test_a_workspace_is_outgrown_seven_times_at_most(client):
    """Limits in any order: what is there has room for the last ones, never shrinks, and is replaced at most seven times."""
    rng = random.Random(6)
    most = 0
    for _ in range(300):
        limits = [(rng.choice([1, 4096, 4097, 2 ** rng.randint(0, 30), 2 ** 31 - 1, rng.randint(1, 200000)]), rng.randint(1, 256))
                  for _ in range(rng.randint(1, 40))]
        rooms = [tuple(map(int, x.split())) for x in client(["room %d %s" % (len(limits), " ".join("%d %d" % x for x in limits))])]
        assert len(rooms) == len(limits)
        for (rows, dim), (want_rows, want_dim) in zip(rooms, limits):
            assert rows >= min(want_rows, 131072) and dim >= want_dim and (rows, dim) <= (131072, 256)
        for a, b in zip(rooms, rooms[1:]):
            assert b[0] >= a[0] and b[1] >= a[1]
        most = max(most, len(set(rooms)) - 1)
    slowly = [(4096 << i, 64) for i in range(6)] + [(1, 128), (1, 256)]
    rooms = client(["room %d %s" % (len(slowly), " ".join("%d %d" % x for x in slowly))])
    assert most <= 7 and len(set(rooms)) - 1 == 7 == int(client(["kept"])[0])


def _rule(client, c):
    e, groups = (2 if c["dtype"] == "bf16" else 4), c["groups"] or []
    saved, at = 0, 0
    for m, p in groups:                                      # whole tiles of what is stated and there, two of them at least
        tokens = min(p, c["lens"][at]) // 64 * 64
        saved += (m - 1) * tokens if m > 1 and tokens >= 128 else 0
        at += m
    got = client(["rule %d %d %d %d %d %d %d %d %d %d %d" % (
        c["dtype"] == "bf16" and c["d"] <= 128, sum(c["n_q"]), c["Hq"] // c["Hk"], c["Hk"], len(c["lens"]), len(groups), max(c["n_q"]),
        c["max_kv"], 2 * c["d"] * e * c["Hk"], 2 * (1 << 17) + 131072, saved)])[0]
    own, shared, host, device, joined = map(int, got.split())
    return (own, shared if host and device else 0), joined


def test_the_cases_take_the_kernels_that_they_are_for(client):
    cases = paged_paths.shared_cases() + paged_paths.tile_cases() + paged_paths.leap_cases() + paged_paths.large_cases()
    for c in cases:
        kinds, joined = _rule(client, c)
        assert kinds == c["kinds"] and not joined, c["name"]
    taken = {c["kinds"] for c in cases}
    assert taken >= {(16, 16), (16, 64), (16, 128), (64, 16), (64, 64), (64, 128), (64, 0), (128, 0)}


# ------------------------------------------------------------------------------------------------- the binding
class _Recorder:
    """Stands in for the library: keeps what the paged calls are given."""

    def __init__(self):
        self.attn, self.rows, self.idx_rows = [], [], []

    def asl_paged_attention(self, h, pages, attn, *pointers):
        self.attn.append(libasl.AslAttn.from_buffer_copy(attn._obj))
        return libasl.ASL_OK

    def asl_pages_write(self, h, pages, src, *rest):
        self.rows.append(libasl.AslRows.from_buffer_copy(src._obj))
        return libasl.ASL_OK

    def asl_pages_compact(self, h, pages, src, dst, cu, n, total, idx, idx_rows, *rest):
        self.idx_rows.append(idx_rows)
        return libasl.ASL_OK

    def asl_destroy(self, h):
        return libasl.ASL_OK


@pytest.fixture
def recorded(monkeypatch):
    monkeypatch.setattr(libasl, "_stream", lambda: 0)
    x = libasl.Asl.__new__(libasl.Asl)
    x.lib, x.h, x.device = _Recorder(), ctypes.c_void_p(1), 0
    return x


def _attend_on_cpu(x, attn, q, out):
    import torch
    i = torch.zeros(4, dtype=torch.int32)
    x.asl_paged_attention(libasl.make_pages(4, 2, 8, 16, 1, 1, 1), attn, q, q, q, i, i, i, out)


def test_a_call_leaves_the_description_of_its_batch_alone(recorded):
    import torch
    attn = libasl.make_attn(2, 3, 2, 100, causal=False)
    before = bytes(attn)
    q, wide = torch.zeros(3, 4, 8), torch.zeros(3, 4, 24)[..., :8]
    _attend_on_cpu(recorded, attn, q, wide)
    _attend_on_cpu(recorded, attn, q.transpose(0, 1).contiguous().transpose(0, 1), q)
    assert bytes(attn) == before
    a, b = recorded.lib.attn
    assert (a.n_seqs, a.total_q, a.max_q_len, a.max_kv_len, a.flags) == (2, 3, 2, 100, 0)
    assert (a.q_stride_tok, a.q_stride_head, a.out_stride_tok, a.out_stride_head) == (32, 8, 96, 24)
    assert (b.q_stride_tok, b.q_stride_head, b.out_stride_tok, b.out_stride_head) == (8, 24, 32, 8)


def test_rows_that_are_not_contiguous_are_refused(recorded):
    import torch
    attn, good = libasl.make_attn(2, 3, 2, 100), torch.zeros(3, 4, 8)
    bad = torch.zeros(3, 8, 4).transpose(1, 2)
    for q, out, word in ((bad, good, "q"), (good, bad, "out"), (good[..., :4].expand(3, 4, 4)[..., ::2], good, "q")):
        with pytest.raises(libasl.AslError, match="last dimension of " + word) as e:
            _attend_on_cpu(recorded, attn, q, out)
        assert e.value.status == libasl.ASL_EUNSUPPORTED
    pages, i = libasl.make_pages(2, 2, 8, 16, 1, 1, 1), torch.zeros(4, dtype=torch.int32)
    k = torch.zeros(2, 3, 8)
    write = lambda k, v: recorded.asl_pages_write(pages, k, v, i, i, 1, 3, i, i, k, k)
    for a, b, status in ((torch.zeros(2, 8, 3).transpose(1, 2), k, libasl.ASL_EUNSUPPORTED),
                         (k, torch.zeros(2, 8, 3).transpose(1, 2), libasl.ASL_EUNSUPPORTED),
                         (k, k[:, :2], libasl.ASL_EINVAL), (k, k[:1], libasl.ASL_EINVAL)):    # v ends before k does
        with pytest.raises(libasl.AslError) as e:
            write(a, b)
        assert e.value.status == status
    assert not recorded.lib.attn and not recorded.lib.rows
    write(k.transpose(0, 1).contiguous().transpose(0, 1), k)
    src = recorded.lib.rows[0]
    assert (src.n_src, src.k_stride_head, src.k_stride_tok, src.v_stride_head, src.v_stride_tok) == (3, 8, 16, 24, 8)


def test_indices_and_normalisers_with_gaps_are_refused(recorded):
    """What a selection leaves is [Hk + 1, k + W]: a slice of its columns is no list that the calls can read."""
    import torch
    pages, i = libasl.make_pages(2, 2, 8, 16, 1, 1, 1), torch.zeros(4, dtype=torch.int32)
    k, picked = torch.zeros(2, 9, 8), torch.zeros(3, 6, dtype=torch.int32)
    calls = (lambda idx, n: recorded.asl_pages_write(pages, k, k, i, i, 1, n, i, i, k, k, idx=idx),
             lambda idx, n: recorded.asl_pages_compact(pages, i, i, i, 1, n, idx, i, i, k, k))
    for call in calls:
        for idx, n in ((picked[:2, :4], 4), (picked[:2], 4), (picked[:2], 7), (picked[:1], 7), (picked[:2, ::2], 3), (picked[:1, ::2], 3),
                       (picked.t()[:2], 3), (picked[:2, :1], 1)):
            with pytest.raises(libasl.AslError, match="idx") as e:
                call(idx, n)
            assert e.value.status == libasl.ASL_EINVAL
        for idx, n in ((picked[:2], 6), (picked[2:], 6), (picked[:1], 4), (picked[:1, :4], 4), (picked[:1, ::2], 1), (picked[:2, :1].contiguous(), 1),
                       (picked[:1, :0], 0)):
            call(idx, n)
    assert [r.idx_rows for r in recorded.lib.rows] == recorded.lib.idx_rows == [2, 1, 1, 1, 1, 2, 1]
    attn, q, lse = libasl.make_attn(1, 3, 3, 100), torch.zeros(3, 4, 8), torch.zeros(4, 5)
    attend = lambda lse: recorded.asl_paged_attention(libasl.make_pages(4, 2, 8, 16, 1, 1, 1), attn, q, q, q, i, i, i, q, lse=lse)
    for bad in (lse[:, :3], lse[:, 4:], lse.t()):
        with pytest.raises(libasl.AslError, match="lse") as e:
            attend(bad)
        assert e.value.status == libasl.ASL_EUNSUPPORTED
    attend(lse), attend(None)
    assert len(recorded.lib.attn) == 2
