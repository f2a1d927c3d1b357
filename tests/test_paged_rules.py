"""The rules of the paged calls without a GPU."""
import os
import random
import shutil
import subprocess

import pytest

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
