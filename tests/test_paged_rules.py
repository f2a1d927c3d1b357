"""The rules of the paged calls without a GPU."""
import os
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
