"""The order of the work items of drafted trees, without a GPU."""
import os
import shutil
import subprocess

import numpy as np

from test_bound import ROOT


def test_items_of_the_same_keys_are_a_multiple_of_eight_apart(tmp_path):
    """Every row tile of every split of every head once; row tiles of the same keys on one of eight dies, but for the last splits, fewer than
    take turns."""
    exe = str(tmp_path / "client")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2601_07667_amd", "csrc"), os.path.join(ROOT, "tests", "draft_items_client.cpp"),
                    "-o", exe], check=True)
    cases = [(Hk, tiles, splits) for Hk in range(1, 8) for tiles in (2, 3, 4, 7) for splits in (1, 2, 3, 7, 8, 9, 16, 25, 64)]
    out = subprocess.run([exe], input="\n".join("%d %d %d" % c for c in cases) + "\n", check=True, capture_output=True, text=True).stdout
    for (Hk, tiles, splits), line in zip(cases, out.splitlines()):
        got = np.array(line.split(), dtype=int).reshape(-1, 2)
        place = {(e % Hk, *x): e for e, x in enumerate(map(tuple, got.tolist()))}
        assert set(place) == {(h, t, s) for h in range(Hk) for t in range(tiles) for s in range(splits)}, (Hk, tiles, splits)
        whole = splits // (8 // np.gcd(8, Hk)) * (8 // np.gcd(8, Hk))
        for h in range(Hk):
            for s in range(whole):
                assert len({place[h, t, s] % 8 for t in range(tiles)}) == 1, (Hk, tiles, splits, h, s)
