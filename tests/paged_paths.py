"""Calls of the paged attention by the kernels that they take: split items of 16 rows (16), tiles of 64 or 128 rows, and the same for
the prefixes that are read apart (0: none).  tests/test_paged_rules.py holds each against the library's rule, tests/test_gpu_paged_paths.py
runs them.  `wide` is a stated max_kv_len that changes the cut alone."""

WIDE = 1 << 20


def case(name, kinds, lens, n_q, Hq, Hk, d, ps=16, dtype="bf16", causal=True, groups=None, max_kv=None):
    return dict(name=name, kinds=kinds, lens=lens, n_q=n_q, Hq=Hq, Hk=Hk, d=d, ps=ps, dtype=dtype, causal=causal, groups=groups,
                max_kv=max_kv or max(lens))


def _own(n, seed, lo=1, hi=300):
    return [lo + (seed + 7919 * i * i + 104729 * i) % (hi - lo + 1) for i in range(n)]


def _behind(prefix, n, seed, lo=1, hi=300):
    return [prefix + x for x in _own(n, seed, lo, hi)]


def shared_cases():
    P = 2112
    out = [
        case("one group, one token", (16, 16), _behind(P, 17, 1), [1] * 17, 32, 8, 128, groups=[(17, P)]),
        case("tiles of 128 for the prefix", (16, 128), _behind(P, 17, 2), [1] * 17, 32, 8, 128, 64, groups=[(17, P)], max_kv=WIDE),
        case("tiles of 64 for the prefix", (16, 64), _behind(P, 17, 3), [1] * 17, 24, 8, 128, 64, groups=[(17, P)], max_kv=WIDE),
        case("drafts", (64, 128), _behind(2090, 48, 4, 6, 200), [2 + i % 4 for i in range(48)], 28, 4, 128, groups=[(6, 2090)] * 8),
        case("tiles for both", (64, 64), _behind(P, 20, 5, 25), [1 + 19 * (i % 6 == 2) for i in range(20)], 8, 8, 128,
             groups=[(6, P), (8, P), (6, P)], max_kv=WIDE),
        case("tiles beside split prefixes", (64, 16), _behind(P, 24, 6, 25), [20 if i == 9 else 1 for i in range(24)], 8, 8, 128,
             groups=[(3, P)] * 8, max_kv=WIDE),
        case("a group of one and one that shares nothing", (16, 16), _behind(P, 17, 7) + [50, 2000] + [5, 60, 1], [2] * 22, 16, 8, 128,
             groups=[(17, P), (1, 50), (1, 2000), (3, 0)]),
        case("many groups", (16, 16), _behind(130, 350, 8, 3, 40), [1 + i % 3 for i in range(350)], 16, 8, 128, groups=[(5, 130)] * 70),
        case("many groups, tiles", (16, 64), _behind(130, 350, 9, 3, 40), [1 + i % 5 for i in range(350)], 16, 8, 128,
             groups=[(5, 130)] * 70, max_kv=WIDE),
        case("fp32", (16, 16), _behind(P, 10, 10), [1 + i % 3 for i in range(10)], 16, 8, 128, dtype="f32", groups=[(10, P)]),
        case("fp32, many groups", (16, 16), _behind(130, 210, 11, 3, 40), [1 + i % 3 for i in range(210)], 8, 8, 128, dtype="f32",
             groups=[(3, 130)] * 70),
        case("fp32, d = 256", (16, 16), _behind(P, 6, 12), [1] * 6, 16, 8, 256, dtype="f32", groups=[(6, P)]),
        case("fp32, d = 100", (16, 16), _behind(P, 12, 13), [2] * 12, 16, 8, 100, dtype="f32", groups=[(12, P)]),
        case("d = 256", (16, 16), _behind(P, 10, 14), [1 + i % 2 for i in range(10)], 16, 8, 256, groups=[(10, P)]),
        case("d = 64, tiles", (16, 128), _behind(P, 34, 15), [1] * 34, 32, 8, 64, groups=[(34, P)], max_kv=WIDE),
        case("d = 64", (16, 16), _behind(P, 34, 16), [1] * 34, 8, 8, 64, groups=[(34, P)]),
        case("d = 80, tiles", (16, 128), _behind(P, 27, 17), [1] * 27, 32, 8, 80, groups=[(27, P)], max_kv=WIDE),
        case("d = 72", (64, 64), _behind(P, 32, 18, 30), [30 if i == 3 else 1 for i in range(32)], 8, 8, 72, groups=[(32, P)], max_kv=WIDE),
    ]
    for c in list(out):                                      # every query sees every key
        if c["name"] in ("one group, one token", "drafts", "tiles beside split prefixes", "many groups", "fp32"):
            out.append(dict(c, name=c["name"] + ", all seen", causal=False))
    # members that end before the prefix does, one without keys, queries that reach back into it
    short = _behind(P, 17, 19) + [2000, 700, 63, 64, 0, 1]
    for kinds, far, max_kv in (((16, 16), 9, None), ((64, 128), 39, WIDE)):
        reach = [1 + far * (i % 4 == 1) for i in range(23)]
        out.append(case("members of any length", kinds, short, reach, 8, 8, 128, groups=[(23, P)], max_kv=max_kv))
        out.append(case("members of any length, all seen", kinds, short, reach, 8, 8, 128, causal=False, groups=[(23, P)], max_kv=max_kv))
    return out


def tile_cases():
    out = []
    for Hq, Hk, d in ((4, 2, 64), (8, 8, 128), (28, 4, 128), (6, 2, 80), (12, 3, 120), (3, 3, 8), (32, 2, 128)):
        for causal in (True, False):
            out.append(case("ragged %d/%d heads of %d, %s" % (Hq, Hk, d, "causal" if causal else "all seen"),
                            (128 if 40 * Hq // Hk > 64 else 64, 0), [70, 5, 0, 200, 9, 130, 33], [17, 9, 3, 40, 0, 1, 33], Hq, Hk, d, 32,
                            causal=causal, max_kv=WIDE))
    for n_q in (5, 8, 9, 16, 17, 31, 32, 33, 64, 65, 129):
        out.append(case("%d tokens" % n_q, (64 if 4 * n_q <= 64 else 128, 0), [200 + n_q, 260], [n_q, max(1, n_q - 1)], 8, 2, 64, max_kv=WIDE))
    for ps in (16, 64, 256, 4096):                           # spans that are cut, rows that end within a tile
        out.append(case("cut, pages of %d" % ps, (128, 0), [5000, 700, 65], [70, 19, 65], 8, 2, 128, ps))
        out.append(case("cut, 64 rows, pages of %d" % ps, (64, 0), [4100, 1700, 64], [16, 15, 9], 8, 2, 64, ps, max_kv=WIDE))
    out.append(case("one sequence that sees little", (128, 0), [1500, 20, 1], [100, 300, 200], 4, 2, 128, max_kv=WIDE))
    out.append(case("a chunk beside decoding", (128, 0), [3000] + _own(40, 20, 1, 900), [300] + [1] * 40, 8, 2, 128, 64))
    out.append(case("cross", (128, 0), [4000, 1, 129], [90, 90, 40], 8, 2, 128, causal=False))
    return out


LEAP_PREFIX = 3328


def leap_cases():
    """Every pair of kinds, 4 query heads on each of 8 KV heads; for d = 64 those of tiles."""
    P, out = LEAP_PREFIX, []
    for d in (64, 128, 80):
        for kinds, groups, n_q in (((64, 0), None, [16] * 3), ((128, 0), None, [33] * 3), ((16, 16), [(24, P)], [1] * 24),
                                   ((16, 64), [(12, P)] * 2, [1] * 24), ((16, 128), [(24, P)], [1] * 24),
                                   ((64, 16), [(3, P)] * 12, [6] + [1] * 35), ((64, 64), [(12, P)] * 2, [1] * 20 + [6] + [1] * 3),
                                   ((64, 128), [(24, P)], [1] * 9 + [16] + [1] * 14)):
            if d == 64 and 16 in kinds:
                continue
            lens = [P + 40 + 3 * (i % 50) for i in range(len(n_q))]
            out.append(case("leaps, d = %d, kinds %d and %d" % ((d,) + kinds), kinds, lens, n_q, 32, 8, d, 64, groups=groups,
                            max_kv=None if kinds == (16, 16) else WIDE))
    return out


def large_cases():
    """Calls of more rows than the workspace's pieces grow with (131072): many queries, and so many sequences behind a prefix that there is
    room for their rows' own and shared parts, but for no further piece of the long one among them."""
    n = 4095
    return [
        case("192000 rows", (128, 0), [70, 64, 1, 90, 0, 33, 300, 65], [600] * 8, 40, 8, 64, causal=False, max_kv=WIDE),
        case("171990 rows behind a prefix", (16, 128), [130 + (10000 if i == 77 else 1 + i % 20) for i in range(n)], [1] * n, 42, 6, 64,
             groups=[(n, 130)], max_kv=WIDE),
    ]
