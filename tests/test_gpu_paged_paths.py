"""The paged calls on the GPU where their paths part: head sizes that leave a part of a store."""
import numpy as np
import pytest

from paper_2601_07667_amd import asl
from test_gpu_paged import Cache, _check, _dt, _ints, _oracle, _queries, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("f32", 68), ("f32", 100), ("f32", 132), ("f32", 252), ("f32", 4), ("f32", 60),
                                     ("bf16", 72), ("bf16", 136), ("bf16", 248)])
@pytest.mark.parametrize("lens,n_q", [([100, 128, 7, 64], [1, 3, 2, 1]),               # rows written whole
                                      ([1900, 300, 20, 700], [1, 2, 5, 1]),            # pieces joined within the launch
                                      ([3000, 260, 5], [2, 1, 4])])                    # pieces joined by a launch of their own
def test_rows_of_head_sizes_that_leave_a_part_of_a_store(ctx, gpu_device, lens, n_q, dtype, d):
    """Elements behind a row, between the heads and behind the last row of `out`, keep what they hold."""
    import torch
    Hq, Hk, total = 6, 2, sum(n_q)
    c = Cache(gpu_device, lens, Hk, d, 16, dtype, 21)
    q = _queries(total, Hq, d, dtype, gpu_device, 22)
    ref = _oracle(c, q, n_q)
    cu = _ints(np.concatenate([[0], np.cumsum(n_q)]), gpu_device)
    lse = torch.empty((Hq, total), dtype=torch.float32, device=gpu_device)
    a = asl.make_attn(len(lens), total, max(n_q), max(lens))
    for pad in (0, 8):
        room = torch.full((total * Hq * (d + pad) + 64,), 77.0, dtype=_dt(dtype), device=gpu_device)
        rows = room[:total * Hq * (d + pad)].view(total, Hq, d + pad)
        ctx.asl_paged_attention(c.desc(Hq), a, q, c.k, c.v, c.table, c.kv_len, cu, rows[..., :d], lse=lse)
        _check(rows[..., :d], lse, ref, d, max(lens), dtype, "d %d, pad %d" % (d, pad))
        assert bool((rows[..., d:] == 77).all()) and bool((room[total * Hq * (d + pad):] == 77).all())
    assert ctx.asl_device_fault() == 0
