"""The binding of the drafting calls without a GPU: lists and tensors that the calls would read past their end, or as other numbers."""
import pytest

from paper_2601_07667_amd import asl as libasl
from test_draft import recorded  # noqa: F401  (a fixture)


def test_an_empty_list_of_slots_is_a_list(recorded):
    """What the call is given for one is not what it is given for none, though a tensor without elements has no address."""
    import torch
    pages, i = libasl.make_pages(4, 2, 8, 16, 1, 1, 1), torch.zeros(4, dtype=torch.int32)
    path = torch.zeros(2, 4, dtype=torch.int32)
    accept = lambda slot: recorded.asl_pages_accept(pages, i, i, 1, i, i, path, i, 2, i, i, i, slot=slot)
    some = torch.zeros(5, dtype=torch.int64)
    for slot in (None, some[:0], some):
        accept(slot)
    none, empty, full = [seen[11:13] for seen in recorded.lib.seen]
    assert none == (None, 0) and full == (some.data_ptr(), 5)
    assert empty[0] and empty[1] == 0


def test_tensors_of_smaller_elements_are_refused(recorded):
    """A bf16 tensor under a description of fp32 would be read past its end."""
    import torch
    r, pages = libasl.make_rotation(4, 2, 8, 6, dtype=libasl.ASL_F32), libasl.make_pages(4, 2, 8, 16, 1, 1, 1, dtype=libasl.ASL_F32)
    q, k = torch.zeros(3, 4, 8), torch.zeros(3, 2, 8)
    pos, f, slot = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.float64), torch.zeros(3, dtype=torch.int64)
    good = dict(q=q, k=k, pos=pos, freqs=f, q_out=q, k_out=k)
    into = dict(q=q, k=k, v=k, pos=pos, slot=slot, freqs=f, q_out=q, k_pages=k, v_pages=k)
    for call, args in ((lambda **a: recorded.asl_rotate(r, **a), good), (lambda **a: recorded.asl_rotate_write(pages, r, **a), into)):
        for name in args:
            if args[name] is q or (args[name] is k and not name.endswith("pages")):
                for t in (args[name].bfloat16(), args[name].half(), args[name].byte()):
                    with pytest.raises(libasl.AslError, match=name) as e:
                        call(**{**args, name: t})
                    assert e.value.status == libasl.ASL_EINVAL
        assert not recorded.lib.seen
        call(**args)
        recorded.lib.seen.clear()


def test_frequencies_of_the_host_are_refused(recorded):
    """rotation_freqs gives them there; the other tensors stand for the GPU's."""
    import torch
    r, pages = libasl.make_rotation(4, 2, 8), libasl.make_pages(4, 2, 8, 16, 1, 1, 1)
    there = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="meta")
    q, k, pos, slot = there(3, 4, 8), there(3, 2, 8), there(3, dtype=torch.int32), there(3, dtype=torch.int64)
    f = libasl.rotation_freqs(8)
    for call in (lambda f: recorded.asl_rotate(r, q, k, pos, f, q, k), lambda f: recorded.asl_rotate_write(pages, r, q, k, k, pos, slot, f, q, k, k)):
        with pytest.raises(libasl.AslError, match="freqs") as e:
            call(f)
        assert e.value.status == libasl.ASL_EINVAL and not recorded.lib.seen
        call(f.to("meta"))
        recorded.lib.seen.clear()


def _wrong(n):
    """What is no list of n int32 one behind the other."""
    import torch
    return [torch.zeros(n, dtype=t) for t in (torch.int64, torch.float32, torch.int16)] + [torch.zeros(2 * n, dtype=torch.int32)[::2][:n], None] \
        + ([torch.zeros(n - 1, dtype=torch.int32)] if n > 1 else [])


def test_lists_of_accepting_are_checked(recorded):
    import torch
    pages, i = libasl.make_pages(4, 2, 8, 16, 1, 1, 1), torch.zeros(4, dtype=torch.int32)
    good = dict(rows=i[:3], cu=i, path=torch.zeros(3, 4, dtype=torch.int32), n_path=i[:3])
    accept = lambda a, n=3: recorded.asl_pages_accept(pages, i, i, 1, a["rows"], a["cu"], a["path"], a["n_path"], n, i, i, i)
    bad = [(name, t) for name, n in (("rows", 3), ("cu", 4), ("n_path", 3)) for t in _wrong(n)] + [("path", torch.zeros(3, 4)), ("path", torch.zeros(3, 4).int().T)]
    for name, t in bad:
        with pytest.raises(libasl.AslError, match=name) as e:
            accept({**good, name: t})
        assert e.value.status == libasl.ASL_EINVAL
    assert not recorded.lib.seen
    accept(good), accept({**good, "path": torch.zeros(3, 0, dtype=torch.int32)})
    accept({**good, "path": torch.zeros(4097, 1, dtype=torch.int32)}, 4097)      # (refused by the call, for its size)
    accept({**good, "rows": i[:0], "cu": i[:1], "n_path": i[:0]}, 0)
    assert len(recorded.lib.seen) == 4


def test_lists_of_plans_are_checked(recorded):
    import torch
    pages, i = libasl.make_pages(4, 2, 8, 16, 1, 1, 1), torch.zeros(4, dtype=torch.int32)
    slot, pos = torch.zeros(5, dtype=torch.int64), torch.zeros(5, dtype=torch.int32)
    plan = lambda rows, add, n=3, cu=i: recorded.asl_pages_plan(pages, rows, add, n, 5, i, i, i, cu, slot, pos)
    for t in _wrong(3):
        for name, args in (("rows", (t, i[:3])), ("add", (i[:3], t))):
            with pytest.raises(libasl.AslError, match=name) as e:
                plan(*args)
            assert e.value.status == libasl.ASL_EINVAL
    assert not recorded.lib.seen
    plan(i[:3], i), plan(None, None, 0)
    plan(i, i, 4097, torch.zeros(4098, dtype=torch.int32))   # (refused by the call, for its size)
    assert len(recorded.lib.seen) == 3


def test_tensors_of_tree_attention_are_checked(recorded):
    import torch
    pages, attn, i = libasl.make_pages(4, 2, 8, 16, 1, 1, 1, dtype=libasl.ASL_F32), libasl.make_attn(3, 5, 5, 10, n_groups=3), torch.zeros(5, dtype=torch.int32)
    q = torch.zeros(5, 4, 8)
    good = dict(q=q, k_pages=q, v_pages=q, table=i, kv_len=i, cu_q=i[:4], parent=i, out=q, lse=torch.zeros(4, 5), rows=i[:3], group_start=i[:4], prefix_len=i[:3])
    call = lambda attn=attn, **change: recorded.asl_tree_attention(pages, attn, **{**good, **change})
    for name, n in (("cu_q", 4), ("rows", 3), ("group_start", 4), ("prefix_len", 3), ("parent", 5)):
        for t in _wrong(n):
            if name == "rows" and t is None:
                continue
            with pytest.raises(libasl.AslError, match=name) as e:
                call(**{name: t})
            assert e.value.status == libasl.ASL_EINVAL
    for name in ("q", "out"):
        for t in (q[:4], q[:, :3], q[..., :4], q.bfloat16(), q.half()):
            with pytest.raises(libasl.AslError, match=name):
                call(**{name: t})
    for t in (torch.zeros(4, 4), torch.zeros(4, 5).bfloat16(), torch.zeros(4, 5).double(), torch.zeros(5, 4).T):
        with pytest.raises(libasl.AslError, match="lse"):
            call(lse=t)
    assert not recorded.lib.seen
    call(), call(lse=None, rows=None), call(q=torch.zeros(7, 4, 8), out=torch.zeros(6, 5, 16)[:, :4, :8])
    call(libasl.make_attn(3, 5, 5, 10), group_start=None, prefix_len=None)
    call(libasl.make_attn(4097, 5, 5, 10))                   # (refused by the call, for its size)
    assert len(recorded.lib.seen) == 5


def test_pointers_of_accepting_are_checked(recorded):
    """A list of fewer pointers than layers would be read past its end, and what stands there be followed."""
    import torch
    pages, i, path = libasl.make_pages(4, 2, 8, 16, 1, 1, 1), torch.zeros(4, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int32)
    p = torch.zeros(3, dtype=torch.int64)
    accept = lambda k, v, layers, n=2: recorded.asl_pages_accept(pages, k, v, layers, i, i, path, i, n, i, i, i)
    for bad in (p[:2], p.int(), torch.zeros(6, dtype=torch.int64)[::2], None):
        for name, args in (("k_ptrs", (bad, p)), ("v_ptrs", (p, bad))):
            with pytest.raises(libasl.AslError, match=name) as e:
                accept(*args, 3)
            assert e.value.status == libasl.ASL_EINVAL
    assert not recorded.lib.seen
    accept(p, p, 3), accept(None, None, 0), accept(None, None, 3, 0), accept(p, p, 16385)     # (the last is refused by the call, for its size)
    assert len(recorded.lib.seen) == 4
