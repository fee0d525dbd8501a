"""Packed prompts and paged caches: what the host side does with a program's tensors and numbers, without a GPU."""
import ctypes as C

import pytest
import torch

import paper_2412_03409_amd as P
from paper_2412_03409_amd import binding as Bd
from paper_2412_03409_amd.pipeline import PagedPath


def a_path(S=3, L=2, H=4, Hkv=2, D=64):
    return PagedPath(S, L, H, Hkv, D, torch.ones(L), P.rope_plan(D, device="cpu"), num_pages=4, max_pages=2, device="cpu")


def test_the_places_that_end_are_those_of_any_iterable():
    path = a_path()
    path.cache.lens.fill_(5)
    for places in ([0, 2], (s for s in (0, 2)), iter([2, 0])):
        with pytest.raises(ValueError, match="GPU"):        # (the call itself; what it asks for is there)
            path.end(places)
        assert path.target.tolist() == [[0, 0], [5, 5], [0, 0]]


def test_a_path_refuses_rows_before_its_first_step(monkeypatch):
    """What the attention, the search or the store would refuse: nothing has been rotated, and no page given, by then."""
    import paper_2412_03409_amd.pipeline as pipeline
    path = a_path()
    for name in ("prefixkv_rope", "prefixkv_page_append"):
        monkeypatch.setattr(pipeline.B_, name, lambda *a, **kw: pytest.fail("a step was made"))
    T, bf = 9000, torch.bfloat16
    rows = lambda h, dtype=bf, D=64: torch.zeros((2, h, T, D), dtype=dtype)
    q, k, pos = rows(4), rows(2), torch.zeros((1, T), dtype=torch.int32)
    wrong = [(q, k, rows(4), pos), (q, rows(4), k, pos), (rows(2), k, k, pos), (q, k, k.float(), pos), (q.float(), k.float(), k.float(), pos),
             (q, k, k[:, :, 1:], pos), (q, k, rows(2, D=128), pos), (q, k[:1], k[:1], pos), (q[0], k, k, pos),
             (q, k, rows(2, D=128)[..., ::2], pos), (q, k, rows(2, D=68)[..., :64], pos), (q, k, rows(2, D=72)[..., 4:68], pos),
             (q, k, k[:, :, :1].expand(-1, -1, T, -1), pos), (q, k, k, pos[:, 1:]), (q, k, k, pos.long()),
             (q, k, k, pos.expand(2, -1)), (q, k, k, torch.zeros((1, 2 * T), dtype=torch.int32)[:, ::2])]
    for x in wrong:
        with pytest.raises(ValueError):
            path.prefill([0], [100], *x, [10])
        with pytest.raises(ValueError):
            path.extend([1, 0, 2], *x)
    for places, lengths, budgets in (([0], [8193], [10]), ([0, 1], [5, 6], [5, 0]), ([0], [5], [-1]), ([0], [5], [1 << 63]), ([], [], [])):
        with pytest.raises(ValueError):
            path.prefill(places, lengths, q, k, k, pos, budgets)


def test_a_path_refuses_a_scale_and_tensors_of_another_device(monkeypatch):
    for scale in (torch.ones(2).double(), torch.ones(1), torch.ones(2, 1), torch.ones(4)[::2]):
        with pytest.raises(ValueError, match="scale"):
            PagedPath(3, 2, 4, 2, 64, scale, P.rope_plan(64, device="cpu"), num_pages=4, max_pages=2, device="cpu")
    import paper_2412_03409_amd.pipeline as pipeline
    path = a_path()
    for name in ("prefixkv_rope", "prefixkv_page_append"):
        monkeypatch.setattr(pipeline.B_, name, lambda *a, **kw: pytest.fail("a step was made"))

    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 3
    q, k = (torch.zeros((2, h, 9, 64), dtype=torch.bfloat16) for h in (4, 2))
    pos = torch.zeros((1, 9), dtype=torch.int32)
    there = lambda x: x.as_subclass(Elsewhere)
    for x in ((there(q), k, k, pos), (q, there(k), k, pos), (q, k, there(k), pos), (q, k, k, there(pos))):
        with pytest.raises(ValueError, match="GPU"):
            path.prefill([0], [5], *x, [10])
        with pytest.raises(ValueError, match="GPU"):
            path.extend([1, 0, 2], *x)


def test_a_rotation_goes_by_where_the_plan_s_tensors_are():
    """Tensors whose storage is replaced: the old one may belong to somebody else by the next call."""
    plan, other = P.rope_plan(64, [16, 16], device="cpu"), P.rope_plan(32, [8, 8], theta=500.0, device="cpu")
    before = plan._args()
    assert plan._args() is before and before._obj.freq == plan.freq.data_ptr() and before._obj.rot_dim == 64
    plan.freq.data, plan.axis.data = other.freq.clone(), other.axis.clone()
    now = plan._args()._obj
    assert (now.freq, now.axis) == (plan.freq.data_ptr(), plan.axis.data_ptr())
    assert now.rot_dim == 32 and now.axes == 2


def test_rows_of_an_output_are_its_own():
    """A layer or head stride of 0 repeats an input; as an output, or rotated in place, it is refused.  (A
    workspace off by four bytes, which is looked at behind the strides, tells that an input was not.)"""
    A, odd, dims = C.c_void_p(4096), C.c_void_p(4100), dict(S=1, L=2, H=4, Hkv=2, T=10, D=64)
    ST, lib = Bd._Strides(0, 8192, 128, 4096), P.load()
    shape = C.byref(Bd._Packed(*dims.values(), P.PKV_BF16))
    rope = C.byref(Bd._Rope(4096, 4096, 64, 1, 0))
    paging = C.byref(Bd._Paging(8, 16, 4, 2))
    calls = [  # the call, its output strides, and where its keys' strides are
        (lib.prefixkv_rope, [shape, rope, A, A, ST, A, ST, A, ST, A, ST, None], (8, 10)),
        (lib.prefixkv_rope_store, [shape, rope, A, A, ST, A, ST, A, ST, A, ST, A, paging, A, A, None], (10,)),
        (lib.prefixkv_prefill_attn_packed, [shape, A, ST, A, ST, A, ST, A, A, A, ST, A, A, 1 << 30, None], (10,)),
        (lib.prefixkv_chunk_attn, [shape, A, ST, A, paging, 0, A, A, A, A, A, 10, A, ST, A, 1 << 30, None], (13,))]
    for f, args, outs in calls:
        for i in outs:
            for st in (Bd._Strides(0, 0, 128, 4096), Bd._Strides(0, 8192, 0, 4096)):
                assert f(*[st if j == i else x for j, x in enumerate(args)]) == 4
        ins = [i for i, x in enumerate(args) if x is ST and i not in outs]
        for i in ins:
            for st in (Bd._Strides(0, 0, 128, 4096), Bd._Strides(0, 8192, 0, 4096)):
                bad = [st if j == i else x for j, x in enumerate(args)]
                if f is lib.prefixkv_prefill_attn_packed or f is lib.prefixkv_chunk_attn:
                    bad[-3] = odd                                   # the workspace, which is looked at behind the strides
                    need = P.attn_workspace_bytes(**dims, dtype=torch.bfloat16, max_rows=10 if f is lib.prefixkv_chunk_attn else 0)
                    if need:
                        assert f(*bad) == 5


def test_numbers_that_an_int_does_not_hold_are_refused(monkeypatch):
    """Not taken modulo 2^32: rows or layers of another number would be worked on."""
    class Library:
        prefixkv_attn_workspace_bytes = P.load().prefixkv_attn_workspace_bytes
        prefixkv_page_workspace_bytes = P.load().prefixkv_page_workspace_bytes

        def __getattr__(self, name):
            return lambda *a: pytest.fail(f"{name} was called")
    monkeypatch.setattr(Bd, "_here", lambda *a: 0)
    monkeypatch.setattr(Bd, "load", Library)
    cache = P.paged_cache(1, 2, 2, 64, 16, 4, 4, device="cpu")
    off, scale = torch.tensor([0, 3], dtype=torch.int32), torch.ones(1)
    q, kv = torch.zeros((1, 4, 3, 64), dtype=torch.bfloat16), torch.zeros((1, 1, 2, 3, 64), dtype=torch.bfloat16)
    order, lengths = torch.zeros((1, 1, 3), dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int32)
    for x in ((1 << 32) + 1, 1 << 31, -(1 << 32)):
        with pytest.raises(ValueError, match="max_rows"):
            P.prefixkv_chunk_attn(cache, q, off, scale, x)
        with pytest.raises(ValueError, match="l0"):
            P.prefixkv_chunk_attn(cache, q, off, scale, 3, l0=x)
        with pytest.raises(ValueError, match="l0"):
            P.prefixkv_compact_paged(cache, kv, kv, order, lengths, l0=x)
        with pytest.raises(ValueError, match="T"):
            P.prefixkv_page_append(cache, off, x)
        with pytest.raises(ValueError, match="max_rows"):
            P.attn_workspace_bytes(1, 1, 4, 2, 3, 64, torch.bfloat16, max_rows=x)
