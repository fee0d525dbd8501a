"""Beam search over the paged cache and attention to states of another length: what the C entry points refuse, before anything is enqueued, and what the binding refuses;
the plain forms against hand-worked numbers."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import beam_reference as R
import paper_2412_03409_amd as P
from paper_2412_03409_amd import binding as Bd
from test_serving_boundary_cpu import A, BAD_PACKED, BAD_PAGING, BIG, ODD, ST, packed, paging, with_null


def but(args, i, x):
    return [x if j == i else y for j, y in enumerate(args)]


def test_select_refuses():
    lib = P.load()
    f = lib.prefixkv_beam_select
    need = P.beam_workspace_bytes(2, 4, 1000, torch.float32)
    args = [2, 4, 1000, P.PKV_F32, A, 1000, A, A, 7, A, A, A, A, A, need, None]
    for bad in with_null(args, optional=(7, 13)):
        assert f(*bad) == 1
    for i, xs in ((0, (0, 4097)), (1, (0, 33)), (2, (0, (1 << 20) + 1)), (8, (-2, 1000))):
        for x in xs:
            assert f(*but(args, i, x)) == 2
    assert f(*but(args, 8, -1)) == 2                                     # beams that have ended, and nothing that ends them
    assert f(*but(args, 3, 2)) == 3
    assert f(*but(args, 5, -1)) == 4 and f(*but(args, 4, C.c_void_p(4098))) == 4
    assert f(*but(but(args, 3, P.PKV_BF16), 4, C.c_void_p(4097))) == 4
    for i, x in ((13, None), (13, C.c_void_p(4104)), (14, need - 1)):
        assert f(*but(args, i, x)) == 5
    for bad in ((0, 4, 10), (2, 33, 10), (2, 4, 0), (2, 4, (1 << 20) + 1)):
        assert P.beam_workspace_bytes(*bad, torch.float32) == 0


def test_reorder_refuses():
    lib = P.load()
    f = lib.prefixkv_page_reorder
    need = P.reorder_workspace_bytes(8, 2)
    args = [8, 4, 2, 64, P.PKV_BF16, paging(), A, A, A, A, A, A, A, A, A, A, A, A, need, None]
    for bad in with_null(args, optional=(17,)):
        assert f(*bad) == 1
    assert f(*but(args, 5, None)) == 1
    for i, xs in ((0, (0, 4097, 9)), (1, (0, 3, 33, 64)), (2, (0, 2049)), (3, (32, 96, 256))):
        for x in xs:
            assert f(*but(args, i, x)) == 2
    for kw in BAD_PAGING:
        assert f(*but(args, 5, paging(**kw))) == 2
    assert f(*but(args, 4, 2)) == 3
    for i in (14, 15):
        assert f(*but(args, i, ODD)) == 4
    for i, x in ((17, None), (17, C.c_void_p(4104)), (18, need - 1)):
        assert f(*but(args, i, x)) == 5
    # 4096 * 64 segments of 2048 heads: more workgroups than a launch has
    assert f(*but(but(but(args, 0, 4096), 2, 2048), 5, paging(layers=64, page_size=256, max_pages=1))) == 7
    assert P.reorder_workspace_bytes(0, 2) == 0 and P.reorder_workspace_bytes(4097, 1) == 0 and P.reorder_workspace_bytes(4, 65) == 0


def test_cross_attention_refuses():
    lib = P.load()
    f = lib.prefixkv_cross_attn
    args = [packed(), A, ST, A, 100, A, ST, A, ST, A, A, A, 10, A, ST, A, BIG, None]
    for bad in with_null(args, optional=(10, 15)):
        assert f(*bad) == 1
    assert f(*but(args, 0, None)) == 1
    for kw in BAD_PACKED:
        assert f(*but(args, 0, packed(**kw))) == 2, kw
    for i, xs in ((4, (0, -1, (1 << 22) + 1)), (12, (0, 11))):
        for x in xs:
            assert f(*but(args, i, x)) == 2
    assert f(*but(args, 0, packed(dtype=5))) == 3
    for i in (1, 5, 7, 13):
        assert f(*but(args, i, ODD)) == 4
    for i in (2, 6, 8, 14):
        for bad in (Bd._Strides(0, 8192, 130, 4096), Bd._Strides(0, -8192, 128, 4096), Bd._Strides(0, 8192, 128, 0)):
            assert f(*but(args, i, bad)) == 4
    assert f(*but(but(args, 0, packed(L=2)), 14, Bd._Strides(0, 0, 128, 4096))) == 4
    assert f(*but(args, 14, Bd._Strides(0, 8192, 0, 4096))) == 4
    for i in (6, 8):
        assert f(*but(args, i, Bd._Strides(0, 8192, 128, 1 << 26))) == 7
    assert f(*but(args, 0, packed(T=1 << 22, H=2048, Hkv=1, S=1))) == 7
    # (blocks of the states in more than 31 bits: so many layers and heads that tiles are too many first)
    for S, rows in ((2, 10), (1, 10)):
        need = P.cross_workspace_bytes(S, 1, 4, 2, 10, 100, 128, torch.bfloat16, rows)
        if need:
            for i, x in ((15, None), (15, C.c_void_p(4104)), (16, need - 1)):
                assert f(*but(but(args, 0, packed(S=S)), i, x)) == 5
    for bad in (dict(T=0), dict(D=96), dict(S=0), dict(M=0), dict(M=(1 << 22) + 1), dict(max_rows=0), dict(max_rows=11)):
        d = {**dict(S=2, L=1, H=4, Hkv=2, T=10, M=100, D=128, max_rows=10), **bad}
        assert P.cross_workspace_bytes(dtype=torch.bfloat16, **d) == 0
    assert P.cross_workspace_bytes(2, 1, 4, 2, 10, 100, 128, torch.float32, 10) == 0


def test_cross_binding_refuses(monkeypatch):
    q, kv = torch.zeros((1, 4, 6, 64)), torch.zeros((1, 2, 30, 64))
    off, to, scale = torch.tensor([0, 6], dtype=torch.int32), torch.tensor([0, 30], dtype=torch.int32), torch.ones(1)
    good = dict(q=q, k=kv, v=kv, row_off=off, state_off=to, scale=scale, max_rows=6)
    with pytest.raises(ValueError, match="GPU"):
        P.prefixkv_cross_attn(**good)

    class Library:
        prefixkv_cross_workspace_bytes = P.load().prefixkv_cross_workspace_bytes

        def __getattr__(self, name):
            return lambda *a: pytest.fail(f"{name} was called")
    monkeypatch.setattr(Bd, "_here", lambda *a: 0)
    monkeypatch.setattr(Bd, "load", Library)
    for bad in (dict(k=kv[:, :, :20]), dict(v=kv.bfloat16()), dict(k=kv.bfloat16(), v=kv.bfloat16()), dict(k=kv[0], v=kv[0]),
                dict(k=kv[..., :32], v=kv[..., :32]), dict(q=q.half(), k=kv.half(), v=kv.half()), dict(out=q[:, :2]), dict(out=q.bfloat16()),
                dict(row_off=off.long()), dict(state_off=to[:1]), dict(state_off=torch.zeros(3, dtype=torch.int32)),
                dict(scale=scale.double()), dict(scale=torch.ones(2)), dict(seen=torch.zeros(5, dtype=torch.int32)),
                dict(seen=torch.zeros(6, dtype=torch.int64)), dict(seen=torch.zeros(12, dtype=torch.int32)[::2]),
                dict(max_rows=1 << 32), dict(q=q.transpose(2, 3).contiguous().transpose(2, 3))):
        with pytest.raises((ValueError, TypeError)):
            P.prefixkv_cross_attn(**{**good, **bad})


def test_binding_refuses(monkeypatch):
    x, sc = torch.zeros((2, 3, 10)), torch.zeros((2, 3))
    with pytest.raises(ValueError, match="GPU"):
        P.prefixkv_beam_select(x, sc)
    c = P.paged_cache(6, 2, 2, 64, 16, 5, 2, device="cpu")
    par = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        P.prefixkv_page_reorder(c, par)

    class Library:
        prefixkv_beam_workspace_bytes = P.load().prefixkv_beam_workspace_bytes
        prefixkv_reorder_workspace_bytes = P.load().prefixkv_reorder_workspace_bytes

        def __getattr__(self, name):
            return lambda *a: pytest.fail(f"{name} was called")
    monkeypatch.setattr(Bd, "_here", lambda *a: 0)
    monkeypatch.setattr(Bd, "load", Library)
    ended = torch.zeros((2, 3), dtype=torch.bool)
    out = torch.zeros((2, 3), dtype=torch.int32)
    for bad in (dict(logits=x[0]), dict(logits=x[:, :, ::2]), dict(logits=torch.zeros((3, 2, 10)).transpose(0, 1)), dict(logits=x.double()),
                dict(logits=x[:, :2]), dict(scores=sc.double()), dict(scores=sc[:1]), dict(scores=torch.zeros((3, 2)).t()),
                dict(ended=ended), dict(ended_out=ended), dict(ended=ended.int(), end_token=1), dict(ended=ended[:1], end_token=1),
                dict(end_token=10), dict(end_token=-1), dict(end_token=(1 << 32) + 1), dict(tokens=out.long()), dict(parents=out[:1]),
                dict(scores_out=sc.double()), dict(ended_out=ended.int(), end_token=2), dict(ws=torch.zeros(16))):
        with pytest.raises((ValueError, TypeError)):
            P.prefixkv_beam_select(**{**dict(logits=x, scores=sc), **bad})
    for bad in (dict(parents=par.long()), dict(parents=par[0]), dict(parents=par[:1]), dict(parents=torch.zeros((3, 2), dtype=torch.int32).t()),
                dict(status=out), dict(table_out=c.table[:1]), dict(lens_out=c.lens.long()), dict(state_out=out), dict(ws=torch.zeros(4))):
        with pytest.raises(ValueError):
            P.prefixkv_page_reorder(c, **{**dict(parents=par), **bad})


def test_paths_refuse(monkeypatch):
    import paper_2412_03409_amd.pipeline as pipeline

    def path(**kw):
        return pipeline.PagedPath(6, 1, 2, 1, 64, torch.ones(1), P.rope_plan(64, device="cpu"), num_pages=4, max_pages=2, device="cpu", **kw)
    for beams in (0, 4, 33, -1):
        with pytest.raises(ValueError, match="beams"):
            path(beams=beams)
    for name in ("prefixkv_rope", "prefixkv_page_reorder", "prefixkv_beam_select", "prefixkv_cross_attn"):
        monkeypatch.setattr(pipeline.B_, name, lambda *a, **kw: pytest.fail("a step was made"))
    three, one = path(beams=3), path()
    q, k = torch.zeros((1, 2, 6, 64), dtype=torch.bfloat16), torch.zeros((1, 1, 6, 64), dtype=torch.bfloat16)
    pos = torch.zeros((1, 6), dtype=torch.int32)
    with pytest.raises(ValueError, match="first place"):
        three.prefill([1], [5], q, k, k, pos, [5])
    for bad in (torch.zeros((3, 2), dtype=torch.int32), torch.zeros(6, dtype=torch.int32)):
        with pytest.raises(ValueError, match="parents"):
            three.follow(bad)
    with pytest.raises(ValueError, match="one beam"):
        one.follow(torch.zeros((6, 1), dtype=torch.int32))
    with pytest.raises(ValueError, match="one beam"):
        one.advance(torch.zeros((6, 1, 9)), torch.zeros((6, 1)))
    with pytest.raises(ValueError, match="logits"):
        three.advance(torch.zeros((6, 9)), torch.zeros((2, 3)))
    for lengths in ([1, 1], [1, 1, 1, 1, 1, 2], [-1, 1, 1, 1, 1, 1]):
        with pytest.raises(ValueError, match="place"):
            three.cross(lengths, q, k, k, torch.zeros(3, dtype=torch.int32))


def test_plain_forms_on_hand_worked_numbers():
    inf = math.inf
    # two beams over two tokens: 1/4, 3/4 of the first, halves of the second; scores log 1/2 and log 1
    x = np.log(np.array([[[1.0, 3.0], [5.0, 5.0]]]))
    t, p, s, over, gap = R.select(x, np.log([[0.5, 1.0]]), None, None)
    assert (t.tolist(), p.tolist()) == ([[0, 1]], [[1, 1]])
    np.testing.assert_allclose(np.exp(s), [[0.5, 0.5]])
    # the second has ended by token 1; the first may not take token 1; a third one that is dead
    x = np.array([[[0.0, -inf], [9.0, 9.0], [0.0, 0.0]]])
    t, p, s, over, _ = R.select(x, np.array([[-2.0, -1.0, -inf]]), np.array([[False, True, False]]), 1)
    assert (t.tolist(), p.tolist(), s.tolist(), over.tolist()) == ([[1, 0, -1]], [[1, 0, -1]], [[-1, -2, -inf]], [[True, False, False]])
    # pages of 2: place 0 has 3 entries on pages 5, 7, place 1 one on page 2; both become place 0: page 7 is copied to 9, 2 is free
    pool = np.arange(10.0).repeat(2).reshape(10, 1, 2, 1) * 10 + np.array([0, 1]).reshape(1, 1, 2, 1)
    st, table, lens, ring, state, (kp,) = R.reorder(np.array([[0, 0]]), np.array([[[5, 7]], [[2, -1]]]), np.array([[3], [1]]),
                                                    np.array([0, 9, 1, -1, -1, -1, -1, -1, -1, -1]), np.array([1, 2]), 2, [pool])
    assert (st, table.tolist(), lens.tolist(), state.tolist()) == (0, [[[5, 7]], [[5, 9]]], [[3], [3]], [2, 2])
    assert ring.tolist()[:4] == [0, 9, 1, 2] and kp[9, 0, :, 0].tolist() == [70, 91] and kp[7, 0, :, 0].tolist() == [70, 71]
    # both are empty: the shared page comes back once
    st, table, lens, ring, state, _ = R.reorder(np.array([[-1, -1]]), table, lens, ring, state, 2)
    assert (st, lens.tolist(), state.tolist(), ring.tolist()[4:7]) == (0, [[0], [0]], [2, 5], [5, 7, 9])
