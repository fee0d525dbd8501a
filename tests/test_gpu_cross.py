"""Attention of packed rows to states of another length, against its plain form in 64 bits, with the bars of the other attention
operators (test_gpu_serving.py)."""
import numpy as np
import pytest
import torch

import beam_reference as R
import paper_2412_03409_amd as P
from test_gpu_serving import BF16, DEV, F32, close, f64, gen, i32, offsets, projected

pytestmark = pytest.mark.gpu


def inputs(seed, L, H, Hkv, n, m, D, dtype, first=0, pad=0, before=0, behind=0):
    """Rows and states as projections leave them, rows and states of nobody on both sides."""
    g = gen(seed)
    off, to = offsets(n, first), offsets(m, before)
    T, M = int(off[-1]) + pad, max(1, int(to[-1]) + behind)
    q, _, _ = projected(g, L, H, Hkv, T, D, dtype)
    kv = torch.randn((L, M, 2 * Hkv, D), generator=g)
    kv[:, ::7, :Hkv] *= 3
    kv = kv.to(dtype).to(DEV)
    k, v = kv[:, :, :Hkv].permute(0, 2, 1, 3), kv[:, :, Hkv:].permute(0, 2, 1, 3)
    scale = torch.tensor([0.1 if i % 2 else -0.2 for i in range(L)], device=DEV)
    return q, k, v, off, to, scale


def check(q, k, v, off, to, scale, most, seen=None, max_rows=None):
    L, H, T, D = q.shape
    out = torch.full((L, T, H, D), 9.0, dtype=q.dtype, device=DEV).permute(0, 2, 1, 3)
    got = P.prefixkv_cross_attn(q, k, v, i32(off), i32(to), scale, most, seen=None if seen is None else i32(seen), out=out)
    assert got is out
    want, mag = R.cross(f64(q), off, f64(k), f64(v), to, scale.double().cpu().numpy(), seen, max_rows)
    close(out, want, mag, q.dtype)
    assert bool((out[torch.from_numpy(np.isnan(want)).to(DEV)] == 9).all())     # rows of nobody are left as they were
    return out


CASES = [  # rows, states, H, Hkv, D
    ([1], [1], 1, 1, 64), ([1], [577], 32, 8, 128), ([4, 4, 4], [100, 0, 33], 4, 4, 128), ([1, 0, 1], [31, 500, 32], 7, 1, 64),
    ([3], [2000], 8, 8, 64), ([8, 8], [64, 65], 4, 1, 128), ([1, 1], [0, 0], 2, 2, 64),
    ([40], [577], 4, 2, 128), ([33, 1, 129], [64, 1, 130], 6, 2, 64), ([200, 0, 70], [0, 900, 63], 3, 3, 128), ([128, 64], [65, 128], 2, 1, 64),
    ([5, 90], [700, 2], 12, 4, 128), ([300], [40], 2, 2, 64), ([17, 100, 3, 64], [130, 1000, 10, 129], 8, 2, 128),
]


@pytest.mark.parametrize("n,m,H,Hkv,D", CASES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("edges", [False, True])
def test_cross_attn(n, m, H, Hkv, D, dtype, edges):
    kw = dict(first=2, pad=3, before=5, behind=4) if edges else {}
    q, k, v, off, to, scale = inputs(sum(n) + sum(m), 2, H, Hkv, n, m, D, dtype, **kw)
    check(q, k, v, off, to, scale, max(max(n), 1))


@pytest.mark.parametrize("n,m,H,Hkv,D", CASES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("what", ["any", "rising", "few"])
def test_cross_attn_of_the_first_states(n, m, H, Hkv, D, dtype, what):
    """Rows see any number of states, also none, more than there are, or fewer than none; what they do not see is NaN and infinite."""
    q, k, v, off, to, scale = inputs(sum(n) * sum(m) + H, 1, H, Hkv, n, m, D, dtype, first=1, pad=2)
    T = q.shape[2]
    r = np.random.default_rng(T)
    if what == "any":
        seen = r.integers(-3, max(m) + 5, size=T)
    elif what == "rising":
        seen = np.arange(T) * max(m) // T
    else:
        seen = np.minimum(3, r.integers(0, 40, size=T))
    seen[r.random(T) < 0.1] = 1 << 30
    seen[r.random(T) < 0.1] = -(1 << 31)
    check(q, k, v, off, to, scale, max(max(n), 1), seen)
    # states that no row sees, and those that some rows do not
    for s in range(len(n)):
        rows = seen[off[s]:off[s + 1]]
        most = int(np.clip(rows, 0, m[s]).max()) if len(rows) else 0
        a, b = to[s] + most, to[s + 1]
        k[:, :, a:b] = float("nan")
        v[:, :, a:b] = float("inf")
        least = int(np.clip(rows, 0, m[s]).min()) if len(rows) else 0
        if least < most:
            v[:, :, to[s] + least, ::3] = float("-inf")
            k[:, :, to[s] + least] = 0.25
    L, H, T, D = q.shape
    out = P.prefixkv_cross_attn(q, k, v, i32(off), i32(to), scale, max(max(n), 1), seen=i32(seen))
    want, mag = R.cross(f64(q), off, f64(k), f64(v), to, scale.double().cpu().numpy(), seen)
    finite = np.isfinite(want) & np.isfinite(mag)
    masked = torch.from_numpy(finite).to(DEV)
    assert bool((~torch.isfinite(out.float()))[torch.from_numpy(np.isinf(want)).to(DEV)].all())
    close(torch.where(masked, out, torch.zeros_like(out)), np.where(finite, want, 0.0), np.where(finite, mag, 0.0), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,most", [([9, 30, 2], 4), ([200, 90, 150], 100)])
def test_cross_attn_of_the_first_rows(dtype, n, most):
    """Sequences with more rows than the call names: the further ones stay as they are."""
    q, k, v, off, to, scale = inputs(3, 1, 4, 2, n, [100, 70, 300], 64, dtype)
    check(q, k, v, off, to, scale, most, max_rows=most)
    check(q, k, v, off, to, scale, most, seen=np.arange(sum(n)) * 3, max_rows=most)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [[2, 1], [70, 40]])
def test_cross_attn_lowest_values_and_infinities(dtype, n):
    H, Hkv, D, m = 2, 1, 64, [300, 90]
    q, k, v, off, to, _ = inputs(6, 1, H, Hkv, n, m, D, dtype)
    q = torch.zeros_like(q)
    q[..., 0] = 1.0
    k[..., 1:] = 0
    k[:, :, :20, 0] = float("-inf")
    k[:, :, 20:300, 0] = torch.finfo(dtype).min
    k[:, :, 300:, 0] = float("-inf")
    out = check(q, k, v, off, to, torch.ones(1, device=DEV), max(n))
    assert bool((out[:, :, off[1]:] == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_cross_attn_strides(dtype):
    """Heads first, layers and heads that are repeated, rows far apart; K and V of different layouts."""
    L, H, Hkv, D, n, m = 2, 4, 2, 64, [3, 50], [90, 130]
    q, k, v, off, to, scale = inputs(8, L, H, Hkv, n, m, D, dtype)
    check(q.contiguous(), k.contiguous(), v, off, to, scale, 50)
    check(q, k[:1].expand(2, -1, -1, -1), v[:, :1].expand(-1, 2, -1, -1), off, to, scale, 50)
    room = torch.empty((L, Hkv, sum(m), 5 * D), dtype=dtype, device=DEV)
    room[..., 2 * D:3 * D] = k
    check(q, room[..., 2 * D:3 * D], v, off, to, scale, 50)


def test_cross_attn_more_texts_than_lanes():
    n, m = [1 + i % 4 for i in range(70)], [(37 * i) % 200 for i in range(70)]
    q, k, v, off, to, scale = inputs(9, 1, 2, 1, n, m, 64, BF16)
    check(q, k, v, off, to, scale, 4)
    n = [1] * 33 + [40, 0] + [1] * 35
    m = [20] * 33 + [2500, 5] + [60] * 35
    q, k, v, off, to, scale = inputs(10, 1, 2, 1, n, m, 64, BF16)
    check(q, k, v, off, to, scale, 40)


@pytest.mark.parametrize("n,m,H,Hkv,seen", [([130], [6000], 2, 1, False), ([130], [6000], 2, 1, True), ([64, 100], [9000, 3000], 4, 1, False),
                                            ([64, 100], [9000, 300], 4, 4, True)])
def test_cross_attn_cut_over_the_states(n, m, H, Hkv, seen):
    """Few tiles over many states: tiles are cut, and parts may lie behind what their rows see."""
    q, k, v, off, to, scale = inputs(12, 1, H, Hkv, n, m, 128, BF16)
    limit = (np.arange(sum(n)) * 97) % 2500 if seen else None
    assert P.cross_workspace_bytes(len(n), 1, H, Hkv, sum(n), sum(m), 128, BF16, max(n)) > 0
    check(q, k, v, off, to, scale, max(n), limit)


def test_cross_attn_offsets_that_cannot_be():
    """Rows or states of a sequence whose offsets descend or pass the end: none."""
    q, k, v, _, _, scale = inputs(13, 1, 2, 2, [10], [40], 64, BF16)
    for dtype in (BF16, F32):
        q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
        for off, to, good in (([0, 4, 2, 10], [0, 40, 40, 40], [(0, 4)]), ([0, 5, 10], [0, 41, 41], []), ([-1, 5, 10], [0, 20, 40], [(5, 10)]),
                              ([0, 5, 11], [0, 20, 40], [(0, 5)]), ([0, 5, 10], [30, 10, 40], [(5, 10)]), ([0, 5, 10], [-5, 10, 40], [(5, 10)])):
            out = torch.full_like(q, 9.0)
            P.prefixkv_cross_attn(q, k, v, i32(off), i32(to), scale, 10, out=out)
            for s in range(len(off) - 1):
                a, b, x, y = off[s], off[s + 1], to[s], to[s + 1]
                if not 0 <= a < b <= 10 or any(off[i] > off[i + 1] for i in range(len(off) - 1)):
                    continue
                here = out[:, :, a:b]
                if not 0 <= x < y <= 40:
                    assert bool((here == 0).all())
                else:
                    want, mag = R.cross(f64(q), [a, b], f64(k), f64(v), [x, y], scale.double().cpu().numpy())
                    close(here, want[:, :, a:b], mag[:, :, a:b], dtype)


@pytest.mark.parametrize("n,m", [([4, 1, 3], [700, 33, 2000]), ([9, 150, 30], [90, 700, 31]), ([100, 2], [6000, 300])])
def test_cross_attn_is_repeatable_and_replays_from_a_graph(n, m):
    H, Hkv, D = 8, 2, 128
    q, k, v, off, to, scale = inputs(14, 1, H, Hkv, n, m, D, BF16)
    off, to, seen = i32(off), i32(to), i32(np.arange(sum(n)) * 20)
    ws = torch.empty(max(1, P.cross_workspace_bytes(len(n), 1, H, Hkv, sum(n), sum(m), D, BF16, max(n))), dtype=torch.uint8, device=DEV)
    for lim in (None, seen):
        want = P.prefixkv_cross_attn(q, k, v, off, to, scale, max(n), seen=lim).clone()
        out = torch.empty_like(q)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            P.prefixkv_cross_attn(q, k, v, off, to, scale, max(n), seen=lim, out=out)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            P.prefixkv_cross_attn(q, k, v, off, to, scale, max(n), seen=lim, out=out, ws=ws)
        for i in range(4):
            out.zero_()
            ws.fill_(255 * (i % 2))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            assert torch.equal(P.prefixkv_cross_attn(q, k, v, off, to, scale, max(n), seen=lim), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_states_behind_the_first_four_gigabytes(dtype):
    """Rows of states 2^24 elements apart: 150 of them pass 2^32 bytes."""
    H, Hkv, D, n, m = 2, 1, 64, [3, 67], [20, 150]
    q, k, v, off, to, scale = inputs(15, 1, H, Hkv, n, m, D, dtype)
    want = P.prefixkv_cross_attn(q, k, v, i32(off), i32(to), scale, 67)
    few = P.prefixkv_cross_attn(q, k, v, i32([0, 3, 6]), i32(to), scale, 3)
    room = torch.empty(sum(m) << 24, dtype=dtype, device=DEV).view(sum(m), 1 << 24)
    far = []
    for x, at in ((k, 0), (v, 1024)):
        y = room[:, at:at + Hkv * D].view(sum(m), Hkv, D).permute(1, 0, 2)[None]
        y.copy_(x)
        far.append(y)
    assert torch.equal(P.prefixkv_cross_attn(q, *far, i32(off), i32(to), scale, 67), want)
    assert torch.equal(P.prefixkv_cross_attn(q, *far, i32([0, 3, 6]), i32(to), scale, 3)[:, :, :6], few[:, :, :6])


def large(seed, n, m, H, Hkv, D, heads_tiles=230, **kw):
    """Inputs with so many rows and states of nobody that a call looks at what the rows see before it shares them out."""
    S, grp = len(n), H // Hkv
    T = heads_tiles // Hkv * 128 // grp
    M = S * 64 * (8192 // heads_tiles + 3)
    q, k, v, off, to, scale = inputs(seed, 1, H, Hkv, n, m, D, BF16, pad=max(0, T - sum(n)), behind=max(0, M - sum(m)), **kw)
    tiles = (q.shape[2] * grp // 128 + min(S, q.shape[2])) * Hkv
    assert tiles < 2048 and tiles * k.shape[2] / S / 64 >= 8192
    return q, k, v, off, to, scale


LARGE = [  # rows, states, H, Hkv, D
    ([40], [2600], 2, 2, 128), ([33, 1, 129], [64, 1, 2130], 6, 2, 64), ([200, 0, 70], [0, 3000, 900], 3, 3, 128), ([128, 64], [65, 6000], 2, 1, 64),
    ([5, 90], [700, 2], 12, 4, 128), ([17, 100, 3, 64], [1300, 1000, 10, 4097], 8, 1, 64), ([1, 34], [5000, 3], 8, 8, 64),
]


@pytest.mark.parametrize("n,m,H,Hkv,D", LARGE)
@pytest.mark.parametrize("what", ["any", "rising", "few", "none", "all"])
def test_cross_attn_shared_out_by_what_rows_see(n, m, H, Hkv, D, what):
    q, k, v, off, to, scale = large(sum(n) + H, n, m, H, Hkv, D, first=3, before=7)
    T = q.shape[2]
    r = np.random.default_rng(sum(m))
    seen = {"any": r.integers(-3, max(m) + 5, size=T), "rising": (np.arange(T) - 3) * max(m) // sum(n), "few": np.minimum(3, r.integers(0, 40, size=T)),
            "none": np.full(T, -1), "all": np.full(T, 1 << 30)}[what].clip(-(1 << 31), 1 << 30)
    for s in range(len(n)):                                     # what no row sees
        rows = seen[off[s]:off[s + 1]]
        most = int(np.clip(rows, 0, m[s]).max()) if len(rows) else 0
        k[:, :, to[s] + most:to[s + 1]] = float("nan")
        v[:, :, to[s] + most:to[s + 1]] = float("inf")
    check(q, k, v, off, to, scale, max(n), seen)
    check(q, k, v, off, to, scale, 35, seen, max_rows=35)


def test_cross_attn_shared_out_values_that_some_rows_must_not_see():
    n, m = [64, 40], [3000, 500]
    q, k, v, off, to, scale = large(21, n, m, 4, 2, 64)
    seen = np.full(q.shape[2], 1 << 20)
    seen[:30], seen[70:90] = 1111, 130
    v[:, :, 1111, ::3] = float("inf")
    v[:, :, to[1] + 130, 5] = float("nan")
    out = P.prefixkv_cross_attn(q, k, v, i32(off), i32(to), scale, 64, seen=i32(seen))
    want, mag = R.cross(f64(q), off, f64(k), f64(v), to, scale.double().cpu().numpy(), seen)
    want, mag, out = want[:, :, :104], mag[:, :, :104], out[:, :, :104]
    finite = np.isfinite(want) & np.isfinite(mag)
    assert not finite.all() and finite[:, :, :30].all() and finite[:, :, 70:90].all()
    here = torch.from_numpy(finite).to(DEV)
    assert bool((~torch.isfinite(out.float()))[~here].all())
    close(torch.where(here, out, torch.zeros_like(out)), np.where(finite, want, 0.0), np.where(finite, mag, 0.0), BF16)


def test_cross_attn_shared_out_among_many_texts():
    """More texts than there are lanes, most of them short; and as many as a call is shared out for, and one more."""
    n = [1 + i % 4 for i in range(100)]
    n[41], n[99] = 150, 40
    m = [(37 * i) % 200 for i in range(100)]
    m[41], m[99] = 2500, 300
    for S in (100, 1024, 1025):
        rows, states = n + [1] * (S - 100), m + [9] * (S - 100)
        q, k, v, off, to, scale = inputs(22, 1, 1, 1, rows, states, 64, BF16, pad=20000, behind=S * 64 * (8192 // (20000 // 128 + S) + 2))
        assert (q.shape[2] // 128 + S) * k.shape[2] / S / 64 >= 8192 and q.shape[2] // 128 + S < 2048
        check(q, k, v, off, to, scale, 150, np.arange(q.shape[2]) % 2000)


def test_cross_attn_shared_out_offsets_that_cannot_be():
    q, k, v, _, _, scale = large(23, [50, 50, 50], [900, 900, 900], 2, 2, 64)
    T, M = q.shape[2], k.shape[2]
    seen = np.arange(T) * 7
    for off, to, good in (([0, 60, 40, 150], [0, 900, 1800, 2700], {0: (0, 60), 2: (40, 150)}), ([-1, 50, 100, T + 1], [0, 900, 1800, 2700], {1: (50, 100)}),
                          ([0, 50, 100, 150], [0, 900, 800, M + 1], {0: (0, 50)}), ([0, 50, 100, 150], [-5, 900, 1800, M], {1: (50, 100), 2: (100, 150)})):
        out = torch.full_like(q, 9.0)
        P.prefixkv_cross_attn(q, k, v, i32(off), i32(to), scale, 110, seen=i32(seen), out=out)
        for s in range(3):
            a, b, x, y = off[s], off[s + 1], to[s], to[s + 1]
            if s not in good:
                if 0 <= a < b <= T:
                    assert bool((out[:, :, a:b] == 0).all())
                continue
            if off[1] > off[2]:                                 # rows of two texts: either's answer
                a, b = (a, 40) if s == 0 else (60, b)
            want, mag = R.cross(f64(q), [a, b], f64(k), f64(v), [x, y], scale.double().cpu().numpy(), seen)
            close(out[:, :, a:b], want[:, :, a:b], mag[:, :, a:b], BF16)
        assert bool((out[:, :, 150:] == 9).all())


def test_cross_attn_shared_out_is_repeatable_and_replays_from_a_graph():
    n, m, H, Hkv, D = [150, 9, 40], [3000, 500, 2000], 8, 2, 128
    q, k, v, off, to, scale = large(24, n, m, H, Hkv, D)
    T, M = q.shape[2], k.shape[2]
    off, to = i32(off), i32(to)
    lims = [i32(np.arange(T) * 20), i32(3000 - np.arange(T) * 17)]
    wants = [P.prefixkv_cross_attn(q, k, v, off, to, scale, 150, seen=x, out=torch.zeros_like(q)) for x in lims]
    ws = torch.empty(P.cross_workspace_bytes(3, 1, H, Hkv, T, M, D, BF16, 150), dtype=torch.uint8, device=DEV)
    out, seen = torch.zeros_like(q), lims[0].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.prefixkv_cross_attn(q, k, v, off, to, scale, 150, seen=seen, out=out, ws=ws)
    for i in range(6):
        seen.copy_(lims[i % 2])
        out.zero_()
        ws.fill_(255 * (i // 2 % 2))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, wants[i % 2])
        assert torch.equal(P.prefixkv_cross_attn(q, k, v, off, to, scale, 150, seen=lims[i % 2], out=torch.zeros_like(q)), wants[i % 2])


FEW = [  # rows, states, H, Hkv, D, layers: rows of a head 1 ... 32; units 1 ... 1152, a workgroup of 8, 4 or 2 wavefronts each
    ([1], [1], 1, 1, 64, 1), ([1], [577], 32, 8, 128, 1), ([4, 4, 4], [100, 0, 33], 4, 4, 128, 2), ([1, 0, 1], [31, 700, 32], 7, 1, 64, 1),
    ([3], [767], 8, 8, 64, 1), ([8, 8], [64, 65], 4, 1, 128, 1), ([32, 1, 17], [257, 256, 255], 2, 2, 128, 1), ([1] * 30, [20 + i for i in range(30)], 10, 10, 64, 1),
    ([2, 0, 1] * 12, [(i * 23) % 70 for i in range(36)], 16, 16, 128, 2), ([3, 1] * 35, [(i * 37) % 90 for i in range(70)], 4, 2, 64, 1),
]


@pytest.mark.parametrize("n,m,H,Hkv,D,L", FEW)
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("what", ["all", "any", "rising", "few"])
def test_cross_attn_of_few_rows(n, m, H, Hkv, D, L, shared, what):
    """A unit a workgroup; and, with so many states of nobody that long units are to be expected, shared out over the wavefronts."""
    S = len(n)
    q, k, v, off, to, scale = inputs(sum(n) + sum(m) + H, L, H, Hkv, n, m, D, BF16, first=1, pad=2, before=3, behind=S * 32 * 66 if shared else 4)
    T = q.shape[2]
    assert (P.cross_workspace_bytes(S, L, H, Hkv, T, k.shape[2], D, BF16, max(n)) > 0) == shared
    r = np.random.default_rng(T)
    seen = {"all": None, "any": r.integers(-3, max(m) + 5, size=T), "rising": np.arange(T) * max(m) // T, "few": np.minimum(3, r.integers(0, 40, size=T))}[what]
    if seen is not None:
        seen[r.random(T) < 0.1] = 1 << 30
        seen[r.random(T) < 0.1] = -(1 << 31)
        for s in range(S):                                      # what no row sees
            rows = seen[off[s]:off[s + 1]]
            most = int(np.clip(rows, 0, m[s]).max()) if len(rows) else 0
            k[:, :, to[s] + most:to[s + 1]] = float("nan")
            v[:, :, to[s] + most:to[s + 1]] = float("inf")
    check(q, k, v, off, to, scale, max(n), seen)
    if max(n) > 2:
        check(q, k, v, off, to, scale, 2, seen, max_rows=2)


@pytest.mark.parametrize("shared", [False, True])
def test_cross_attn_of_few_rows_values_that_some_rows_must_not_see(shared):
    n, m = [4, 3], [400, 90]
    q, k, v, off, to, scale = inputs(31, 1, 8, 2, n, m, 128, BF16, behind=2 * 32 * 66 if shared else 0)
    seen = np.array([400, 77, 300, 90, 90, 1, 89])
    v[:, :, 77, ::5] = float("inf")
    v[:, :, 300:310, 3] = float("nan")
    v[:, :, to[1] + 89, 9] = float("-inf")
    out = P.prefixkv_cross_attn(q, k, v, i32(off), i32(to), scale, 4, seen=i32(seen))
    want, mag = R.cross(f64(q), off, f64(k), f64(v), to, scale.double().cpu().numpy(), seen)
    finite = np.isfinite(want) & np.isfinite(mag)
    assert finite[:, :, [1, 5, 6]].all() and not finite.all()
    here = torch.from_numpy(finite).to(DEV)
    assert bool((~torch.isfinite(out.float()))[~here].all())
    close(torch.where(here, out, torch.zeros_like(out)), np.where(finite, want, 0.0), np.where(finite, mag, 0.0), BF16)


@pytest.mark.parametrize("n", [[2, 1], [20, 12]])
def test_cross_attn_of_few_rows_shared_out_lowest_values_and_infinities(n):
    """Scores that are all the type's lowest number weigh the same; keys of -inf weigh nothing."""
    H, Hkv, D, m = 1, 1, 64, [300, 90]
    for behind in (0, 2 * 32 * 66):
        q, k, v, off, to, _ = inputs(32, 1, H, Hkv, n, m, D, BF16, behind=behind)
        q = torch.zeros_like(q)
        q[..., 0] = 1.0
        k[..., 1:] = 0
        k[:, :, :m[0], 0] = torch.finfo(BF16).min
        k[:, :, m[0]:, 0] = float("-inf")
        k[:, :, m[0] + 40, 0] = 1.0
        scale = torch.tensor([1.0], device=DEV)
        out = P.prefixkv_cross_attn(q, k, v, i32(off), i32(to), scale, max(n))
        x = f64(v)[0, 0]
        for s, want in ((0, x[:m[0]].mean(0)), (1, x[m[0] + 40])):
            got = out[0, 0, off[s]:off[s + 1]].double().cpu().numpy()
            bar = 2.0 ** -8 * np.abs(want) + (2.0 ** -16 + 2e-4) * np.abs(x[:m[0]]).mean(0) * (s == 0) + 1e-30
            assert (np.abs(got - want) <= bar).all()


@pytest.mark.parametrize("shared", [False, True])
def test_cross_attn_of_few_rows_is_repeatable_and_replays_from_a_graph(shared):
    n, m, H, Hkv, D = [4, 1, 3], [700, 33, 500], 8, 2, 128
    q, k, v, off, to, scale = inputs(33, 1, H, Hkv, n, m, D, BF16, behind=3 * 32 * 66 if shared else 0)
    off, to = i32(off), i32(to)
    lims = [i32(np.arange(8) * 90), i32(600 - np.arange(8) * 70)]
    wants = [P.prefixkv_cross_attn(q, k, v, off, to, scale, 4, seen=x) for x in lims]
    ws = torch.empty(P.cross_workspace_bytes(3, 1, H, Hkv, 8, k.shape[2], D, BF16, 4), dtype=torch.uint8, device=DEV)
    out, seen = torch.zeros_like(q), lims[0].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.prefixkv_cross_attn(q, k, v, off, to, scale, 4, seen=seen, out=out, ws=ws)
    for i in range(6):
        seen.copy_(lims[i % 2])
        out.zero_()
        ws.fill_(255 * (i // 2 % 2))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, wants[i % 2])
        assert torch.equal(P.prefixkv_cross_attn(q, k, v, off, to, scale, 4, seen=lims[i % 2]), wants[i % 2])
