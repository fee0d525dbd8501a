"""Packed prompts and paged caches: every operator against its plain form in 64 bits, at the sizes and masks where it can go
wrong, and all of them together as a serving program uses them.

Bars.  Whole numbers and moved rows: equality.  Rotation: sine and cosine are off by at most 2.5e-7 (Taylor remainder 2e-9,
fp32 evaluation 2 ulp), the two products and their sum by 2^-23 of |a| + |b|, in all 5e-7 (|a| + |b|), and half a step of the
storage type.  Attention: half a step of the output, and of every probability where they are rounded to bf16 (bf16 storage),
relative to sum p|v|; the logits are fp32 sums of D products, off by at most D 2^-24 sum|q k| scale, below 1e-4 for these
inputs, which a probability doubles: 2e-4 of sum p|v|."""
import numpy as np
import pytest
import torch

import paper_2412_03409_amd as P
import serving_reference as R
from tolerances import LSE_ATOL, LSE_RTOL

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().double().cpu().numpy()


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def offsets(n, first=0):
    return np.concatenate([[first], first + np.cumsum(n)]).astype(np.int64)


def projected(g, L, H, Hkv, T, D, dtype):
    """q, k, v as a fused projection leaves them: heads side by side, token by token."""
    x = torch.randn((L, T, H + 2 * Hkv, D), generator=g).to(dtype).to(DEV)
    return tuple(t.permute(0, 2, 1, 3) for t in (x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]))


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ---- pages -------------------------------------------------------------------------------------------
def page_state(seed, S, layers, ps, width, spare, ctx, empty=()):
    r = np.random.default_rng(seed)
    lens = r.integers(0, ctx + 1, size=(S, layers))
    for s in empty:
        lens[s] = 0
    held = -(-lens // ps)
    total = int(held.sum()) + spare
    perm = r.permutation(total)
    table = np.full((S, layers, width), -1, dtype=np.int64)
    at = 0
    for s in range(S):
        for l in range(layers):
            table[s, l, :held[s, l]] = perm[at:at + held[s, l]]
            at += held[s, l]
    head = int(r.integers(0, total)) if total else 0
    ring = np.full(total, -1, dtype=np.int64)
    ring[(head + np.arange(spare)) % total] = perm[at:]
    return lens, table, ring, np.array([head, spare])


def as_cache(lens, table, ring, state, ps):
    pool = torch.empty((len(ring), 1, ps, 64), dtype=BF16, device=DEV)
    return P.PagedCache(kp=pool, vp=pool, table=i32(table), lens=i32(lens), ring=i32(ring), state=i32(state))


@pytest.mark.parametrize("S,layers,ps,ctx,n,first,pad", [
    (1, 1, 16, 0, [1], 0, 0),                                  # the first token of an empty cache
    (3, 2, 16, 40, [0, 5, 0], 0, 0),                           # sequences without rows
    (4, 3, 32, 100, [1, 1, 1, 1], 2, 3),                       # a decode step, rows of nobody on both sides
    (5, 4, 16, 64, [17, 1, 200, 0, 33], 0, 1),
    (2, 1, 256, 1000, [3000, 1], 0, 0),
    (130, 40, 16, 50, [1] * 130, 0, 0),                        # more segments than one workgroup keeps
    (3, 33, 64, 300, [700, 129, 3], 1, 0),                     # more slots than one workgroup gives out
    (64, 64, 16, 30, [2] * 64, 0, 0),                          # exactly 4096 segments
])
@pytest.mark.parametrize("in_place", [False, True])
def test_page_append(S, layers, ps, ctx, n, first, pad, in_place):
    off = offsets(n, first)
    T = int(off[-1]) + pad
    lens, table, ring, state = page_state(S + T, S, layers, ps, -(-(ctx + max(n)) // ps), 7 + layers * (S + T // ps), ctx)
    want = R.append(lens, off, T, table, ring, state, ps)
    c = as_cache(lens, table, ring, state, ps)
    kw = {} if in_place else dict(lens_out=torch.empty_like(c.lens), state_out=torch.empty_like(c.state))
    for _ in range(1 if in_place else 2):     # with outputs of its own a call can be made again
        slots, status = P.prefixkv_page_append(c, i32(off), T, **kw)
    got = (int(status), *(x.cpu().numpy() for x in (kw.get("lens_out", c.lens), c.table, kw.get("state_out", c.state), slots)))
    for a, b in zip(got, want):
        np.testing.assert_array_equal(a, b)
    np.testing.assert_array_equal(c.ring.cpu().numpy(), ring)


@pytest.mark.parametrize("S,layers,ps,ctx,big", [(1, 1, 16, 100, 100), (4, 3, 16, 64, 90), (7, 5, 32, 500, 500),
                                                 (70, 64, 16, 60, 80), (9, 2, 128, 5000, 9000)])
def test_page_resize(S, layers, ps, ctx, big):
    r = np.random.default_rng(S)
    lens, table, ring, state = page_state(S, S, layers, ps, -(-big // ps), S * layers * -(-big // ps), ctx, empty=(0,))
    target = np.where(r.random((S, layers)) < 0.3, 0, r.integers(0, big + 1, size=(S, layers)))
    status, *want = R.resize(lens, target, table, ring, state, ps)
    assert status == 0
    c = as_cache(lens, table, ring, state, ps)
    assert int(P.prefixkv_page_resize(c, i32(target))) == 0
    for a, b in zip((c.lens, c.table, c.ring, c.state), want):
        np.testing.assert_array_equal(a.cpu().numpy(), b)
    # everything ends: every page is free again, none twice
    assert int(P.prefixkv_page_resize(c, torch.zeros_like(c.lens))) == 0
    assert int(c.state[1]) == len(ring) and int(c.lens.abs().sum()) == 0
    free = np.sort(c.ring.cpu().numpy())
    np.testing.assert_array_equal(free, np.arange(len(ring)))


@pytest.mark.parametrize("what,status", [("few", 1), ("long", 2), ("negative", 2), ("old", 2), ("head", 2), ("count", 2),
                                         ("many", 2), ("descending", 2), ("past", 2), ("before", 2)])
@pytest.mark.parametrize("layers", [3, 40])
def test_page_calls_that_are_refused_on_the_device(what, status, layers):
    S, ps, width = 120, 16, 20
    lens, table, ring, state = page_state(5, S, layers, ps, width, 40, 50)
    target, n, off = lens.copy(), np.zeros(S, dtype=int), None
    if what == "few":
        target[1:4, 0] += 16 * 14      # 42 pages
        n[2] = 16 * 15
    elif what == "long":
        target[1, 1] = width * ps + 1
        n[1] = width * ps + 1
    elif what == "negative":
        target[2, 0] = -1
    elif what == "old":
        lens[3, 0] = -5
    elif what == "head":
        state[0] = len(ring)
    elif what == "count":
        state[1] = -1
    elif what == "many":
        state[1] = len(ring)           # more free pages than can be: what comes back has no room
        target[1] = 0
        lens[1] = 33
    off = offsets(n)
    T = int(off[-1]) + 10
    if what == "descending":
        off[2:] += 3
        off[3] = 1
    elif what == "past":
        off[-1] = T + 1
    elif what == "before":
        off[0] = -1
    calls = []
    if what not in ("descending", "past", "before"):
        calls.append("resize")
    if what not in ("negative", "many"):
        calls.append("append")
    for call in calls:
        c = as_cache(lens, table, ring, state, ps)
        if call == "resize":
            st = P.prefixkv_page_resize(c, i32(target))
        else:
            slots, st = P.prefixkv_page_append(c, i32(off), T)
            assert bool((slots == -1).all())
        want = 1 if what == "few" else status
        assert int(st) == want, call
        for a, b in zip((c.lens, c.table, c.ring, c.state), (lens, table, ring, state)):
            np.testing.assert_array_equal(a.cpu().numpy(), b)


# ---- rotary positions ----------------------------------------------------------------------------------
def check_rotated(got, x, pos, axis, theta, rot, inter, dtype):
    want = R.rope(f64(x), pos.cpu().numpy(), axis, theta, rot, inter)
    a = np.abs(f64(x))
    mag = np.zeros_like(a)
    i = np.arange(rot // 2)
    first, second = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
    mag[..., first] = mag[..., second] = a[..., first] + a[..., second]
    assert np.all(np.abs(f64(got) - want) <= half_step(dtype) * np.abs(want) + 5e-7 * mag)
    np.testing.assert_array_equal(f64(got)[..., rot:], f64(x)[..., rot:])


ROPES = [
    # L, H, Hkv, T, D, rot, sections, interleaved, far
    (1, 1, 1, 1, 64, 64, [32], False, 0),
    (1, 4, 2, 1, 128, 128, [16, 24, 24], False, 100),
    (2, 3, 1, 33, 64, 32, [6, 5, 5], True, 10 ** 6),
    (1, 32, 8, 70, 128, 128, [64], True, 2 ** 31 - 1),
    (1, 7, 7, 257, 128, 48, [8, 8, 8], False, 10 ** 6),
    (3, 5, 5, 19, 64, 16, [4, 0, 4], True, 5000),
    (1, 28, 4, 700, 128, 64, [16, 16], False, 8192),
]


@pytest.mark.parametrize("L,H,Hkv,T,D,rot,sections,inter,far", ROPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("in_place", [False, True])
def test_rope(L, H, Hkv, T, D, rot, sections, inter, far, dtype, in_place):
    g = gen(T + H)
    q, k, _ = projected(g, L, H, Hkv, T, D, dtype)
    pos = torch.randint(-far, far + 1, (len(sections), T), generator=g).to(torch.int32).to(DEV)
    plan = P.rope_plan(rot, sections, theta=10000.0, interleaved=inter, cycled=T == 19, device=DEV)
    axis = plan.axis.cpu().numpy()
    q0, k0 = q.clone(), k.clone()
    qo, ko = P.prefixkv_rope(q, k, pos, plan, **(dict(q_out=q, k_out=k) if in_place else {}))
    check_rotated(qo, q0, pos, axis, 10000.0, rot, inter, dtype)
    check_rotated(ko, k0, pos, axis, 10000.0, rot, inter, dtype)


@pytest.mark.parametrize("L,H,Hkv,T,D,rot,sections,inter,far", ROPES)
@pytest.mark.parametrize("dtype,ps", [(BF16, 16), (F32, 64)])
def test_rope_store(L, H, Hkv, T, D, rot, sections, inter, far, dtype, ps):
    g = gen(T + H)
    q, k, v = projected(g, L, H, Hkv, T, D, dtype)
    pos = torch.randint(0, far + 1, (len(sections), T), generator=g).to(torch.int32).to(DEV)
    plan = P.rope_plan(rot, sections, theta=500000.0, interleaved=inter, device=DEV)
    pages = L * T // ps + 2
    c = P.paged_cache(1, L, Hkv, D, ps, pages, 4, dtype, DEV)
    c.kp.fill_(7.0), c.vp.fill_(-7.0)
    slots = torch.randperm(pages * ps, generator=g)[:L * T].view(L, T)
    if T > 3:
        slots[:, 1], slots[0, 2] = -1, pages * ps     # a row that pads the batch, a slot past the pool
    qo = P.prefixkv_rope_store(c, q, k, v, pos, plan, slots.contiguous().to(DEV))
    check_rotated(qo, q, pos, plan.axis.cpu().numpy(), 500000.0, rot, inter, dtype)
    used = torch.zeros(pages * ps, dtype=torch.bool)
    kp, vp = (x.permute(0, 2, 1, 3).reshape(pages * ps, Hkv, D) for x in (c.kp, c.vp))
    for l in range(L):
        real = (slots[l] >= 0) & (slots[l] < pages * ps)
        used[slots[l][real]] = True
        at = slots[l][real].to(DEV)
        t = real.nonzero()[:, 0].to(DEV)
        np.testing.assert_array_equal(f64(vp[at]), f64(v[l][:, t].transpose(0, 1)))
        check_rotated(kp[at].transpose(0, 1)[None], k[l:l + 1][:, :, t], pos[:, t], plan.axis.cpu().numpy(), 500000.0, rot,
                      inter, dtype)
    rest = (~used).to(DEV)
    assert bool((kp[rest] == 7).all()) and bool((vp[rest] == -7).all())


# ---- compaction into pages ---------------------------------------------------------------------------
@pytest.mark.parametrize("B,L,Hkv,N,D,dtype,ps,l0,extra", [
    (1, 1, 1, 1, 64, BF16, 16, 0, 0), (2, 3, 2, 65, 64, F32, 16, 1, 2), (1, 4, 3, 680, 128, BF16, 16, 0, 0),
    (2, 2, 4, 700, 128, BF16, 64, 2, 1), (1, 2, 1, 8192, 64, BF16, 256, 0, 0), (1, 2, 2, 1300, 128, F32, 32, 0, 0)])
def test_compact_paged(B, L, Hkv, N, D, dtype, ps, l0, extra):
    r = np.random.default_rng(N)
    layers = l0 + L + extra
    k = torch.randn((B, L, Hkv, N, 2 * D), generator=gen(N)).to(dtype).to(DEV)
    k, v = k[..., :D], k[..., D:]
    order = np.stack([r.permutation(N) for _ in range(B * L)]).reshape(B, L, N)
    lengths = r.integers(0, N + 1, size=(B, L))
    lengths[0, 0] = N
    lengths[-1, -1] = max(0, N - 1) if B * L > 1 else N
    width = -(-N // ps)
    c = P.paged_cache(B, layers, Hkv, D, ps, int((-(-lengths // ps)).sum()) + 3, width, dtype, DEV)
    c.kp.fill_(3.0), c.vp.fill_(4.0)
    target = np.zeros((B, layers), dtype=int)
    target[:, l0:l0 + L] = lengths
    assert int(P.prefixkv_page_resize(c, i32(target))) == 0
    kept = torch.full((B, L, N), -9, dtype=torch.int32, device=DEV)
    P.prefixkv_compact_paged(c, k, v, i32(order), i32(lengths), kept_pos=kept, l0=l0)
    table, used = c.table.cpu().numpy(), np.zeros((c.kp.shape[0], ps), dtype=bool)
    for b in range(B):
        for l in range(L):
            n = lengths[b, l]
            pos = np.sort(order[b, l, :n])
            np.testing.assert_array_equal(kept[b, l].cpu().numpy(), np.concatenate([pos, np.full(N - n, -9)]))
            j = np.arange(n)
            page = table[b, l0 + l, j // ps]
            used[page, j % ps] = True
            for pool, x in ((c.kp, k), (c.vp, v)):
                got = pool[torch.from_numpy(page).long().to(DEV), :, torch.from_numpy(j % ps).to(DEV)]
                assert torch.equal(got, x[b, l][:, torch.from_numpy(pos).to(DEV)].transpose(0, 1))
    rest = torch.from_numpy(~used).to(DEV)
    assert bool((c.kp.transpose(1, 2)[rest] == 3).all()) and bool((c.vp.transpose(1, 2)[rest] == 4).all())
    # without the positions; a page outside the pool is not written
    bad = int(table[0, l0, 0])
    c.table[0, l0, 0] = c.kp.shape[0]
    c.kp.fill_(3.0)
    P.prefixkv_compact_paged(c, k, v, i32(order), i32(lengths), l0=l0)
    assert bool((c.kp[bad] == 3).all())


# ---- packed prompts ------------------------------------------------------------------------------------
def close(got, want, mag, dtype):
    """(rows of nobody are NaN in `want` and left out)"""
    real = ~np.isnan(want)
    step = half_step(dtype)
    bar = step * np.abs(want) + (step * (dtype == BF16) + 2e-4) * mag
    off = np.abs(f64(got) - want)
    assert np.all(off[real] <= bar[real]), float(np.max((off - bar)[real]))


PROMPTS = [
    # L, H, Hkv, D, lengths, first, pad
    (1, 1, 1, 64, [1], 0, 0),
    (1, 2, 1, 128, [5, 0, 1, 70], 0, 0),
    (2, 4, 2, 64, [31, 32, 33, 64, 65], 3, 2),
    (1, 7, 1, 128, [127, 128, 129], 0, 5),
    (1, 3, 3, 128, [257, 1, 300], 0, 0),
    (1, 8, 2, 128, [0, 0, 513], 0, 0),
    (1, 5, 5, 64, [1] * 70, 0, 0),
    (3, 12, 4, 64, [200, 17], 0, 0),
    (1, 16, 2, 128, [90, 1, 40], 0, 0),
    (1, 1, 1, 128, [1200], 0, 0),
    (1, 2, 1, 64, [2500, 1, 200], 0, 1),                         # few long tiles: cut and joined
]


@pytest.mark.parametrize("L,H,Hkv,D,n,first,pad", PROMPTS)
@pytest.mark.parametrize("negative", [False, True])
def test_prefill_attn_packed(L, H, Hkv, D, n, first, pad, negative):
    off = offsets(n, first)
    T = int(off[-1]) + pad
    q, k, v = projected(gen(T + H), L, H, Hkv, T, D, BF16)
    scale = (torch.rand(L, generator=gen(1)) + 0.5) / D ** 0.5 * (-1 if negative else 1)
    for x in (q, k, v):      # what belongs to nobody is not looked at
        x[:, :, :first], x[:, :, int(off[-1]):] = float("nan"), float("inf")
    out, lse = torch.full_like(q, 77.0), torch.full((L * H * T,), 77.0, device=DEV)
    P.prefixkv_prefill_attn_packed(q, k, v, i32(off), scale.to(DEV), out=out, lse=lse)
    want, mag, wlse = R.prompt(f64(q), f64(k), f64(v), off, scale.double().numpy())
    close(out, want, mag, BF16)
    assert bool((out[torch.from_numpy(np.isnan(want)).to(DEV)] == 77).all())
    real = ~np.isnan(wlse)
    z = f64(lse)
    assert np.all(z[~real] == 77)
    assert np.all(np.abs(z - wlse)[real] <= LSE_RTOL * np.abs(wlse[real]) + LSE_ATOL)


def test_prefill_attn_packed_later_rows_do_not_reach_earlier_ones():
    """NaN and infinities in a key or a value reach the rows from that position on, and no row before it."""
    H, Hkv, D, n = 4, 2, 128, [150, 70]
    off = offsets(n)
    q, k, v = projected(gen(3), 1, H, Hkv, sum(n), D, BF16)
    scale = torch.full((1,), D ** -0.5, device=DEV)
    clean = P.prefixkv_prefill_attn_packed(q, k, v, i32(off), scale)[0].clone()
    for at, bad in ((0, 140), (0, 77), (1, 33), (0, 64)):
        for x in (k, v):
            for value in (float("nan"), float("inf"), float("-inf")):
                y = x.clone()
                y[:, :, off[at] + bad, 5] = value
                out = P.prefixkv_prefill_attn_packed(q, y if x is k else k, y if x is v else v, i32(off), scale)[0]
                before = slice(int(off[at]), int(off[at]) + bad)
                other = slice(int(off[1]), None) if at == 0 else slice(0, int(off[1]))
                # (a tile with such a value may be summed in another order: half a step of the output apart)
                for part in (before, other):
                    assert torch.allclose(out[:, :, part].float(), clean[:, :, part].float(), rtol=2.0 ** -7, atol=2.0 ** -7)
                if x is v:
                    assert not bool(torch.isfinite(out[:, :, int(off[at]) + bad:int(off[at + 1]), 5]).any())


def test_prefill_attn_packed_feeds_the_importance():
    """The packed log-sum-exp of a sequence is what prefixkv_importance takes, rows and all."""
    L, H, Hkv, D, n = 2, 4, 2, 64, [130, 1, 67]
    off = offsets(n)
    q, k, v = projected(gen(9), L, H, Hkv, sum(n), D, BF16)
    scale = torch.tensor([0.1, 0.3], device=DEV)
    _, lse = P.prefixkv_prefill_attn_packed(q, k, v, i32(off), scale)
    for a, b in zip(off[:-1], off[1:]):
        qs, ks = q[None, :, :, a:b], k[None, :, :, a:b]
        mine = lse[L * H * a:L * H * b].view(1, L, H, b - a)
        got, want = P.prefixkv_importance(qs, ks, scale, lse=mine), P.prefixkv_importance(qs, ks, scale)
        assert torch.allclose(got, want, rtol=1e-3, atol=1e-6)


# ---- chunks over the paged cache -----------------------------------------------------------------------
def chunk_state(seed, S, layers, Hkv, D, ps, lens, dtype, width=None):
    """A pool of pages in no order; everything that is not an entry is NaN."""
    r = np.random.default_rng(seed)
    held = -(-lens // ps)
    width = int(max(1, held.max())) if width is None else width
    total = int(held.sum()) + 2
    perm = r.permutation(total)
    table = np.full((S, layers, width), 1 << 30, dtype=np.int64)
    c = P.PagedCache(kp=torch.full((total, Hkv, ps, D), float("nan"), dtype=dtype, device=DEV),
                     vp=torch.full((total, Hkv, ps, D), float("inf"), dtype=dtype, device=DEV),
                     table=i32(np.zeros((S, layers, width))), lens=i32(lens), ring=i32(np.zeros(total)), state=i32([0, 0]))
    at, g = 0, gen(seed)
    for s in range(S):
        for l in range(layers):
            for j in range(held[s, l]):
                table[s, l, j] = perm[at]
                m = min(ps, lens[s, l] - j * ps)
                for pool in (c.kp, c.vp):
                    pool[perm[at], :, :m] = torch.randn((Hkv, m, D), generator=g).to(dtype).to(DEV)
                at += 1
    c.table.copy_(i32(table))
    return c, table


CHUNKS = [
    # L, H, Hkv, D, ps, lens per sequence (after the append), n, first, pad, l0
    (1, 1, 1, 64, 16, [1], [1], 0, 0, 0),
    (1, 4, 4, 128, 16, [300, 1, 17], [1, 1, 1], 0, 0, 0),                   # a decode step
    (2, 8, 2, 128, 16, [65, 64, 0, 33], [1, 1, 0, 1], 1, 2, 1),             # a sequence that waits, padding, later layers
    (1, 7, 1, 64, 32, [500, 31], [2, 4], 0, 0, 0),
    (1, 32, 4, 128, 64, [129, 1000, 5], [4, 4, 4], 0, 1, 0),
    (1, 6, 2, 128, 128, [700, 40], [150, 40], 0, 0, 0),                     # a first question among others
    (3, 4, 1, 64, 256, [513, 100], [33, 32], 2, 0, 2),
    (1, 2, 2, 64, 16, [3, 0, 10], [8, 4, 10], 0, 0, 0),                     # more new rows than entries: rows that see nothing
    (1, 16, 16, 128, 16, [2000], [1], 0, 0, 0),
    (1, 64, 1, 128, 16, [900, 33], [1, 2], 0, 0, 0),
    (1, 3, 1, 128, 32, [2100], [260], 0, 0, 0),
    (1, 4, 4, 64, 16, [50, 0, 150], [150, 140, 10], 1, 1, 0),               # whole tiles that see nothing
    (1, 8, 2, 128, 64, [5000, 70, 640], [100, 2, 64], 0, 0, 0),             # few long tiles: cut and joined
    (2, 2, 1, 64, 16, [4100, 3000], [130, 128], 0, 0, 1),
]


@pytest.mark.parametrize("L,H,Hkv,D,ps,sizes,n,first,pad,l0", CHUNKS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_chunk_attn(L, H, Hkv, D, ps, sizes, n, first, pad, l0, dtype):
    r = np.random.default_rng(H)
    layers, off = l0 + L + 1, offsets(n, first)
    T = int(off[-1]) + pad
    lens = np.array(sizes)[:, None] + (np.arange(layers) - l0)[None, :] * r.integers(0, 3, size=(len(sizes), 1))
    lens = np.maximum(lens, 0)
    c, table = chunk_state(T + H, len(sizes), layers, Hkv, D, ps, lens, dtype)
    q, _, _ = projected(gen(H), L, H, Hkv, T, D, dtype)
    scale = (torch.rand(L, generator=gen(2)) + 0.5) / D ** 0.5 * (-1 if H % 4 == 0 else 1)
    out = torch.full((L, T, H, D), 55.0, dtype=dtype, device=DEV).permute(0, 2, 1, 3)
    P.prefixkv_chunk_attn(c, q, i32(off), scale.to(DEV), max(n), l0=l0, out=out)
    want, mag = R.chunk(f64(q), off, f64(c.kp), f64(c.vp), table, lens, scale.double().numpy(), l0)
    close(out, want, mag, dtype)
    assert bool((out[torch.from_numpy(np.isnan(want)).to(DEV)] == 55).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [[1, 1], [3, 2], [140, 90]])
def test_chunk_attn_pages_outside_the_pool_and_rows_beyond_the_most(dtype, n):
    L, H, Hkv, D, ps = 1, 4, 2, 64, 16
    lens = np.array([[400], [171]])
    c, table = chunk_state(8, 2, 1, Hkv, D, ps, lens, dtype)
    table[0, 0, 3], table[1, 0, 0], table[0, 0, 24] = -1, c.kp.shape[0], 1 << 30
    c.table.copy_(i32(table))
    off = offsets(n)
    q, _, _ = projected(gen(4), L, H, Hkv, int(off[-1]), D, dtype)
    scale = torch.full((1,), 0.2, device=DEV)
    for most in {max(n), max(1, max(n) - 1)}:
        out = torch.full_like(q, 9.0)
        P.prefixkv_chunk_attn(c, q, i32(off), scale, most, out=out)
        want, mag = R.chunk(f64(q), off, f64(c.kp), f64(c.vp), table, lens, scale.double().cpu().numpy(), max_rows=most)
        close(out, want, mag, dtype)
        assert bool((out[torch.from_numpy(np.isnan(want)).to(DEV)] == 9).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [[1, 1], [70, 40]])
def test_chunk_attn_lowest_values_and_infinities(dtype, n):
    """Scores of the type's lowest value count like any other; keys that score -inf weigh nothing, also all of them."""
    H, Hkv, D, ps = 2, 1, 64, 16
    lens = np.array([[300], [90]])
    c, table = chunk_state(6, 2, 1, Hkv, D, ps, lens, dtype)
    off = offsets(n)
    q = torch.zeros((1, H, int(off[-1]), D), dtype=dtype, device=DEV)
    q[..., 0] = 1.0
    k = c.kp.clone()
    k[..., 1:] = 0
    k[table[0, 0, 0], :, :, 0] = float("-inf")
    k[table[0, 0, 3:18].astype(int), :, :, 0] = torch.finfo(dtype).min
    k[table[1, 0, :6].astype(int), :, :, 0] = float("-inf")
    c.kp.copy_(k)
    scale = torch.ones(1, device=DEV)
    out = P.prefixkv_chunk_attn(c, q, i32(off), scale, max(n))
    want, mag = R.chunk(f64(q), off, f64(c.kp), f64(c.vp), table, lens, np.ones(1))
    close(out, want, mag, dtype)
    assert bool((out[:, :, off[1]:] == 0).all())


def test_chunk_attn_more_segments_than_lanes():
    """70 sequences: single tokens, and one of 40 rows over a long cache among them (tiles that are cut)."""
    H, Hkv, D, ps = 2, 1, 64, 16
    for n, sizes in (([1] * 70, [(37 * i) % 300 + 1 for i in range(70)]),
                     ([1] * 33 + [40] + [0] + [1] * 35, [20] * 33 + [2500] + [0] * 2 + [60] * 34)):
        lens = np.array(sizes)[:, None]
        c, table = chunk_state(11, 70, 1, Hkv, D, ps, lens, BF16, width=800)
        off = offsets(n)
        q, _, _ = projected(gen(12), 1, H, Hkv, int(off[-1]), D, BF16)
        scale = torch.full((1,), 0.15, device=DEV)
        out = P.prefixkv_chunk_attn(c, q, i32(off), scale, max(n))
        want, mag = R.chunk(f64(q), off, f64(c.kp), f64(c.vp), table, lens, scale.double().cpu().numpy())
        close(out, want, mag, BF16)


@pytest.mark.parametrize("n,sizes", [([1, 1, 1], [700, 33, 2000]), ([9, 150, 30], [90, 700, 31]), ([100, 2], [6000, 300])])
def test_chunk_attn_is_repeatable_and_replays_from_a_graph(n, sizes):
    """The same bits from every call, from another stream, and from a captured graph that is replayed with eager work between."""
    H, Hkv, D, ps = 8, 2, 128, 32
    lens = np.array(sizes)[:, None]
    c, _ = chunk_state(3, len(n), 1, Hkv, D, ps, lens, BF16)
    off = i32(offsets(n))
    q, _, _ = projected(gen(5), 1, H, Hkv, sum(n), D, BF16)
    scale = torch.full((1,), 0.1, device=DEV)
    ws = torch.empty(P.attn_workspace_bytes(len(n), 1, H, Hkv, sum(n), D, BF16, max_rows=max(n)), dtype=torch.uint8, device=DEV)
    want = P.prefixkv_chunk_attn(c, q, off, scale, max(n), ws=ws).clone()
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.prefixkv_chunk_attn(c, q, off, scale, max(n), out=out)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.prefixkv_chunk_attn(c, q, off, scale, max(n), out=out, ws=ws)
    for i in range(4):
        out.zero_()
        ws.fill_(255 * (i % 2))            # nothing is carried in it
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        torch.cuda.synchronize()
        assert torch.equal(P.prefixkv_chunk_attn(c, q, off, scale, max(n)), want)


def test_page_calls_replay_from_a_graph():
    """A captured append: every replay gives the next tokens their slots."""
    S, layers, ps, width = 6, 4, 16, 8
    lens, table, ring, state = page_state(2, S, layers, ps, width, 200, 40)
    c = as_cache(lens, table, ring, state, ps)
    off = offsets([1] * S)
    slots = torch.empty((layers, S), dtype=torch.int64, device=DEV)
    status = torch.empty(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(P.page_workspace_bytes(S, layers), dtype=torch.uint8, device=DEV)
    offd = i32(off)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.prefixkv_page_append(c, offd, S, slots=slots, status=status, ws=ws)
    for _ in range(40):
        g.replay()
        torch.cuda.synchronize()
        st, lens, table, state, want = R.append(lens, off, S, table, ring, state, ps)
        assert int(status) == st
        for a, b in zip((c.lens, c.table, c.state, slots), (lens, table, state, want)):
            np.testing.assert_array_equal(a.cpu().numpy(), b)


# ---- together ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,Hkv,D,ps", [(4, 2, 64, 16), (7, 1, 128, 64)])
def test_sequences_come_ask_again_and_go(H, Hkv, D, ps):
    """Packed prompts, what the search keeps of them in pages, a second question, decode steps, an end, a new prompt in the
    freed pages: every output against the definitions in 64 bits on the positions that were kept."""
    from paper_2412_03409_amd.pipeline import PagedPath
    L, S = 2, 4
    g = gen(H)
    scale = torch.tensor([0.15, 0.3])
    plan = P.rope_plan(D, [D // 2 - 2 * (D // 6), D // 6, D // 6], device=DEV)
    axis = plan.axis.cpu().numpy()
    path = PagedPath(S, L, H, Hkv, D, scale.to(DEV), plan, num_pages=52 if ps == 64 else 150, max_pages=400 // ps + 1, page_size=ps, device=DEV)
    keys = [[None] * L for _ in range(S)]      # rotated keys and values [Hkv,len,D] of every segment, as the cache must hold them

    def rows(T):
        x = projected(g, L, H, Hkv, T, D, BF16)
        pos = torch.randint(0, 3000, (3, T), generator=g).to(torch.int32).to(DEV)
        return (*x, pos)

    def rotated(x, pos):       # as the storage type holds it
        return torch.from_numpy(R.rope(f64(x), pos.cpu().numpy(), axis, 10000.0, D, False)).to(BF16).double().numpy()

    def prefill(places, lengths, budgets):
        q, k, v, pos = rows(sum(lengths))
        qr, kr, vr = rotated(q, pos), rotated(k, pos), f64(v)
        kept = []
        out = path.prefill(places, lengths, q, k, v, pos, budgets, kept_pos=kept)
        assert int(path.status) == 0
        off = offsets(lengths)
        want, mag, _ = R.prompt(qr, kr, vr, off, scale.double().numpy())
        close(out, want, mag, BF16)
        for i, (s, b) in enumerate(zip(places, budgets)):
            total = 0
            for l in range(L):
                pos_l = kept[i][l].cpu().numpy()
                pos_l = pos_l[pos_l >= 0]
                assert len(pos_l) == int(path.cache.lens[s, l])
                total += len(pos_l)
                keys[s][l] = [x[l][:, off[i] + pos_l] for x in (kr, vr)]
            assert total == b
    def extend(lengths, pad=0):
        T = sum(lengths) + pad
        q, k, v, pos = rows(T)
        qr, kr, vr = rotated(q, pos), rotated(k, pos), f64(v)
        out = path.extend(lengths, q, k, v, pos)
        assert int(path.status) == 0
        off = offsets(lengths)
        for s in range(S):
            t = slice(off[s], off[s + 1])
            for l in range(L):
                if lengths[s] == 0:
                    continue
                keys[s][l] = [np.concatenate([old, x[l][:, t]], axis=1) for old, x in zip(keys[s][l], (kr, vr))]
                kk, vv = keys[s][l]
                assert kk.shape[1] == int(path.cache.lens[s, l])
                for h in range(H):
                    o, m, _ = R.attend(qr[l, h, t], kk[h // (H // Hkv)], vv[h // (H // Hkv)], float(scale[l]), kk.shape[1] - lengths[s])
                    close(out[l:l + 1, h:h + 1, t], o[None, None], m[None, None], BF16)

    prefill([0, 2, 3], [70, 1, 130], [56, 2, 100])
    extend([5, 0, 1, 40], pad=3)
    for _ in range(3):
        extend([1, 0, 1, 1])
    free = int(path.cache.state[1])
    path.end([0])
    assert int(path.cache.state[1]) > free and path.cache.lens[0].tolist() == [0, 0]
    prefill([0, 1], [200, 33], [200, 20])
    extend([1, 2, 33, 60])
    extend([1, 1, 1, 1])
    # more than the pool has: nothing changes
    before = [x.clone() for x in (path.cache.lens, path.cache.table, path.cache.ring, path.cache.state)]
    P.prefixkv_page_resize(path.cache, torch.full_like(path.cache.lens, 399), status=path.status)
    assert int(path.status) == 1
    for a, b in zip((path.cache.lens, path.cache.table, path.cache.ring, path.cache.state), before):
        assert torch.equal(a, b)


def test_a_prompt_without_pages_leaves_the_path_as_it_was():
    """A prompt for a place that still has a sequence, refused for want of pages: every page, table row and length stays."""
    from paper_2412_03409_amd.pipeline import PagedPath
    L, H, Hkv, D = 2, 4, 2, 64
    g = gen(11)
    path = PagedPath(2, L, H, Hkv, D, torch.tensor([0.2, 0.3], device=DEV), P.rope_plan(D, device=DEV), num_pages=6, max_pages=8,
                     page_size=16, device=DEV)
    path.cache.kp.zero_(), path.cache.vp.zero_()

    def prefill(place, n, budget, kept):
        pos = torch.arange(n, dtype=torch.int32, device=DEV)[None]
        return path.prefill([place], [n], *projected(g, L, H, Hkv, n, D, BF16), pos, [budget], kept_pos=kept)

    kept = []
    prefill(0, 40, 60, kept)
    assert int(path.status) == 0 and int((kept[0] >= 0).sum()) == 60
    c = path.cache
    before = [x.clone() for x in (c.kp, c.vp, c.lens, c.table, c.ring, c.state)]
    kept = []
    prefill(0, 100, 200, kept)
    assert int(path.status) == 1 and int((kept[0] >= 0).sum()) == 0
    for a, b in zip((c.kp, c.vp, c.lens, c.table, c.ring, c.state), before):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pages_behind_the_first_four_gigabytes(dtype):
    """The same sequences in the last pages of a pool of more than 2^32 bytes and in a small one: rotation with the store, paged
    compaction and attention give the same bits."""
    S, H, Hkv, D, ps, n = 2, 8, 4, 128, 256, [40, 3]
    page = Hkv * ps * D * torch.finfo(dtype).bits // 8
    high = (1 << 32) // page + 9
    off, T = i32(offsets(n)), sum(n)
    scale = torch.full((1,), 0.1, device=DEV)
    plan = P.rope_plan(D, device=DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)[None]
    outs = []
    for pages in (12, high):
        g = gen(21)
        q, k, v = projected(g, 1, H, Hkv, T, D, dtype)
        kk, vv = torch.randn((2, S, 1, Hkv, 700, D), generator=g).to(dtype).to(DEV)
        order = torch.stack([torch.randperm(700, generator=g) for _ in range(S)]).to(torch.int32).to(DEV)[:, None].contiguous()
        lengths = i32([[600], [350]])
        c = P.paged_cache(S, 1, Hkv, D, ps, pages, 4, dtype, DEV)
        c.state.copy_(i32([pages - 8, 8]))                 # only the last eight pages are free
        assert int(P.prefixkv_page_resize(c, lengths)) == 0
        P.prefixkv_compact_paged(c, kk, vv, order, lengths)
        slots, status = P.prefixkv_page_append(c, off, T)
        assert int(status) == 0 and int(slots.min()) >= (pages - 8) * ps
        q = P.prefixkv_rope_store(c, q, k, v, pos, plan, slots)
        outs.append([P.prefixkv_chunk_attn(c, q, off, scale, 40)] +
                    [x[c.table[s, 0, :-(-int(c.lens[s, 0]) // ps)].long()].reshape(-1, Hkv, ps, D) for s in range(S) for x in (c.kp, c.vp)])
    for s in range(S):         # the entries (what is behind them in a page is nobody's)
        held = lengths[s, 0] + n[s]
        for i in (1 + 2 * s, 2 + 2 * s):
            a, b = (o[i].permute(0, 2, 1, 3).reshape(-1, Hkv, D)[:int(held)] for o in outs)
            assert torch.equal(a, b)
    assert torch.equal(outs[0][0], outs[1][0])


def test_packed_rows_far_apart():
    """Rows of 2^25 elements: 70 of them pass 2^32 bytes."""
    H, Hkv, D, n = 2, 1, 64, [3, 67]
    q, k, v = projected(gen(31), 1, H, Hkv, sum(n), D, BF16)
    off, scale = i32(offsets(n)), torch.full((1,), 0.2, device=DEV)
    want, want_lse = P.prefixkv_prefill_attn_packed(q, k, v, off, scale)
    room = torch.empty(sum(n) << 25, dtype=BF16, device=DEV).view(sum(n), 1 << 25)
    far = []
    for x, at in ((q, 0), (k, 1024), (v, 2048), (torch.empty_like(q), 4096)):
        y = room[:, at:at + x.shape[1] * D].view(sum(n), x.shape[1], D).permute(1, 0, 2)[None]
        y.copy_(x)
        far.append(y)
    _, lse = P.prefixkv_prefill_attn_packed(*far[:3], off, scale, out=far[3])
    assert torch.equal(far[3], want) and torch.equal(lse, want_lse)
    rq, rk = P.prefixkv_rope(q, k, torch.arange(sum(n), dtype=torch.int32, device=DEV)[None], P.rope_plan(D, device=DEV))
    P.prefixkv_rope(far[0], far[1], torch.arange(sum(n), dtype=torch.int32, device=DEV)[None], P.rope_plan(D, device=DEV),
                    q_out=far[0], k_out=far[1])
    assert torch.equal(far[0], rq) and torch.equal(far[1], rk)
