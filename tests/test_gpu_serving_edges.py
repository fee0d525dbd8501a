"""Packed prompts and paged caches where a serving program's state is unusual: sequences that wait beside others, a ring of free
pages whose ends cannot be, scores as large as the type holds, tiles that several workgroups share.  Every output against its
plain form in 64 bits, with the bars of test_gpu_serving.py."""
import numpy as np
import pytest
import torch

import paper_2412_03409_amd as P
import serving_reference as R
from test_gpu_serving import BF16, DEV, F32, as_cache, chunk_state, close, f64, gen, i32, offsets, page_state, projected
from tolerances import LSE_ATOL, LSE_RTOL

pytestmark = pytest.mark.gpu


# ---- sequences that wait -------------------------------------------------------------------------------
@pytest.mark.parametrize("H,Hkv,D,ps", [(8, 2, 128, 64), (3, 3, 64, 16)])
@pytest.mark.parametrize("rows", [1, 3, 70])
@pytest.mark.parametrize("waits", [[0], [1], [3], [0, 3], [0, 1, 2], [1, 2, 3], [0, 1, 2, 3]])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_chunk_attn_beside_sequences_that_wait(H, Hkv, D, ps, rows, waits, dtype):
    """Sequences without rows whose caches are long, at the front, in the middle and at the end, where the rows of the call end too:
    the others' results are theirs, and no row of nobody's is written."""
    L, S = 2, 4
    lens = np.array([[900, 40], [33, 1500], [1200, 64], [700, 2100]])
    n = [0 if s in waits else rows for s in range(S)]
    off = offsets(n)
    T = int(off[-1]) + (0 if sum(n) else 2)           # (a call has a row, if only one of nobody's)
    c, table = chunk_state(rows + H, S, L, Hkv, D, ps, lens, dtype)
    q, _, _ = projected(gen(H), L, H, Hkv, T, D, dtype)
    scale = torch.tensor([0.1, 0.2], device=DEV)
    out = torch.full((L, T, H, D), 55.0, dtype=dtype, device=DEV).permute(0, 2, 1, 3)
    P.prefixkv_chunk_attn(c, q, i32(off), scale, min(rows, T), out=out)
    want, mag = R.chunk(f64(q), off, f64(c.kp), f64(c.vp), table, lens, scale.double().cpu().numpy())
    close(out, want, mag, dtype)
    assert bool((out[torch.from_numpy(np.isnan(want)).to(DEV)] == 55).all())


# ---- the ring of free pages ----------------------------------------------------------------------------
@pytest.mark.parametrize("S,layers,width", [(3, 2, 8), (130, 40, 8), (40, 60, 16)])      # one launch; more segments, more places than one holds
@pytest.mark.parametrize("moved", [1, 3])
def test_pages_that_come_back_need_room_before_the_call(S, layers, width, moved):
    """A ring that is full although segments hold pages: what one segment gives back has no place, also when another takes as many."""
    ps = 16
    lens, table, ring, state = page_state(7, S, layers, ps, width, 20, 3 * ps)
    lens[0, 0], lens[1, 1] = 4 * ps, 0
    table[0, 0, :4], table[1, 1, :4] = [0, 1, 2, 3], -1
    ring[:] = np.arange(len(ring))
    state[:] = len(ring) - 1, len(ring)
    target = lens.copy()
    target[0, 0], target[1, 1] = (4 - moved) * ps, moved * ps
    c = as_cache(lens, table, ring, state, ps)
    assert int(P.prefixkv_page_resize(c, i32(target))) == 2
    for a, b in zip((c.lens, c.table, c.ring, c.state), (lens, table, ring, state)):
        np.testing.assert_array_equal(a.cpu().numpy(), b)
    # with room for them the same call is done, and the ring's ends come round
    state[:] = len(ring) - 1, len(ring) - moved
    c.state.copy_(i32(state))
    status, *want = R.resize(lens, target, table, ring, state, ps)
    assert status == 0 and int(P.prefixkv_page_resize(c, i32(target))) == 0
    for a, b in zip((c.lens, c.table, c.ring, c.state), want):
        np.testing.assert_array_equal(a.cpu().numpy(), b)


# ---- scores of any size ----------------------------------------------------------------------------------
# Queries have ones in two columns and zeros elsewhere, so a score is k[0] + k[1], exact in fp32; the 64-bit form gets the same.
SIZES = [("decode", [1, 1], [300, 90]), ("few", [4, 2], [2500, 90]), ("tiles", [70, 40], [400, 90]), ("cut", [100, 90], [6000, 90])]


def lowest_and_highest(dtype):
    top = torch.finfo(dtype).max
    return [("lowest", -top, 1.0), ("lowest, scaled", -top, 0.125), ("highest", top, 1.0), ("lowest, above one", -top, 40.0),
            ("highest, negative", top, -3.0), ("lowest, by nothing", -top, 0.0)]


def one_hot_state(seed, n, sizes, dtype, H=2, Hkv=1, D=64, ps=16):
    lens = np.array(sizes)[:, None]
    c, table = chunk_state(seed, len(n), 1, Hkv, D, ps, lens, dtype)
    off = offsets(n)
    q = torch.zeros((1, H, int(off[-1]), D), dtype=dtype, device=DEV)
    q[..., 0] = q[..., 1] = 1.0
    c.kp.zero_()
    return c, table, lens, off, q


def place(c, table, s, x, column, ps=16):
    """Column `column` of the keys of sequence s, entry by entry."""
    for j0 in range(0, len(x), ps):
        m = min(ps, len(x) - j0)
        c.kp[int(table[s, 0, j0 // ps]), :, :m, column] = x[j0:j0 + m].to(c.kp.dtype).to(DEV)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("what,n,sizes", SIZES)
@pytest.mark.parametrize("case", range(6))
def test_chunk_attn_where_every_score_is_the_lowest_or_the_highest(dtype, what, n, sizes, case):
    """Every visible key of a sequence has one score, the type's lowest or highest finite value: the mean of the values."""
    _, value, scale = lowest_and_highest(dtype)[case]
    c, table, lens, off, q = one_hot_state(21, n, sizes, dtype)
    place(c, table, 0, torch.full((sizes[0],), value), 0)
    place(c, table, 1, torch.randn(sizes[1], generator=gen(3)), 0)
    sc = torch.tensor([scale], device=DEV)
    out = P.prefixkv_chunk_attn(c, q, i32(off), sc, max(n))
    want, mag = R.chunk(f64(q), off, f64(c.kp), f64(c.vp), table, lens, sc.double().cpu().numpy())
    close(out, want, mag, dtype)
    assert bool((out[:, :, 0].float().abs() > 0).any())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("what,n,sizes", SIZES)
@pytest.mark.parametrize("big", [2.0 ** 11, 2.0 ** 16, -2.0 ** 16])
@pytest.mark.parametrize("scale", [1.0, -0.5])
def test_chunk_attn_scores_far_from_zero(dtype, what, n, sizes, big, scale):
    """Scores that differ by a little and are large, from some key on or throughout; lowest and ordinary ones among them."""
    c, table, lens, off, q = one_hot_state(22, n, sizes, dtype)
    g = gen(7)
    for s, length in enumerate(sizes):
        x = torch.full((length,), big)
        if s == 0:
            x[:length // 3] = 0                          # ordinary ones first: the maximum moves by a long way
        else:
            x[5:9] = torch.finfo(dtype).min if scale > 0 else torch.finfo(dtype).max
        place(c, table, s, x, 0)
        place(c, table, s, torch.randint(-12, 13, (length,), generator=g) / 4, 1)
    sc = torch.tensor([scale], device=DEV)
    out = P.prefixkv_chunk_attn(c, q, i32(off), sc, max(n))
    want, mag = R.chunk(f64(q), off, f64(c.kp), f64(c.vp), table, lens, sc.double().cpu().numpy())
    close(out, want, mag, dtype)


@pytest.mark.parametrize("n", [[3, 70], [300, 1], [2500, 40]])        # (the last one is cut)
@pytest.mark.parametrize("case", range(4))
def test_prefill_attn_packed_where_every_score_is_the_lowest_or_the_highest(n, case):
    """The mean of the values that a row sees, and a finite log-sum-exp where the scaled score is one."""
    _, value, scale = lowest_and_highest(BF16)[case]
    H, Hkv, D, off = 2, 1, 64, offsets(n)
    _, _, v = projected(gen(5), 1, H, Hkv, int(off[-1]), D, BF16)
    q = torch.zeros((1, H, int(off[-1]), D), dtype=BF16, device=DEV)
    q[..., 0] = 1.0
    k = torch.zeros((1, Hkv, int(off[-1]), D), dtype=BF16, device=DEV)
    k[..., 0] = value
    sc = torch.tensor([scale], device=DEV)
    out, lse = P.prefixkv_prefill_attn_packed(q, k, v, i32(off), sc)
    want, mag, wlse = R.prompt(f64(q), f64(k), f64(v), off, sc.double().cpu().numpy())
    close(out, want, mag, BF16)
    if abs(value * scale) <= torch.finfo(F32).max:
        assert np.all(np.abs(f64(lse) - wlse) <= 1e-4 * np.abs(wlse))


# ---- the path --------------------------------------------------------------------------------------------
def small_path(S=2, L=2, H=4, Hkv=2, D=64, num_pages=6, **kw):
    from paper_2412_03409_amd.pipeline import PagedPath
    path = PagedPath(S, L, H, Hkv, D, torch.tensor([0.2, 0.3], device=DEV)[:L], P.rope_plan(D, device=DEV), num_pages=num_pages,
                     max_pages=8, page_size=16, device=DEV, **kw)
    path.cache.kp.zero_(), path.cache.vp.zero_()
    return path


def path_state(path):
    c = path.cache
    return [x.clone() for x in (c.kp, c.vp, c.lens, c.table, c.ring, c.state)]


def path_rows(path, g, T):
    return (*projected(g, path.L, path.H, path.Hkv, T, path.D, BF16), torch.arange(T, dtype=torch.int32, device=DEV)[None])


def test_rows_without_pages_leave_the_path_as_it_was_and_answer_zeros():
    g, path = gen(13), small_path(num_pages=12)
    path.prefill([0, 1], [40, 9], *path_rows(path, g, 49), [60, 10])
    assert int(path.status) == 0
    before = path_state(path)
    out = path.extend([1, 70], *path_rows(path, g, 71))
    assert int(path.status) == 1 and not bool(out.any())
    for a, b in zip(path_state(path), before):
        assert torch.equal(a, b)
    out = path.extend([1, 2], *path_rows(path, g, 3))          # what has room goes on
    assert int(path.status) == 0 and bool(out.any())
    assert torch.equal(path.cache.lens - before[2], i32([[1, 1], [2, 2]]))


def test_a_prompt_that_the_search_cannot_rank_is_told():
    """NaN in a query of one prompt of three: no entries for it, the search's verdict at its place, the others as they are."""
    g, path = gen(14), small_path(S=4, num_pages=40)
    q, k, v, pos = path_rows(path, g, 90)
    q[1, 2, 45, 3] = float("nan")
    path.prefill([3, 0, 2], [30, 30, 30], q, k, v, pos, [20, 20, 20])
    assert int(path.status) == 0
    assert path.search.tolist() == [1, 0, 0, 0] and path.cache.lens.sum(1).tolist() == [0, 0, 20, 20]
    path.prefill([0], [30], *path_rows(path, g, 30), [20])
    assert path.search.tolist() == [0, 0, 0, 0] and path.cache.lens.sum(1).tolist() == [20, 0, 20, 20]


def test_sequences_that_any_iterable_names_end():
    g, path = gen(15), small_path(S=3, num_pages=30)
    path.prefill([0, 1, 2], [20, 20, 20], *path_rows(path, g, 60), [10, 10, 10])
    path.end(s for s in (0, 2))
    assert path.cache.lens.sum(1).tolist() == [0, 10, 0]
    path.end(np.array([1, 1]))
    assert int(path.cache.lens.sum()) == 0 and int(path.cache.state[1]) == 30
    path.end([])
    assert int(path.status) == 0


# ---- single tokens keep their probabilities ----------------------------------------------------------------
@pytest.mark.parametrize("H,Hkv,D,ps,n,sizes", [(16, 2, 128, 16, [1, 1, 1], [5, 64, 2100]), (6, 3, 64, 32, [4, 16, 2], [40, 16, 900]),
                                                (4, 4, 128, 64, [32, 1], [33, 300]), (32, 1, 128, 16, [1] * 40, [3] * 39 + [700])])
def test_chunk_attn_of_few_rows_rounds_its_output_only(H, Hkv, D, ps, n, sizes):
    """Decode steps weigh bf16 values with more than bf16 probabilities, as prefixkv_decode_attn does.  A probability is the sum of two
    bf16 numbers, the second below 2^-7 of it and rounded by 2^-9 of itself: 2^-16 of sum p|v|, next to the logits' 2e-4."""
    lens = np.array(sizes)[:, None]
    c, table = chunk_state(23, len(n), 1, Hkv, D, ps, lens, BF16)
    off = offsets(n)
    q, _, _ = projected(gen(24), 1, H, Hkv, int(off[-1]), D, BF16)
    scale = torch.tensor([0.1], device=DEV)
    out = P.prefixkv_chunk_attn(c, q, i32(off), scale, max(n))
    want, mag = R.chunk(f64(q), off, f64(c.kp), f64(c.vp), table, lens, scale.double().cpu().numpy())
    bar = 2.0 ** -8 * np.abs(want) + (2.0 ** -16 + 2e-4) * mag
    assert np.all(np.abs(f64(out) - want) <= bar), float(np.max(np.abs(f64(out) - want) / bar))


def test_chunk_attn_of_few_rows_infinite_values_stay_infinite():
    """Values that every row sees: an infinite one makes its column infinite (NaN with one of either sign), and no other column."""
    H, Hkv, D, ps, n, sizes = 4, 2, 64, 16, [1, 3], [300, 2100]
    lens = np.array(sizes)[:, None]
    c, table = chunk_state(25, 2, 1, Hkv, D, ps, lens, BF16)
    off = offsets(n)
    q, _, _ = projected(gen(26), 1, H, Hkv, int(off[-1]), D, BF16)
    q *= 0.05                          # (weights far from underflow)
    for s, j, column, value in ((0, 7, 3, float("inf")), (0, 250, 9, float("-inf")), (1, 40, 3, float("inf")), (1, 1999, 3, float("-inf")),
                                (1, 900, 20, float("inf")), (1, 31, 21, torch.finfo(BF16).max)):
        c.vp[int(table[s, 0, j // ps]), :, j % ps, column] = value
    out = P.prefixkv_chunk_attn(c, q, i32(off), torch.tensor([0.1], device=DEV), max(n))[0].float()
    inf = torch.isinf(out) | torch.isnan(out)
    want = torch.zeros_like(inf)
    want[:, :1, [3, 9]] = True
    want[:, 1:, [3, 20]] = True
    assert torch.equal(inf, want)
    assert bool((out[:, 0, 3] == float("inf")).all()) and bool((out[:, 0, 9] == float("-inf")).all())
    assert bool(torch.isnan(out[:, 1:, 3]).all()) and bool((out[:, 1:, 20] == float("inf")).all())


# ---- tiles that several workgroups share -------------------------------------------------------------------
@pytest.mark.parametrize("L,H,Hkv,n,first", [(2, 4, 2, [2500, 1, 200], 0), (1, 8, 8, [2047], 3)])
@pytest.mark.parametrize("sign", [1, -1])
def test_cut_prompts(L, H, Hkv, n, first, sign):
    """Head dimension 128, several layers: outputs and log-sum-exps that the join writes."""
    D, off = 128, offsets(n, first)
    T = int(off[-1]) + 1
    assert P.attn_workspace_bytes(len(n), L, H, Hkv, T, D, BF16) > 0          # (only a launch that cuts tiles has one)
    q, k, v = projected(gen(27), L, H, Hkv, T, D, BF16)
    scale = torch.tensor([0.08, 0.13][:L]) * sign
    out, lse = torch.full_like(q, 77.0), torch.full((L * H * T,), 77.0, device=DEV)
    P.prefixkv_prefill_attn_packed(q, k, v, i32(off), scale.to(DEV), out=out, lse=lse)
    want, mag, wlse = R.prompt(f64(q), f64(k), f64(v), off, scale.double().numpy())
    close(out, want, mag, BF16)
    assert bool((out[torch.from_numpy(np.isnan(want)).to(DEV)] == 77).all())
    real, z = ~np.isnan(wlse), f64(lse)
    assert np.all(z[~real] == 77)
    assert np.all(np.abs(z - wlse)[real] <= LSE_RTOL * np.abs(wlse[real]) + LSE_ATOL)


@pytest.mark.parametrize("H,Hkv,D,ps", [(8, 2, 128, 64), (2, 1, 64, 16)])
def test_cut_chunks_with_pages_outside_the_pool(H, Hkv, D, ps):
    """Entries on pages that are not there take no part, in whichever workgroup's share they lie, and whole stages of them."""
    L, n = 2, [100, 2, 64]
    lens = np.array([[5000, 4000], [70, 300], [640, 3500]])
    c, table = chunk_state(28, 3, L, Hkv, D, ps, lens, BF16)
    for s, l, entry in ((0, 0, 200), (0, 0, 2600), (0, 0, 4999), (0, 1, 0), (1, 1, 299), (2, 0, 64), (2, 1, 3400)):
        table[s, l, entry // ps] = (-1, c.kp.shape[0], 1 << 30)[entry % 3]
    table[0, 1, 640 // ps:1280 // ps] = -5
    c.table.copy_(i32(table))
    off = offsets(n)
    q, _, _ = projected(gen(29), L, H, Hkv, int(off[-1]), D, BF16)
    scale = torch.tensor([0.1, -0.15], device=DEV)
    out = P.prefixkv_chunk_attn(c, q, i32(off), scale, max(n))
    want, mag = R.chunk(f64(q), off, f64(c.kp), f64(c.vp), table, lens, scale.double().cpu().numpy())
    close(out, want, mag, BF16)
