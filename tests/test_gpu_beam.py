"""Beam search over the paged cache: the choice of continuations and the places that follow them, against their plain forms in 64
bits and whole numbers.

Bars.  Whole numbers and moved rows: equality.  Choices between beams hang on sums of exponentials in 32 bits: with p the
probabilities of a row, the exponent of a term is off by three roundings of m - x, in all 3 * 2^-24 sum p (m - x), and that sum is at
most log V, below 14; the exponential by two steps, a sum by one for each of its up to 32 + 12 additions (a part of a thread's
terms, then trees): 90 * 2^-24 of the sum, and so of its logarithm.  The inputs' choices have to be further apart than twice that,
which is looked at, except for exact ties, whose rows have equal sums.  Scores: the same and a rounding to 32 bits."""
import numpy as np
import pytest
import torch

import beam_reference as R
import paper_2412_03409_amd as P
import serving_reference as RS
from test_gpu_serving import BF16, DEV, F32, f64, gen, i32, offsets, page_state

pytestmark = pytest.mark.gpu
LSE = 90 * 2.0 ** -24


def select_inputs(seed, S, W, V, dtype, end=None, spread=2.5):
    g = gen(seed)
    x = torch.randn((S, W, V), generator=g) * spread + torch.randn((S, 1, V), generator=g)
    x[torch.rand((S, W, V), generator=g) < 0.02] = float("-inf")
    x[torch.rand((S, W, V), generator=g) < 0.01] = float("nan")
    scores = torch.rand((S, W), generator=g) * -4.0 - 100.0
    ended = None
    if end is not None:
        ended = torch.rand((S, W), generator=g) < 0.25
    if W > 2:
        scores[torch.rand((S, W), generator=g) < 0.1] = float("-inf")
    return x.to(dtype), scores, ended


def check_select(x, scores, ended, end, got, ties=False):
    """x, scores and ended on the host, as the call got them."""
    want = R.select(x.double().numpy(), scores.double().numpy(), None if ended is None else ended.numpy(), end)
    assert ties or want[4] > 2 * LSE, "the inputs' choices are too close"
    for a, b in zip(got[:2], want[:2]):
        np.testing.assert_array_equal(a.cpu().numpy(), b)
    s = got[2].cpu().numpy().astype(np.float64)
    real = np.isfinite(want[2])
    np.testing.assert_array_equal(np.isneginf(s), np.isneginf(want[2]))
    assert (np.abs(s[real] - want[2][real]) <= LSE + 2.0 ** -24 * np.abs(want[2][real])).all()
    if end is None:
        assert got[3] is None
    else:
        np.testing.assert_array_equal(got[3].cpu().numpy(), want[3])


SELECT = [(1, 1, 1, F32), (1, 4, 2, BF16), (3, 5, 1003, BF16), (2, 4, 32000, BF16), (1, 32, 5000, F32), (4, 3, 70001, F32), (2, 32, 33, BF16),
          (1, 2, 1 << 20, BF16), (1, 1, (1 << 20) - 3, F32), (9, 16, 30011, F32), (16, 16, 17001, F32), (20, 16, 30011, F32),
          (40, 16, 30011, F32), (40, 32, 30011, BF16), (65, 2, 257, BF16)]


@pytest.mark.parametrize("S,W,V,dtype", SELECT)
@pytest.mark.parametrize("end", [None, 0])
def test_select(S, W, V, dtype, end):
    x, scores, ended = select_inputs(S + W + V, S, W, V, dtype, end)
    got = P.prefixkv_beam_select(x.to(DEV), scores.to(DEV), ended=None if ended is None else ended.to(DEV), end_token=end)
    check_select(x, scores, ended, end, got)


# pieces of 3, 5, 6 and 7 (bf16) and of 6, 10, 12 and 14 (fp32) times 16 bytes a thread, full to the last element or not
@pytest.mark.parametrize("S,W,V,dtype", [(105, 4, 5000, BF16), (16, 32, 9001, BF16), (70, 5, 12288, BF16), (38, 4, 28000, BF16), (95, 4, 5555, F32),
                                         (14, 32, 10001, F32), (44, 4, 24000, F32), (98, 3, 14336, F32)])
def test_select_pieces_that_divide_the_row(S, W, V, dtype):
    x, scores, ended = select_inputs(S + V, S, W, V, dtype, 3)
    got = P.prefixkv_beam_select(x.to(DEV), scores.to(DEV), ended=ended.to(DEV), end_token=3)
    check_select(x, scores, ended, 3, got)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_rows_that_begin_anywhere(dtype):
    """The last step of several, rows of odd length among others; outputs in the inputs' place."""
    S, W, V, end = 3, 4, 4099, 17
    x, scores, ended = select_inputs(5, S, W, V, dtype, end)
    want = P.prefixkv_beam_select(x.to(DEV), scores.to(DEV), ended=ended.to(DEV), end_token=end)
    for steps, before, behind in ((1, 1, 0), (3, 3, 2), (2, 5, 8)):
        room = torch.full((S, W, steps, before + V + behind), 1e30, dtype=dtype, device=DEV)
        y = room[:, :, -1, before:before + V]
        y.copy_(x)
        sc, en = scores.to(DEV), ended.to(DEV)
        got = P.prefixkv_beam_select(y, sc, ended=en, end_token=end, scores_out=sc, ended_out=en)
        assert got[2] is sc and got[3] is en
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("W,V", [(4, 50), (5, 3001), (32, 9001), (32, 40)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_ties_go_to_the_lowest(W, V, dtype):
    """Equal logits everywhere; a few values only; equal beams."""
    g = gen(V)
    flat = torch.zeros((1, W, V))
    few = torch.randint(0, 3, (1, 1, V), generator=g).float().expand(1, W, V).clone()
    few[0, :, 0] = -0.0
    for x in (flat, few):
        x = x.to(dtype)
        scores = torch.full((1, W), -3.0)
        check_select(x, scores, None, None, P.prefixkv_beam_select(x.to(DEV), scores.to(DEV)), ties=True)
    rising = torch.arange(V).float().expand(1, W, V).to(dtype)             # the best ones side by side at the end
    scores = torch.arange(W).float()[None] * -0.37
    check_select(rising, scores, None, None, P.prefixkv_beam_select(rising.to(DEV), scores.to(DEV)), ties=dtype == BF16)


def test_select_values_at_the_ends():
    """Rows without a token, with +inf, with the type's largest values; scores that are NaN or +inf; beams without candidates."""
    inf, V = float("inf"), 777
    x, scores, _ = select_inputs(3, 6, 4, V, F32)
    scores = scores.clamp(min=-200.0)
    x[0] = -inf                                                            # nothing at all
    x[1, 1:] = float("nan")
    x[2, 0, 5] = inf
    x[2, 1] = 3e38
    x[3, 0, 9] = -3e38
    scores[4] = torch.tensor([float("nan"), -inf, -5.0, inf])
    scores[5] = -inf
    got = P.prefixkv_beam_select(x.to(DEV), scores.to(DEV))
    check_select(x[[0, 1, 3, 5]], scores[[0, 1, 3, 5]], None, None, [t[[0, 1, 3, 5]] for t in got[:3]] + [None])
    # +inf is the largest finite number: all of its beam's weight, scores of the others 3e38 lower
    assert got[0][2, 0] == 5 and got[1][2, 0] == 0 or bool(scores[2, 0] < scores[2, 1:].max())
    assert got[1][4, 0] == 3 and not bool(torch.isnan(got[2]).any())


@pytest.mark.parametrize("V", [50, 4096, 5001])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_every_kind_of_nan_is_no_candidate(V, dtype):
    """Quiet and signalling, of both signs, in logits and scores."""
    x, _, _ = select_inputs(V, 1, 3, V, dtype)
    bits = x.view(torch.int16 if dtype == BF16 else torch.int32)
    quiet, sign = ((0x7fc0, 1 << 15) if dtype == BF16 else (0x7fc00000, 1 << 31))
    inf = 0x7f80 if dtype == BF16 else 0x7f800000
    for i, b in enumerate((inf + 1, quiet, inf + 1 - sign, quiet - sign, inf + 5)):
        bits[0, :, 3 + 7 * i] = b
    assert int(torch.isnan(x[0, 0]).sum()) >= 5
    scores = torch.tensor([[-3.0, -3.5, -4.0]])
    check_select(x, scores, None, None, P.prefixkv_beam_select(x.to(DEV), scores.to(DEV)))
    scores.view(torch.int32)[0, 1] = 0x7f800001
    check_select(x, scores, None, None, P.prefixkv_beam_select(x.to(DEV), scores.to(DEV)))


def test_select_is_repeatable_and_replays_from_a_graph():
    S, W, V, end = 5, 4, 20011, 3
    x, scores, ended = (t.to(DEV) for t in select_inputs(8, S, W, V, BF16, end))
    want = [t.clone() for t in P.prefixkv_beam_select(x, scores, ended=ended, end_token=end)]
    ws = torch.empty(P.beam_workspace_bytes(S, W, V, BF16), dtype=torch.uint8, device=DEV)
    outs = [torch.zeros_like(t) for t in want]
    kw = dict(ended=ended, end_token=end, tokens=outs[0], parents=outs[1], scores_out=outs[2], ended_out=outs[3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.prefixkv_beam_select(x, scores, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.prefixkv_beam_select(x, scores, ws=ws, **kw)
    for i in range(4):
        for t in outs:
            t.zero_()
        ws.fill_(255 * (i % 2))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        assert all(torch.equal(a, b) for a, b in zip(P.prefixkv_beam_select(x, scores, ended=ended, end_token=end), want))


def test_select_beams_that_have_all_ended_and_the_first_step():
    """Ended beams go on as they are, the best first; a beam among dead ones fills all places."""
    W, V, end = 6, 5000, 4999
    x, scores, _ = select_inputs(21, 2, W, V, F32)
    scores = torch.tensor([[-5.0, -1.0, -3.0, -1.0, -9.0, -2.0], [0.0] + [float("-inf")] * 5])
    ended = torch.tensor([[True] * W, [False] * W])
    got = P.prefixkv_beam_select(x.to(DEV), scores.to(DEV), ended=ended.to(DEV), end_token=end)
    assert got[0][0].tolist() == [end] * W and got[1][0].tolist() == [1, 3, 5, 2, 0, 4] and bool(got[3][0].all())
    assert got[2][0].tolist() == [-1.0, -1.0, -2.0, -3.0, -5.0, -9.0]
    assert got[1][1].tolist() == [0] * W
    check_select(x, scores, ended, end, got, ties=True)


@pytest.mark.parametrize("S,W,V", [(2, 32, 3000), (1, 32, 600), (3, 16, 1500)])
def test_select_one_beam_has_all_the_best(S, W, V):
    """Scores far apart: a single beam's list holds the W best, more than a wavefront's worth of candidates around them."""
    x, _, _ = select_inputs(S * V, S, W, V, BF16)
    for scores in (torch.arange(W).float().expand(S, W) * -50.0, torch.zeros((S, W)) - 7.0):
        x2 = x if scores[0, 1] < -40 else x[:, :1].expand(S, W, V).contiguous()      # equal beams: ties all over
        scores = scores.contiguous()
        check_select(x2, scores, None, None, P.prefixkv_beam_select(x2.to(DEV), scores.to(DEV)), ties=True)


# ---- places -------------------------------------------------------------------------------------------
def some_parents(r, G, W, empty=0.1):
    p = np.minimum((r.exponential(size=(G, W)) * W / 2.5).astype(np.int64), W - 1)
    p[r.random((G, W)) < empty] = -1
    return p


def as_cache(lens, table, ring, state, ps, Hkv, D, dtype, seed):
    g = gen(seed)
    kp, vp = (torch.randn((len(ring), Hkv, ps, D), generator=g).to(dtype).to(DEV) for _ in range(2))
    return P.PagedCache(kp=kp, vp=vp, table=i32(table), lens=i32(lens), ring=i32(ring), state=i32(state))


def check_cache(c, table, lens, ring, state, ps, pools=None):
    np.testing.assert_array_equal(c.lens.cpu().numpy(), lens)
    np.testing.assert_array_equal(c.state.cpu().numpy(), state)
    np.testing.assert_array_equal(c.ring.cpu().numpy(), ring)
    t = c.table.cpu().numpy()
    reached = np.arange(t.shape[2]) < -(-lens // ps)[..., None]
    np.testing.assert_array_equal(t[reached], table[reached])
    for a, b in zip((c.kp, c.vp), pools or ()):
        np.testing.assert_array_equal(f64(a), b)


REORDER = [(1, 1, 2, 16, 1, 64, BF16, 60), (1, 4, 3, 16, 2, 128, BF16, 100), (3, 5, 2, 32, 2, 64, F32, 90), (2, 32, 2, 16, 1, 64, BF16, 50),
           (5, 3, 4, 64, 3, 128, F32, 300), (2, 2, 1, 256, 8, 128, BF16, 700), (1, 2, 1, 16, 1, 64, BF16, 5000), (35, 2, 60, 16, 1, 64, BF16, 20),
           (1, 17, 2, 16, 1, 64, BF16, 700)]


@pytest.mark.parametrize("G,W,layers,ps,Hkv,D,dtype,ctx", REORDER)
@pytest.mark.parametrize("in_place", [True, False])
def test_reorder(G, W, layers, ps, Hkv, D, dtype, ctx, in_place):
    """Places that share nothing yet, of any lengths, become any of each other."""
    S = G * W
    lens, table, ring, state = page_state(S + ctx, S, layers, ps, -(-ctx // ps) + 2, S * layers, ctx)
    parents = some_parents(np.random.default_rng(W), G, W)
    c = as_cache(lens, table, ring, state, ps, Hkv, D, dtype, ctx)
    status, *want = R.reorder(parents, table, lens, ring, state, ps, [f64(c.kp), f64(c.vp)])
    assert status == 0
    if in_place:
        assert int(P.prefixkv_page_reorder(c, i32(parents))) == 0
        check_cache(c, *want[:4], ps, want[4])
        return
    kw = dict(table_out=torch.full_like(c.table, -7), lens_out=torch.empty_like(c.lens), state_out=torch.empty_like(c.state))
    for _ in range(2):                              # with outputs of its own a call can be made again
        assert int(P.prefixkv_page_reorder(c, i32(parents), **kw)) == 0
    assert torch.equal(c.table.cpu(), torch.from_numpy(table).int()) and torch.equal(c.lens.cpu(), torch.from_numpy(lens).int())
    got = P.PagedCache(kp=c.kp, vp=c.vp, table=kw["table_out"], lens=kw["lens_out"], ring=c.ring, state=kw["state_out"])
    check_cache(got, *want[:4], ps, want[4])
    beyond = np.arange(table.shape[2]) >= -(-want[1] // ps)[..., None]
    assert (kw["table_out"].cpu().numpy()[beyond] == -7).all()


@pytest.mark.parametrize("G,W,layers,ps,steps", [(2, 4, 3, 16, 40), (1, 5, 2, 16, 25), (3, 2, 1, 32, 30), (1, 32, 1, 16, 20)])
def test_a_search_of_many_steps(G, W, layers, ps, steps):
    """A prompt in the first place of every group, a fork, then tokens and reorderings in turn, an end: tables, lengths, ring and rows
    after every call, and every page is free again behind the last."""
    S, r = G * W, np.random.default_rng(W)
    width = -(-(60 + steps) // ps)
    n = np.zeros((S, layers), dtype=np.int64)
    n[::W] = r.integers(1, 60, size=(G, layers))
    total = int((-(-n // ps)).sum()) + S * layers * (2 + -(-steps // ps)) + 5
    c = P.paged_cache(S, layers, 1, 64, ps, total, width, BF16, DEV)
    c.kp.copy_(torch.randn(c.kp.shape, generator=gen(W)))
    c.vp.copy_(torch.randn(c.kp.shape, generator=gen(W + 1)))
    assert int(P.prefixkv_page_resize(c, i32(n))) == 0
    table, lens, ring, state = (x.cpu().numpy().astype(np.int64) for x in (c.table, c.lens, c.ring, c.state))
    pools = [f64(c.kp), f64(c.vp)]
    for step in range(steps):
        parents = np.zeros((G, W), dtype=np.int64) if step == 0 else some_parents(r, G, W, empty=0.03)
        status, table, lens, ring, state, pools = R.reorder(parents, table, lens, ring, state, ps, pools)
        assert status == 0 and int(P.prefixkv_page_reorder(c, i32(parents))) == 0
        check_cache(c, table, lens, ring, state, ps, pools)
        rows = (lens.max(axis=1) > 0).astype(np.int64)
        if step % 2 == 0 and rows.sum() > 0:                     # a token for every beam that there is
            off, T = offsets(rows), int(rows.sum())
            status, lens, table, state, slots = RS.append(lens, off, T, table, ring, state, ps)
            got, st = P.prefixkv_page_append(c, i32(off), T)
            assert status == 0 and int(st) == 0
            np.testing.assert_array_equal(got.cpu().numpy(), slots)
            assert len(np.unique(slots)) == slots.size           # no two beams write the same row
            for pool, ref in zip((c.kp, c.vp), pools):
                new = torch.randn(slots.shape + (64,), generator=gen(step)).to(BF16)
                flat = torch.from_numpy(slots)
                pool[(flat // ps).to(DEV), 0, (flat % ps).to(DEV)] = new.to(DEV)
                ref[slots // ps, 0, slots % ps] = new.double().numpy()
    status, table, lens, ring, state, pools = R.reorder(np.full((G, W), -1), table, lens, ring, state, ps, pools)
    assert int(P.prefixkv_page_reorder(c, i32(np.full((G, W), -1)))) == 0
    check_cache(c, table, lens, ring, state, ps, pools)
    assert int(c.state[1]) == total
    np.testing.assert_array_equal(np.sort(c.ring.cpu().numpy()), np.arange(total))


@pytest.mark.parametrize("what,status", [("parent", 2), ("below", 2), ("long", 2), ("negative", 2), ("head", 2), ("count", 2), ("room", 2),
                                         ("few", 1)])
@pytest.mark.parametrize("G,layers", [(3, 2), (50, 40)])
def test_reorderings_that_are_refused_on_the_device(what, status, G, layers):
    W, ps, width = 3, 16, 6
    S = G * W
    lens, table, ring, state = page_state(5, S, layers, ps, width, 200, 80)
    lens[0] = 33
    table[0, :, :3] = np.arange(3 * layers).reshape(layers, 3)
    parents = np.tile(np.arange(W), (G, 1))
    parents[0] = [0, 0, -1]
    if what == "parent":
        parents[G - 1, 1] = W
    elif what == "below":
        parents[1, 0] = -2
    elif what == "long":
        lens[S - 1, layers - 1] = width * ps + 1
    elif what == "negative":
        lens[4, 0] = -3
    elif what == "head":
        state[0] = -1
    elif what == "count":
        state[1] = len(ring) + 1
    elif what == "room":
        state[1] = len(ring)                                     # pages come back, and the ring is full
    else:
        state[1] = layers - 1
    c = as_cache(lens, table, ring, state, ps, 1, 64, BF16, 3)
    pools = [f64(c.kp), f64(c.vp)]
    assert R.reorder(parents, table, lens, ring, state, ps)[0] == status
    kw = dict(table_out=torch.full_like(c.table, -7), lens_out=torch.empty_like(c.lens), state_out=torch.empty_like(c.state))
    assert int(P.prefixkv_page_reorder(c, i32(parents), **kw)) == status
    assert int(P.prefixkv_page_reorder(c, i32(parents))) == status
    for x, y in ((c.table, table), (c.lens, lens), (c.ring, ring), (c.state, state), (kw["lens_out"], lens), (kw["state_out"], state)):
        np.testing.assert_array_equal(x.cpu().numpy(), y)
    held = np.arange(width) < np.clip(-(-lens // ps), 0, width)[..., None]
    np.testing.assert_array_equal(kw["table_out"].cpu().numpy(), np.where(held, table, -7))
    for x, y in zip((c.kp, c.vp), pools):
        np.testing.assert_array_equal(f64(x), y)


def test_reorder_leaves_pages_outside_the_pool_alone():
    """Ids that are no page, held or in the ring: nothing is copied from or to them, and none goes to the ring."""
    W, layers, ps = 4, 2, 16
    lens, held = np.full((W, layers), 40), W * layers * 3
    table = np.concatenate([np.arange(held).reshape(W, layers, 3), np.full((W, layers, 1), -1)], axis=2)
    ring, state = np.full(held + 9, -1), np.array([5, 9])
    ring[5:14] = held + np.arange(9)
    table[0, 0, 2], table[1, 0, 1], table[3, 1, 0] = -1, len(ring), 1 << 30
    ring[(state[0] + 1) % len(ring)] = -5
    parents = np.array([[0, 0, 2, 2]])
    c = as_cache(lens, table, ring, state, ps, 2, 64, BF16, 4)
    pools = [f64(c.kp), f64(c.vp)]
    assert int(P.prefixkv_page_reorder(c, i32(parents))) == 0
    np.testing.assert_array_equal(c.lens.cpu().numpy(), lens)
    now = c.ring.cpu().numpy()
    new = [now[(state[0] + state[1] + i) % len(ring)] for i in range(int(c.state[1]) - (state[1] - 4))]
    assert all(0 <= x < len(ring) for x in new)
    # taken, in (place, layer) order: one page each for place 1 and place 3; the one copied from page -1 stays as it was
    fresh = [ring[(state[0] + i) % len(ring)] for i in range(4)]
    got = c.table.cpu().numpy()
    assert [got[1, 0, 2], got[1, 1, 2], got[3, 0, 2], got[3, 1, 2]] == fresh
    for x, y in zip((c.kp, c.vp), pools):
        for dst, src in zip(fresh, (table[0, 0, 2], table[0, 1, 2], table[2, 0, 2], table[2, 1, 2])):
            if 0 <= dst < len(ring) and 0 <= src < len(ring):
                y[dst, :, :8] = y[src, :, :8]
        np.testing.assert_array_equal(f64(x), y)


def test_reorder_replays_from_a_graph():
    """A captured reordering in place, replayed: every replay goes on from the last one's places."""
    G, W, layers, ps = 2, 4, 3, 16
    lens, table, ring, state = page_state(9, G * W, layers, ps, 5, 60, 70)
    c = as_cache(lens, table, ring, state, ps, 2, 64, BF16, 5)
    pools = [f64(c.kp), f64(c.vp)]
    parents = i32(np.zeros((G, W)))
    status = torch.empty(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(P.reorder_workspace_bytes(G * W, layers), dtype=torch.uint8, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.prefixkv_page_reorder(c, parents, status=status, ws=ws)
    r = np.random.default_rng(1)
    for i in range(8):
        p = some_parents(r, G, W, empty=0.0)
        parents.copy_(i32(p))
        ws.fill_(255 * (i % 2))
        g.replay()
        torch.cuda.synchronize()
        want, table, lens, ring, state, pools = R.reorder(p, table, lens, ring, state, ps, pools)
        assert int(status) == want
        check_cache(c, table, lens, ring, state, ps, pools)


# ---- together -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,Hkv,D,ps,beams", [(4, 2, 64, 16, 3), (3, 3, 128, 32, 4)])
def test_beam_search_of_a_path(H, Hkv, D, ps, beams):
    """Prompts come into a path, their beams fork, extend, attend to the prompt's encoder's states, and are chosen and reordered for
    some steps; a prompt ends and another comes.  Every output against the definitions in 64 bits, on keys and values that are
    copied with their beam."""
    from paper_2412_03409_amd.pipeline import PagedPath
    from test_gpu_serving import close, projected
    L, G, V, end, g = 2, 2, 301, 4, gen(H)
    S = G * beams
    scale = torch.tensor([0.15, 0.3])
    plan = P.rope_plan(D, device=DEV)
    axis = plan.axis.cpu().numpy()
    path = PagedPath(S, L, H, Hkv, D, scale.to(DEV), plan, num_pages=260, max_pages=12, page_size=ps, device=DEV, beams=beams)
    keys = [[None] * L for _ in range(S)]
    m = [70, 131]
    to = offsets(m)
    kv = torch.randn((L, 2 * Hkv, sum(m), D), generator=g).to(BF16).to(DEV)
    states = kv[:, :Hkv], kv[:, Hkv:]

    def rows(T):
        x = projected(g, L, H, Hkv, T, D, BF16)
        pos = torch.randint(0, 3000, (1, T), generator=g).to(torch.int32).to(DEV)
        return (*x, pos)

    def rotated(x, pos):
        return torch.from_numpy(RS.rope(f64(x), pos.cpu().numpy(), axis, 10000.0, D, False)).to(BF16).double().numpy()

    def prompts(places, lengths, budgets):
        q, k, v, pos = rows(sum(lengths))
        kr, vr = rotated(k, pos), f64(v)
        kept = []
        path.prefill(places, lengths, q, k, v, pos, budgets, kept_pos=kept)
        assert int(path.status) == 0
        off = offsets(lengths)
        for i, s in enumerate(places):
            for b in range(beams):
                keys[s + b] = [[x[l][:, :0] for x in (kr, vr)] for l in range(L)]
            for l in range(L):
                at = kept[i][l].cpu().numpy()
                at = off[i] + at[at >= 0]
                keys[s][l] = [x[l][:, at] for x in (kr, vr)]

    def follow(parents):
        old = list(keys)
        for s in range(S):
            p = parents[s // beams, s % beams]
            keys[s] = [[x[:, :0] for x in seg] for seg in old[s]] if p < 0 else [list(seg) for seg in old[s // beams * beams + p]]
        lens = np.array([[seg[0].shape[1] for seg in k] for k in keys])
        np.testing.assert_array_equal(path.cache.lens.cpu().numpy(), lens)

    def extend():
        q, k, v, pos = rows(S)
        qr, kr, vr = rotated(q, pos), rotated(k, pos), f64(v)
        out = path.extend([1] * S, q, k, v, pos)
        assert int(path.status) == 0
        for s in range(S):
            for l in range(L):
                keys[s][l] = [np.concatenate([old, x[l][:, s:s + 1]], axis=1) for old, x in zip(keys[s][l], (kr, vr))]
                kk, vv = keys[s][l]
                for h in range(H):
                    o, mag, _ = RS.attend(qr[l, h, s:s + 1], kk[h // (H // Hkv)], vv[h // (H // Hkv)], float(scale[l]), kk.shape[1] - 1)
                    close(out[l:l + 1, h:h + 1, s:s + 1], o[None, None], mag[None, None], BF16)
        crossed = path.cross([1] * S, q, *states, i32(to))
        want, mag = R.cross(f64(q), offsets([beams] * G), f64(states[0]), f64(states[1]), to, scale.double().numpy())
        close(crossed, want, mag, BF16)

    def choose(scores, ended, step):
        x, _, _ = select_inputs(100 * H + step, G, beams, V, BF16)
        got = path.advance(x.to(DEV), scores, ended=ended, end_token=end)
        assert int(path.status) == 0
        check_select(x, scores.cpu(), None if ended is None else ended.cpu(), end, got)
        follow(got[1].cpu().numpy())
        return got[2], got[3]

    prompts([0, beams], [90, 41], [120, 60])
    path.follow(torch.zeros((G, beams), dtype=torch.int32, device=DEV))
    follow(np.zeros((G, beams), dtype=int))
    scores, ended = torch.full((G, beams), float("-inf"), device=DEV), None
    scores[:, 0] = 0
    for step in range(3):
        extend()
        scores, ended = choose(scores, ended, step)
    path.end(range(beams))
    follow(np.array([[-1] * beams, list(range(beams))]))
    prompts([0], [60], [70])
    first = np.array([[0] * beams, list(range(beams))])
    path.follow(i32(first))
    follow(first)
    scores[0], ended[0] = float("-inf"), False
    scores[0, 0] = 0
    for step in range(3, 3 + ps):
        extend()
        scores, ended = choose(scores, ended, step)
    path.end(range(S))
    assert int(path.cache.state[1]) == 260 and np.array_equal(np.sort(path.cache.ring.cpu().numpy()), np.arange(260))


def test_calls_on_two_streams_at_once():
    """Each with outputs and workspaces of its own: the same bits as one after the other."""
    S, W, V, layers, ps = 6, 4, 30011, 8, 16
    x, scores, _ = (t if t is None else t.to(DEV) for t in select_inputs(31, S, W, V, BF16))
    states = [page_state(40 + i, S * W, layers, ps, 8, 600, 100) for i in range(2)]
    parents = i32(some_parents(np.random.default_rng(3), S, W, empty=0.0))
    caches = [as_cache(*st, ps, 4, 128, BF16, 9 + i) for i, st in enumerate(states)]
    want = P.prefixkv_beam_select(x, scores)
    refs = []
    for st, c in zip(states, caches):
        refs.append(R.reorder(parents.cpu().numpy(), st[1], st[0], st[2], st[3], ps, [f64(c.kp), f64(c.vp)]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for stream, c in zip(streams, caches):
        with torch.cuda.stream(stream):
            for _ in range(3):
                got.append(P.prefixkv_beam_select(x, scores))
            assert P.prefixkv_page_reorder(c, parents) is not None
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g[:3], want[:3]))
    for (status, *ref), c in zip(refs, caches):
        assert status == 0
        check_cache(c, *ref[:4], ps, ref[4])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_reorder_pages_behind_the_first_four_gigabytes(dtype):
    """A fork in the last pages of a pool of more than 2^32 bytes: rows of every head are copied, nothing else is touched."""
    Hkv, D, ps, W, n = 4, 128, 256, 3, 700
    page = Hkv * ps * D * torch.finfo(dtype).bits // 8
    pages = (1 << 32) // page + 9
    c = P.paged_cache(W, 1, Hkv, D, ps, pages, 4, dtype, DEV)
    c.state.copy_(i32([pages - 8, 8]))                 # only the last eight pages are free
    assert int(P.prefixkv_page_resize(c, i32([[n], [0], [0]]))) == 0
    held = c.table[0, 0, :3].long()
    for x, seed in ((c.kp, 1), (c.vp, 2)):
        x[held] = torch.randn((3, Hkv, ps, D), generator=gen(seed)).to(dtype).to(DEV)
        x[pages - 5:] = 7.0
    assert int(P.prefixkv_page_reorder(c, i32([[0, 0, 0]]))) == 0
    t = c.table[:, 0, :3].cpu()
    assert bool((t[:, :2] == t[0, :2]).all()) and len(set(t[:, 2].tolist())) == 3 and int(t.min()) >= pages - 8
    for x in (c.kp, c.vp):
        for w in (1, 2):
            assert torch.equal(x[int(t[w, 2]), :, :n - 2 * ps], x[int(t[0, 2]), :, :n - 2 * ps])
            assert bool((x[int(t[w, 2]), :, n - 2 * ps:] == 7.0).all())
        assert bool((x[pages - 3:] == 7.0).all())
