"""Attention of packed rows whose offsets cannot be: both storage types agree on whose rows there are."""
import numpy as np
import pytest
import torch

import beam_reference as R
import paper_2412_03409_amd as P
from test_gpu_cross import inputs
from test_gpu_serving import BF16, DEV, F32, close, f64, gen, i32, projected

pytestmark = pytest.mark.gpu
T, M = 10, 40
# offsets of rows and states -> rows that are some sequence's, with their states (None: it has none: zeros)
CASES = [
    ([0, 5, 11], [0, 20, 40], {(0, 5): (0, 20)}),               # the second ends behind the last row: it has none
    ([0, 11, 11], [0, 20, 40], {}),
    ([-1, 5, 10], [0, 20, 40], {(5, 10): (20, 40)}),
    ([0, 4, 2, 10], [0, 20, 20, 40], {(0, 2): (0, 20), (4, 10): (20, 40)}),     # (rows 2 and 3 are two sequences': either's answer)
    ([7, 3, 3, 9], [0, 10, 20, 40], {(3, 9): (20, 40)}),
    ([0, 12, 4, 10], [0, 10, 20, 40], {(4, 10): (20, 40)}),
    ([0, 5, 10], [0, 41, 41], {(0, 5): None, (5, 10): None}),
    ([0, 5, 10], [30, 10, 40], {(0, 5): None, (5, 10): (10, 40)}),
    ([0, 5, 10], [-5, 10, 40], {(0, 5): None, (5, 10): (10, 40)}),
]


def rest_is_left(out, off, whose):
    untouched = set(range(T)) - {t for a, b in whose for t in range(a, b)} - ({2, 3} if off == [0, 4, 2, 10] else set())
    assert all(bool((out[:, :, t] == 9).all()) for t in untouched)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("off,to,whose", CASES)
@pytest.mark.parametrize("most", [2, 10])
def test_cross_attn(off, to, whose, dtype, most):
    q, k, v, _, _, scale = inputs(13, 1, 8, 2, [T], [M], 64, dtype)
    out = torch.full_like(q, 9.0)
    P.prefixkv_cross_attn(q, k, v, i32(off), i32(to), scale, most, out=out)
    named = {}
    for (a, b), xy in whose.items():
        # the first `most` rows of the sequence that has them
        first = max(o for o in off[:-1] if o <= a) if off != [0, 4, 2, 10] or a == 0 else 2
        stop = min(b, first + most)
        if stop <= a:
            continue
        named[(a, stop)] = xy
        if xy is None:
            assert bool((out[:, :, a:stop] == 0).all())
            continue
        want, mag = R.cross(f64(q), [a, stop], f64(k), f64(v), list(xy), scale.double().cpu().numpy())
        close(out[:, :, a:stop], want[:, :, a:stop], mag[:, :, a:stop], dtype)
    rest_is_left(out, off, named)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("off,whose", [([0, 5, 11], [(0, 5)]), ([0, 11, 11], []), ([-1, 5, 10], [(5, 10)]), ([7, 3, 3, 9], [(3, 9)]),
                                       ([0, 12, 4, 10], [(4, 10)])])
def test_chunk_attn(off, whose, dtype):
    """Over a paged cache: rows of a sequence that cannot be are left, the others are what they are with offsets that can."""
    S, ps = len(off) - 1, 16
    cache = P.paged_cache(S, 1, 2, 64, ps, 4 * S, 3, dtype, DEV)
    assert int(P.prefixkv_page_resize(cache, i32([[30 + s] for s in range(S)]))) == 0
    for pool, seed in ((cache.kp, 1), (cache.vp, 2)):
        pool.copy_(torch.randn(pool.shape, generator=gen(seed)).to(dtype))
    q, _, _ = projected(gen(3), 1, 4, 2, T, 64, dtype)
    scale = torch.full((1,), 0.2, device=DEV)
    out, ok = torch.full_like(q, 9.0), torch.full_like(q, 9.0)
    P.prefixkv_chunk_attn(cache, q, i32(off), scale, T, out=out)
    good = [whose[0][0]] * S + [whose[0][1]] if whose else [0] * (S + 1)
    if whose:
        s = [i for i in range(S) if (off[i], off[i + 1]) == whose[0]][0]
        good = [whose[0][0]] * (s + 1) + [whose[0][1]] * (S - s)
    P.prefixkv_chunk_attn(cache, q, i32(good), scale, T, out=ok)
    assert torch.equal(out, ok)
    rest_is_left(out, off, whose)


def test_states_that_many_sequences_name():
    """Offsets that go to and fro name all states 512 times, 2^31 blocks of them: more than are counted.  Nothing is written, and the
    next call, with the same workspace, is as ever."""
    S, heads, most = 1024, 32, 1 << 22
    q, _, _ = projected(gen(4), 1, heads, heads, S, 64, BF16)
    states = torch.zeros((1, 1, most, 64), dtype=BF16, device=DEV)
    states[:, :, :S] = torch.randn((S, 64), generator=gen(5)).to(BF16).to(DEV)
    k = v = states.expand(1, heads, most, 64)
    scale, off = torch.full((1,), 0.2, device=DEV), i32(np.arange(S + 1))
    ws = torch.zeros(P.cross_workspace_bytes(S, 1, heads, heads, S, most, 64, BF16, 1), dtype=torch.uint8, device=DEV)
    assert ws.numel() > 0                                       # units long enough for blocks that are shared out
    ws.fill_(127)
    out = torch.full_like(q, 9.0)
    P.prefixkv_cross_attn(q, k, v, off, i32([most * (i % 2) for i in range(S + 1)]), scale, 1, out=out, ws=ws)
    torch.cuda.synchronize()
    assert bool((out == 9).all())
    P.prefixkv_cross_attn(q, k, v, off, off, scale, 1, out=out, ws=ws)
    assert torch.equal(out, v[:, :, :S])                        # one state each
