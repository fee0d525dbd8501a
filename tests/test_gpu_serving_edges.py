"""Packed prompts and paged caches where a serving program's state is unusual: sequences that wait beside others, a ring of free
pages whose ends cannot be.  Every output against its plain form in 64 bits, with the bars of test_gpu_serving.py."""
import numpy as np
import pytest
import torch

import paper_2412_03409_amd as P
import serving_reference as R
from test_gpu_serving import BF16, DEV, F32, as_cache, chunk_state, close, f64, gen, i32, offsets, page_state, projected

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
