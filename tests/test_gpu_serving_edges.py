"""Packed prompts and paged caches at the places where a serving program's state is unusual: sequences that wait beside others.
Every output against its plain form in 64 bits, with the bars of test_gpu_serving.py."""
import numpy as np
import pytest
import torch

import paper_2412_03409_amd as P
import serving_reference as R
from test_gpu_serving import BF16, DEV, F32, chunk_state, close, f64, gen, i32, offsets, projected

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
