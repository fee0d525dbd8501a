"""Workspace sizes of numbers that 32 bits do not hold: refused, where ctypes would take them modulo 2^32 and answer for others."""
import pytest
import torch

import paper_2412_03409_amd as P

WRAP = 1 << 32
BF16 = torch.bfloat16


@pytest.mark.parametrize("f,good", [
    (P.reorder_workspace_bytes, (8, 2)), (P.page_workspace_bytes, (8, 2)),
    (lambda *a: P.cross_workspace_bytes(*a, BF16, 10), (2, 1, 4, 2, 10, 9000, 128)),
    (lambda *a: P.attn_workspace_bytes(*a, BF16, 4), (2, 1, 4, 2, 10, 128)),
    (lambda *a: P.beam_workspace_bytes(*a, BF16), (2, 4, 1000))])
def test_numbers_that_32_bits_do_not_hold(f, good):
    assert f(*good) > 0
    for i, x in enumerate(good):
        for bad in (WRAP + x, x - WRAP):
            with pytest.raises(ValueError, match="32 bits"):
                f(*good[:i], bad, *good[i + 1:])
