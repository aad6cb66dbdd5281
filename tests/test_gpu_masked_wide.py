"""Masked attention under tables for millions of positions: units and workspace stay few."""
import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests.masked_reference import BF16, F32, Batch
from tests.test_gpu_masked import check, run

MOST = (1 << 31) - (1 << 28)          # positions of a table that are used


@pytest.mark.parametrize("slots", [1 << 20, 1 << 22, 1 << 25, 1 << 27, 1 << 29, MOST, 1 << 31])
@pytest.mark.parametrize("max_q", [1, 2, 8, 9, 200, 1 << 17])
@pytest.mark.parametrize("n_seq,Hq,Hkv", [(1, 8, 8), (1, 32, 4), (16, 16, 8)])
def test_every_table_has_a_workspace(slots, max_q, n_seq, Hq, Hkv):
    """2^20 packed rows in any case; what is asked for is no more than the pieces of the least
    length that the widest window may have."""
    size = ops.attn_masked_workspace_size(n_seq, Hq, Hkv, 64, max_q, slots // 64, 64)
    assert size > 0
    rows, blocks = max_q * Hq // Hkv, -(-min(slots, MOST) // 32)
    # pieces of a 16384th of the table at least, of 4 blocks or more: at most so many of a window of one
    # tile, and one more for each further tile (rows in tiles of 16, 32, 64 or 128)
    per = max(4, blocks // 16384)
    tile = 16 if rows <= 16 else 128
    pieces = -(-blocks // per) + -(-rows // 32) + 1
    assert size <= n_seq * Hkv * (pieces * tile * (64 * 4 + 8) + 4 * (-(-rows // 16) + 1)) + 256


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("slots", [1 << 26, 1 << 27, 1 << 29])
def test_windows_under_such_tables(dt, slots):
    b = Batch([(900, 2), (3000, 1)], 4, 2, 64, 64, dt, seed=3)
    pt, ctx, cu, _ = b.args
    wide = torch.full((2, slots // 64), -1, dtype=torch.int32, device="cuda")
    wide[:, : pt.shape[1]] = pt
    b.args = (wide, ctx, cu, 2)
    out, lse = run(b, softcap=30.0)
    check(b, out, lse, cap=30.0)
    assert np.isfinite(lse.cpu().numpy()).all()
