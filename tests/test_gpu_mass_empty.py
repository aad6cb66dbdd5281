"""Masses of a step in which no sequence has rows."""
import pytest
import torch

from paper_2609_36546_amd import ops
from tests.masked_reference import BF16, F32, Batch
from tests.test_gpu_mass_evict import c_mass, check_mass, masses


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("D,max_q", [(64, 1), (128, 500)])
def test_masses_decay_without_rows(dt, D, max_q):
    b = Batch([(0, 0), (5, 0), (700, 0), (33, 0)], 8, 2, D, 16, dt, seed=1)
    args = b.args[:3] + (max_q,)
    q, lse = torch.zeros(0, 8, D, dtype=dt, device="cuda"), torch.zeros(0, 8, device="cuda")
    m = masses(b)
    slopes = torch.ones(8, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    got = ops.attn_mass(q, b.kc, lse, *args, mass=m.cuda(), decay=0.5, slopes=slopes, first_key=none, validate=True)
    check_mass(b, got, lse, m, 0.5, {})
    some = torch.tensor([2], dtype=torch.int32, device="cuda")
    got = ops.attn_mass(q, b.kc, lse, *args, mass=m.cuda(), decay=0.25, seq_ids=some)
    check_mass(b, got, lse, m, 0.25, {}, seqs=[2])
    out = torch.full((b.kc.shape[0], 2, 16), 3.0, device="cuda")
    ops.attn_mass(q, b.kc, lse, *args, out=out, softcap=30.0)
    check_mass(b, out, lse, torch.full_like(m, 3.0), 0.0, {})


@pytest.mark.gpu
def test_null_arrays_outweigh_the_offsets():
    """Without q and lse there are no rows, whatever cu_q holds."""
    b = Batch([(40, 3), (100, 2)], 4, 2, 64, 16, BF16, seed=2)
    m = masses(b)
    mass = m.cuda()
    pt, ctx, cu, _ = b.args
    st = ops.lib().attn_mass(None, 256, b.kc.data_ptr(), None, pt.data_ptr(), pt.shape[1], ctx.data_ptr(), cu.data_ptr(), None, 2, 3,
                             0.0, 0, None, None, None, mass.data_ptr(), 0.5, mass.data_ptr(), 4, 2, 64, 16, b.kc.shape[0], 0.125, 1,
                             torch.cuda.current_stream().cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    b.k[:] = 0
    b.K = [k[:n] for k, n in zip(b.K, b.ctx)]
    b.cu[:] = 0
    check_mass(b, mass, torch.zeros(0, 4), m, 0.5, {})


# --- refusals (no GPU) ---

@pytest.mark.parametrize("kw", [dict(q=None), dict(lse=None), dict(q=None, lse=None, kc=None), dict(q=None, lse=None, mo=None),
                                dict(q=None, lse=None, cu=None), dict(q=None, lse=None, decay=-1.0), dict(q=None, lse=None, mq=0)])
def test_one_null_array_is_refused(kw):
    assert c_mass(**kw) == -1
