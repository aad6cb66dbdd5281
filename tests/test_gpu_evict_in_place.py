"""Eviction that writes the new lengths over the lengths or the bounds that it was given."""
import pytest
import torch

from paper_2609_36546_amd import ops
from tests.masked_reference import BF16, F32
from tests.test_gpu_mass_evict import check_evict, evicted, masses


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("over", ["ctx_lens", "keep"])
@pytest.mark.parametrize("Hkv,ctx,keep", [(8, [700, 0, 333, 1500, 64, 90, 5], [400, 3, -1, 700, 64, 1, 9]),
                                          (5, [20000, 300], [9000, 100])])
def test_new_lengths_over_the_arguments(dt, over, Hkv, ctx, keep):
    n = [max(0, min(a, c)) for a, c in zip(keep, ctx)]
    b, table, dst, dkeep = evicted(ctx, n, Hkv, 64, 16, dt, 1, keep)
    m = masses(b, 2)
    before = b.kc.cpu(), b.vc.cpu(), m.clone()
    mass, lens = m.cuda(), b.args[1].clone()
    place = lens if over == "ctx_lens" else dkeep
    new_lens, kept = ops.kv_evict(b.kc, b.vc, mass, b.args[0], dst, lens, dkeep, 2, 16, new_lens=place)
    assert new_lens is place and place.tolist() == n
    check_evict(b, table, before, keep, 2, 16, new_lens, kept, mass)


@pytest.mark.gpu
def test_lengths_of_other_sequences_stay():
    ctx, keep = [300, 200, 100, 50], [30, 20, 10, 0]
    b, table, dst, dkeep = evicted(ctx, keep, 4, 64, 16, BF16, 3, keep)
    m = masses(b, 1)
    before = b.kc.cpu(), b.vc.cpu(), m.clone()
    mass, lens = m.cuda(), b.args[1].clone()
    some = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    _, kept = ops.kv_evict(b.kc, b.vc, mass, b.args[0], dst, lens, dkeep, 0, 4, seq_ids=some, new_lens=lens)
    assert lens.tolist() == [30, 200, 100, 0]
    check_evict(b, table, before, keep, 0, 4, lens, kept, mass, seqs=[3, 0])
