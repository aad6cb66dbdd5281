"""rope_window against a 64-bit plain form, and its refusals."""
import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests import q8_reference as ref

BF16, F32 = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().float().cpu().double().numpy()


def bound(want, x, dt, factor):
    """One rounding of the result, and fp32 arithmetic before it: sine and
    cosine off by 4 steps of 2^-24, two products and a sum by one each, all
    relative to the pair's size (at most the row's largest entry twice)."""
    size = factor * 2 * np.abs(x).max(-1, keepdims=True)
    return torch.finfo(dt).eps / 2 * np.abs(want) + 8 * 2.0 ** -24 * size


def batch(windows, dt, Hq, Hkv, D, seed=0, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    ctx = np.array([w[0] for w in windows], np.int32)
    cu = np.concatenate([[0], np.cumsum([w[1] for w in windows])]).astype(np.int32)
    T = int(cu[-1])
    q = torch.randn(T, Hq, D, generator=g).to(dt).to(device)
    k = torch.randn(T, Hkv, D, generator=g).to(dt).to(device)
    pos = np.concatenate([c + np.arange(n) for c, n in windows])
    return q, k, torch.from_numpy(ctx).to(device), torch.from_numpy(cu).to(device), pos


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("layout", [ops.ROPE_HALF, ops.ROPE_INTERLEAVED])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (64, 64), (64, 20), (128, 104), (128, 2), (40, 34), (65, 64)])
def test_rope_matches_the_plain_form(dt, layout, D, rot):
    windows = [(0, 1), (7, 0), (1, 5), (100000, 3), (2 ** 30, 2), (0, 9)]
    q, k, ctx, cu, pos = batch(windows, dt, 6, 2, D)
    f, _ = ops.rope_inv_freq(rot, 1e6)
    for inverse in (False, True):
        a, b = ops.rope_window(q, k, f.cuda(), ctx, cu, 9, layout=layout, factor=1.25, inverse=inverse)
        for x, y in ((q, a), (k, b)):
            want = ref.rope(f64(x), pos, f.numpy(), layout, 1.25, inverse)
            assert (np.abs(f64(y) - want) <= bound(want, f64(x), dt, 1.25)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("shift", [0, 1])
def test_rope_of_strided_rows_in_place_and_unaligned(dt, shift):
    """q and k are slices of one projection; with `shift` no row starts on 16 bytes."""
    Hq, Hkv, D, T = 4, 2, 64, 7
    wide = torch.randn(T, (Hq + 2 * Hkv) * D + shift, generator=torch.Generator().manual_seed(3)).to(dt).cuda()
    q = wide[:, shift: shift + Hq * D].view(T, Hq, D)
    k = wide[:, shift + Hq * D: shift + (Hq + Hkv) * D].view(T, Hkv, D)
    before = wide.clone()
    ctx = torch.tensor([5, 900], dtype=torch.int32).cuda()
    cu = torch.tensor([0, 4, 7], dtype=torch.int32).cuda()
    f = ops.rope_inv_freq(D)[0].cuda()
    a, b = ops.rope_window(q, k, f, ctx, cu, 4)
    pos = [5, 6, 7, 8, 900, 901, 902]
    for x, y in ((q, a), (k, b)):
        want = ref.rope(f64(x), pos, f.cpu().numpy(), 0)
        assert (np.abs(f64(y) - want) <= bound(want, f64(x), dt, 1.0)).all()
    ops.rope_window(q, k, f, ctx, cu, 4, q_out=q, k_out=k)
    assert torch.equal(q, a) and torch.equal(k, b)
    rest = wide[:, shift + (Hq + Hkv) * D:]
    assert torch.equal(rest, before[:, shift + (Hq + Hkv) * D:]) and torch.equal(wide[:, :shift], before[:, :shift])


@pytest.mark.gpu
def test_rope_leaves_other_sequences_and_rows_behind_the_last():
    windows = [(3, 2), (50, 4), (9, 1)]
    q, k, ctx, cu, pos = batch(windows, F32, 2, 1, 64)
    q = torch.cat([q, q[:2]])
    k = torch.cat([k, k[:2]])
    f = ops.rope_inv_freq(64)[0].cuda()
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    ops.rope_window(q, k, f, ctx, cu, 4, seq_ids=torch.tensor([2, 0], dtype=torch.int32).cuda(), q_out=qo, k_out=ko)
    assert (qo[2:6] == 7).all() and (qo[7:] == 7).all() and (ko[2:6] == 7).all()
    want = ref.rope(f64(q[:7]), pos, f.cpu().numpy(), 0)
    live = [0, 1, 6]
    assert (np.abs(f64(qo)[live] - want[live]) <= bound(want, f64(q[:7]), F32, 1.0)[live]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [ops.ROPE_HALF, ops.ROPE_INTERLEAVED])
def test_rope_gradient(layout):
    """The inverse is the transposed map: <g, R x> = <R' g, x>, and the loss's
    differences (linear in x, so they hold for any step)."""
    q, k, ctx, cu, _ = batch([(11, 3), (4000, 6)], F32, 3, 2, 64, seed=1)
    gq, gk, _, _, _ = batch([(11, 3), (4000, 6)], F32, 3, 2, 64, seed=2)
    f = ops.rope_inv_freq(48, 1e4)[0].cuda()
    call = lambda a, b, inv: ops.rope_window(a, b, f, ctx, cu, 6, layout=layout, factor=1.5, inverse=inv)  # noqa: E731
    dq, dk = call(gq, gk, True)
    loss = lambda a, b: (f64(gq) * f64(a)).sum() + (f64(gk) * f64(b)).sum()  # noqa: E731
    y = loss(*call(q, k, False))
    assert abs(y - ((f64(dq) * f64(q)).sum() + (f64(dk) * f64(k)).sum())) < 1e-4
    for at in [(0, 0, 0), (2, 1, 40), (8, 2, 63), (5, 0, 13)]:
        q2 = q.clone()
        q2[at] += 2.0
        assert abs((loss(*call(q2, k, False)) - y) / 2.0 - f64(dq)[at]) < 1e-5


def test_frequencies():
    p = np.arange(32)
    plain = 1e6 ** (-2.0 * p / 64)
    near = lambda a, b: np.allclose(a, b, rtol=2.0 ** -23, atol=0)  # noqa: E731
    f, s = ops.rope_inv_freq(64, 1e6)
    assert near(f.numpy(), plain) and s == 1.0
    f, _ = ops.rope_inv_freq(64, 1e6, ops.ROPE_LINEAR, 4.0)
    assert near(f.numpy(), plain / 4)
    f, _ = ops.rope_inv_freq(64, 1e6, ops.ROPE_NTK, 4.0)
    assert near(f.numpy()[[0, 31]], [1.0, plain[31] / 4])
    f, s = ops.rope_inv_freq(64, 1e6, ops.ROPE_YARN, 4.0, 4096)
    turns = 4096 * plain / (2 * np.pi)
    r = f.numpy() / plain
    assert near(r[turns > 40], 1.0) and near(r[turns < 0.8], 0.25) and (np.diff(r) <= 1e-6).all()
    assert abs(s - (0.1 * np.log(4.0) + 1)) < 1e-6


@pytest.mark.parametrize("kw", [dict(rot=3), dict(rot=0), dict(base=1.0), dict(factor=0.5), dict(kind=4), dict(kind=-1),
                                dict(kind=ops.ROPE_YARN), dict(kind=ops.ROPE_YARN, original_len=100, beta_slow=40.0),
                                dict(rot=2, kind=ops.ROPE_NTK), dict(base=float("inf")), dict(factor=float("nan"))])
def test_frequency_refusals(kw):
    with pytest.raises(ops.IpdvError) as e:
        ops.rope_inv_freq(**{"rot": 64, **kw})
    assert e.value.status == -1


def c_rope(**kw):
    a = dict(q=16, qs=256, k=16, ks=128, qo=32, qos=256, ko=32, kos=128, f=16, ctx=16, cu=16, n=2, mq=3, Hq=4, Hkv=2, D=64,
             rot=64, layout=0, factor=1.0, dtype=1)
    a.update(kw)
    return ops.lib().rope_window(a["q"], a["qs"], a["k"], a["ks"], a["qo"], a["qos"], a["ko"], a["kos"], a["f"], a["ctx"],
                                 a["cu"], None, a["n"], a["mq"], a["Hq"], a["Hkv"], a["D"], a["rot"], a["layout"], a["factor"],
                                 0, a["dtype"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), -1), (dict(ko=None), -1), (dict(f=None), -1), (dict(n=-1), -1), (dict(mq=0), -1), (dict(Hq=0), -1),
    (dict(rot=66), -1), (dict(rot=33), -1), (dict(rot=0), -1), (dict(layout=2), -1), (dict(factor=float("nan")), -1),
    (dict(dtype=2), -2), (dict(dtype=0x11), -2), (dict(D=513, qs=1 << 20, ks=1 << 20, qos=1 << 20, kos=1 << 20), -2),
    (dict(qs=255), -1), (dict(kos=127), -1), (dict(n=65536), -2), (dict(qo=16, qos=512), -1), (dict(n=0, q=None), 0)])
def test_rope_refusals(kw, status):
    assert c_rope(**kw) == status
    assert (ops.lib().ipdv_last_error() != b"") == (status != 0)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", [ops.ROPE_HALF, ops.ROPE_INTERLEAVED])
def test_rope_of_the_farthest_positions(layout):
    """Odd positions whose product with a 24-bit frequency has more than 53 bits: the
    plain form rounds it the same; the library's step to turns adds a constant's and
    a product's rounding, 2^-53 of the angle each."""
    windows = [(2 ** 29 + 12345, 3), (2 ** 30 + 1, 2), (2 ** 31 - 17, 9), (2 ** 24 + 3, 1)]
    q, k, ctx, cu, pos = batch(windows, F32, 3, 2, 64)
    f, _ = ops.rope_inv_freq(64, 1e4)
    f[3] = 0.70710677
    a, b = ops.rope_window(q, k, f.cuda(), ctx, cu, 9, layout=layout)
    angle = 2.0 ** -52 * pos[:, None, None] * float(f.max())
    for x, y in ((q, a), (k, b)):
        want = ref.rope(f64(x), pos, f.numpy(), layout)
        size = 2 * np.abs(f64(x)).max(-1, keepdims=True)
        assert (np.abs(f64(y) - want) <= bound(want, f64(x), F32, 1.0) + angle * size).all()
