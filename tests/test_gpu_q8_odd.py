"""Attention over the 8-bit cache where numbers are odd: rows that are NaN, in
either type; queries that are not finite; queries with one channel far above the
others."""
import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests import q8_reference as ref
from tests.test_gpu_q8 import BF16, F32, check_rows, f64, fill, pool, rows_of

pytestmark = pytest.mark.gpu


def from_scores(q, K, V, L, scale):
    """What the scores' rounding may do to the outputs.  rows_of's rows differ in size by e^3 and more, so that scores reach
    the hundreds: a sum of n products in fp32, whatever its order, is off by n 2^-24 of the products' sizes at most (three
    terms per query channel in fp32 calls, two in bf16 ones; the exponent's product and difference are two more), and
    weights p e^d with |d| <= b move sum p V / sum p by sum p (e^b - 1) |V - out| / sum p e^-b at most."""
    k, Hq, D = q.shape
    G, out = Hq // K.shape[1], np.zeros((k, Hq, D))
    for h in range(Hq):
        s, size = scale * (q[:, h] @ K[:, h // G].T), scale * (np.abs(q[:, h]) @ np.abs(K[:, h // G]).T)
        for i in range(k):
            n = L + i + 1
            w = np.exp(s[i, :n] - s[i, :n].max())
            w /= w.sum()
            b = (3 * D + 2) * 2.0 ** -24 * size[i, :n]
            V_h = V[:n, h // G]
            out[i, h] = (w * np.expm1(b)) @ np.abs(V_h - w @ V_h) / (w @ np.exp(-b))
    return out


def check_scored_rows(got, q, K, V, L, scale, dt):
    """check_rows, and what its tolerance has no part for."""
    want = ref.attention(q, K, V, L, scale)
    slack = from_scores(q, K, V, L, scale)
    off = np.sign(got - want) * np.maximum(np.abs(got - want) - slack, 0)
    check_rows(torch.from_numpy(want + off), want, dt)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("Hq,D", [(4, 64), (8, 128), (32, 64), (32, 128)])
@pytest.mark.parametrize("key", [False, True])
def test_nan_rows_reach_only_the_rows_that_see_them(dt, Hq, D, key):
    """A window token whose value (key) is not finite in one KV head, and slots
    behind the last that are NaN as before."""
    windows = [(70, 6), (20, 3)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, 2, D, 16)
    kv = fill(c, table, ctx, cu, pt, 9, dt)
    k, v = rows_of(windows, 2, D, dt, 3), rows_of(windows, 2, D, dt, 4)
    (k if key else v)[3, 1, 7] = float("inf") if key else float("nan")
    ops.kv_append_q8(k.cuda(), v.cuda(), c, pt, dctx, dcu, 6)
    q = torch.randn(9, Hq, D, generator=torch.Generator().manual_seed(2)).to(dt)
    out = f64(ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, 6))
    nan, half = np.isnan(out), Hq // 2
    assert nan[3:6, half:].all() and not nan[:3].any() and not nan[:6, :half].any() and not nan[6:].any()
    K, V = kv[0][0].copy(), kv[0][1].copy()
    K[70:76], V[70:76] = ref.quantise(f64(k[:6]))[0], ref.quantise(f64(v[:6]))[0]
    check_scored_rows(out[:3], f64(q[:3]), K[:73], V[:73], 70, D ** -0.5, dt)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("Hq,D", [(8, 64), (2, 128)])
@pytest.mark.parametrize("at", [5, 33, 59])
def test_nan_rows_inside_a_tile(dt, Hq, D, at):
    windows = [(70, 60), (20, 3)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, 2, D, 16)
    kv = fill(c, table, ctx, cu, pt, 9, dt)
    k, v = rows_of(windows, 2, D, dt, 3), rows_of(windows, 2, D, dt, 4)
    v[at, 1, 7] = float("nan")
    ops.kv_append_q8(k.cuda(), v.cuda(), c, pt, dctx, dcu, 60)
    q = torch.randn(63, Hq, D, generator=torch.Generator().manual_seed(2)).to(dt)
    out = f64(ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, 60))
    nan, half = np.isnan(out), Hq // 2
    assert nan[at:60, half:].all() and not nan[:at].any() and not nan[:60, :half].any() and not nan[60:].any()
    K, V = kv[0][0].copy(), kv[0][1].copy()
    K[70:130], V[70:130] = ref.quantise(f64(k[:60]))[0], ref.quantise(f64(v[:60]))[0]
    check_scored_rows(out[:at], f64(q[:at]), K[: 70 + at], V[: 70 + at], 70, D ** -0.5, dt)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("Hq,D,k", [(4, 64, 5), (8, 128, 5), (16, 128, 8), (32, 64, 16)])
def test_queries_that_are_not_finite(dt, Hq, D, k):
    """A NaN, an infinity of either sign: their rows and heads become NaN, the others keep every bit."""
    windows = [(200, k), (0, k), (3000, 1)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, 2, D, 16)
    fill(c, table, ctx, cu, pt, 9)
    q = torch.randn(int(cu[-1]), Hq, D, generator=torch.Generator().manual_seed(2)).to(dt).cuda()
    good = ops.verify_attn_q8(q, c, pt, dctx, dcu, k)
    assert torch.isfinite(good).all()
    odd = q.clone()
    hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    for row, h, d, x in ((1, 1, 5, float("nan")), (k - 1, Hq - 1, D - 1, float("inf")), (k + 2, 0, 0, -float("inf")),
                         (2 * k, 2, 40, float("nan"))):
        odd[row, h, d] = x
        hit[row, h] = True
    out = ops.verify_attn_q8(odd, c, pt, dctx, dcu, k)
    assert torch.isnan(out[hit]).all()
    assert torch.equal(out[~hit], good[~hit])


def two_terms(q):
    """What a bf16 call holds of a query row: two e4m3 numbers under the power of two that brings the largest to 224 .. 448,
    the second 2^-4 of the first.  float64 [..., D]."""
    _, e = ref.quantise(q)
    down = 2.0 ** (127.0 - e.astype(np.float64))[..., None]
    e4m3 = lambda x: torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()  # noqa: E731
    hi = e4m3(q * down)
    return (hi + e4m3((q * down - hi) * 16) / 16) / down


@pytest.mark.parametrize("Hq,D,k", [(4, 64, 5), (8, 128, 5), (32, 128, 16)])
@pytest.mark.parametrize("size", [300.0, 1e4, 1e5, 1e6])
def test_queries_with_one_large_channel(Hq, D, k, size):
    """One channel of every query is `size`, over keys that are nearly zero there, and the others decide.  They are held
    to 8 bits down to 2^-14 of the largest, and below to 2^-14 of a number of which the largest is at least 224: that is
    2^-21 of the largest at most."""
    windows = [(200, k), (0, k)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, 2, D, 16)
    n = (ctx + np.diff(cu)).astype(np.int32)
    g = torch.Generator().manual_seed(3)
    key, val = (torch.randn(int(n.sum()), 2, D, generator=g).to(BF16) for _ in range(2))
    key[..., 7] = 0.25 * key[..., 7] / size
    cu_all = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    ops.kv_append_q8(key.cuda(), val.cuda(), c, pt, torch.zeros(2, dtype=torch.int32).cuda(), torch.from_numpy(cu_all).cuda(),
                     int(n.max()))
    K, V = ref.quantise(f64(key))[0], ref.quantise(f64(val))[0]
    q = torch.randn(int(cu[-1]), Hq, D, generator=g).to(BF16)
    q[..., 7] = size
    held, x = two_terms(f64(q)), f64(q)
    top = np.abs(x).max(-1, keepdims=True)
    assert (np.abs(held - x) <= np.where(np.abs(x) >= 2.0 ** -14 * top, 2.0 ** -9 * np.abs(x), 2.0 ** -21 * top)).all()
    out = ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, k)
    for b in range(2):
        a = slice(cu_all[b], cu_all[b + 1])
        want = ref.attention(held[cu[b]: cu[b + 1]], K[a], V[a], int(ctx[b]), D ** -0.5)
        check_rows(out[cu[b]: cu[b + 1]], want, BF16)


@pytest.mark.parametrize("Hq,Hkv,D,ps,k", [(16, 8, 128, 16, 1), (8, 2, 64, 32, 4), (32, 2, 128, 16, 1), (3, 3, 64, 64, 5)])
def test_probabilities_of_few_rows_keep_16_bits(Hq, Hkv, D, ps, k):
    """bf16 calls of up to 16 rows per KV head: half a step of the result, half a step of 2^-16 of each probability (twice the
    half step of two terms of 8 bits; an error of at most 2^-16 of sum p |V|, taken as three times the row's rms), and the
    fp32 sums that check_rows has for fp32 calls."""
    windows = [(1500, k), (0, k), (63, k), (64, 1)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, Hkv, D, ps)
    kv = fill(c, table, ctx, cu, pt, 5)
    q = torch.randn(int(cu[-1]), Hq, D, generator=torch.Generator().manual_seed(6)).to(BF16)
    out = f64(ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, k))
    for b, (K, V) in enumerate(kv):
        want = ref.attention(f64(q[cu[b]: cu[b + 1]]), K, V, int(ctx[b]), D ** -0.5)
        rms = np.sqrt((want ** 2).mean(-1, keepdims=True))
        off = np.abs(out[cu[b]: cu[b + 1]] - want)
        tol = 2.0 ** -8 * np.abs(want) + (3 * 2.0 ** -16 + 2.0 ** -17) * rms
        print("worst", (off / tol).max(), flush=True)
        assert (off <= tol).all()


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("Hq,k", [(4, 2), (8, 12), (32, 40)])
def test_lengths_that_no_table_holds(dt, Hq, k):
    """Context lengths up to the largest 32-bit number: what comes out is not specified, but every index stays in its
    array, other sequences get what is theirs, and the walk ends with the table."""
    windows = [(40, k), (0, k), (33, k)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, 2, 64, 16)
    kv = fill(c, table, ctx, cu, pt, 5)
    own = table[1][table[1] >= 0]
    q = torch.randn(3 * k, Hq, 64, generator=torch.Generator().manual_seed(6)).to(dt)
    kn = torch.randn(3 * k, 2, 64, generator=torch.Generator().manual_seed(7)).to(dt).cuda()
    for L in (65, 4096, 2 ** 31 - 2 ** 28, 2 ** 31 - 200, 2 ** 31 - 100, 2 ** 31 - 65, 2 ** 31 - 11, 2 ** 31 - 1):
        bad = dctx.clone()
        bad[1] = L
        out = torch.full_like(q, 7.0, device="cuda")
        ops.verify_attn_q8(q.cuda(), c, pt, bad, dcu, k, out=out)
        for b in (0, 2):
            want = ref.attention(f64(q[cu[b]: cu[b + 1]]), *kv[b], int(ctx[b]), 0.125)
            check_rows(out[cu[b]: cu[b + 1]], want, dt)
        rk, _ = ops.kv_read_q8(c, pt, bad, dcu, k, 3 * k, dtype=F32)
        for b in (0, 2):
            assert np.array_equal(f64(rk[cu[b]: cu[b + 1]]), kv[b][0][ctx[b]:])
        # what the append may have changed lies in the sequence's own pages
        mine = torch.ones(c.num_pages, dtype=torch.bool)
        mine[torch.from_numpy(own).long()] = False
        mine[0] = False                                     # entries of -1 stand for it
        before = [t.view(torch.uint8).clone() for t in (c.k, c.v, c.scale)]
        only = torch.tensor([1], dtype=torch.int32).cuda()
        ops.kv_append_q8(kn, kn, c, pt, bad, dcu, k, seq_ids=only)
        for t, w in zip((c.k, c.v, c.scale), before):
            assert torch.equal(t.view(torch.uint8)[mine.cuda()], w[mine.cuda()])
            t.view(torch.uint8).copy_(w)
