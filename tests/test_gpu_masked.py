"""Attention with modified scores against 64-bit plain forms: types, heads, lengths,
masks that leave rows empty, what unseen slots hold; and its refusals."""
import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests import masked_reference as ref
from tests.masked_reference import BF16, F32, Batch, check_attention, f64, limits

RAGGED = [(0, 1), (5, 0), (15, 2), (16, 16), (700, 3), (100, 13), (31, 33)]


def run(b, **mod):
    return ops.verify_attn_masked(b.q.cuda(), b.k_new.cuda(), b.v_new.cuda(), b.kc, b.vc, *b.args, lse=True, **mod)


def check(b, out, lse, seqs=None, cap=0.0, window=0, slopes=None, first=None, end=None):
    rounded = b.dt == BF16 and b.max_q * b.Hq // b.Hkv > 16
    for i in range(len(b.ctx)) if seqs is None else seqs:
        L, k, r = int(b.ctx[i]), int(b.k[i]), b.rows(i)
        if k == 0:
            continue
        lo, hi = limits(L, k, window, None if first is None else first[r], None if end is None else end[r])
        want = ref.attention(f64(b.q[r]), b.K[i], b.V[i], L, b.scale, lo, hi, cap, slopes)
        check_attention(out[r], lse[r], want, b.dt, L + k, rounded)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("Hq,Hkv,D,ps", [(4, 2, 64, 16), (3, 1, 128, 32), (32, 4, 128, 16), (5, 5, 64, 64)])
@pytest.mark.parametrize("cap,sloped", [(0.0, False), (20.0, False), (0.0, True), (5.0, True)])
def test_scores(dt, Hq, Hkv, D, ps, cap, sloped):
    b = Batch(RAGGED, Hq, Hkv, D, ps, dt, seed=Hq, spread=1.5)
    slopes = 2.0 ** -np.arange(1.0, Hq + 1) if sloped else None
    out, lse = run(b, softcap=cap, slopes=None if slopes is None else torch.tensor(slopes, dtype=F32).cuda())
    check(b, out, lse, cap=cap, slopes=slopes)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("windows", [[(0, 1)], [(1, 1), (3000, 1)], [(1200, 8), (40, 1), (0, 8)], [(0, 90), (517, 300), (3, 1)]])
@pytest.mark.parametrize("window", [0, 1, 2, 33, 500])
def test_sliding_windows_and_lengths(dt, windows, window):
    b = Batch(windows, 8, 2, 64, 16, dt, seed=window)
    out, lse = run(b, window=window)
    check(b, out, lse, window=window)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("Hq,Hkv,D,ps", [(8, 2, 64, 16), (16, 2, 128, 32), (2, 2, 128, 16)])
@pytest.mark.parametrize("kind", ["documents", "prefix", "random", "window"])
def test_ranges(dt, Hq, Hkv, D, ps, kind):
    """Documents, prefixes and any ranges: empty ones, ones that end behind the window or
    before the row, negative beginnings."""
    windows = [(0, 130), (61, 40), (400, 1), (0, 1), (333, 17)]
    b = Batch(windows, Hq, Hkv, D, ps, dt, seed=7)
    rng = np.random.default_rng(3)
    p = np.concatenate([b.ctx[i] + np.arange(n) for i, n in enumerate(b.k)])
    n = np.repeat(b.ctx + b.k, b.k)
    first, end, window = None, None, 0
    if kind == "documents":
        first = p // 23 * 23
    elif kind == "prefix":
        end = np.maximum(p + 1, n // 2)
    elif kind == "random":
        first, end = rng.integers(-5, n + 3), rng.integers(-5, n + 40)
        end[::9] = first[::9]
    else:
        first, end, window = p // 90 * 90, np.maximum(p + 1, n // 3), 50
    dev = lambda x: None if x is None else torch.from_numpy(x.astype(np.int32)).cuda()  # noqa: E731
    out, lse = run(b, first_key=dev(first), end_key=dev(end), window=window, softcap=30.0)
    check(b, out, lse, first=first, end=end, window=window, cap=30.0)
    if kind == "random":
        assert (out == 0).flatten(1).all(1).any()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("Hq,D", [(8, 64), (16, 128), (2, 128)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_rows_that_do_not_see_a_value_do_not_get_it(dt, Hq, D, value):
    """A value that is not finite among the rows of one tile: rows before it, and of the
    document behind it, are as without it."""
    b = Batch([(70, 60), (20, 3)], Hq, 2, D, 16, dt, seed=2)
    at = 33
    b.v_new[at, 1, 7] = value
    first = np.where(np.arange(63) >= 48, np.concatenate([70 + np.arange(60), 20 + np.arange(3)]) // 4 * 4, 0)
    first[60:] = 0
    first[48:60] = 70 + 48
    out, lse = run(b, first_key=torch.from_numpy(first.astype(np.int32)).cuda())
    got = f64(out)
    sees = np.zeros(63, bool)
    sees[at:48] = True
    h = Hq // 2
    assert not np.isfinite(got[sees][:, h:, 7]).any()
    clean = got.copy()
    clean[:, h:][sees] = 0
    assert np.isfinite(clean).all()
    V = b.V[0].copy()
    V[70 + at, 1, 7] = 0
    lo, hi = limits(70, 60, first=first[:60])
    want = ref.attention(f64(b.q[:60]), b.K[0], V, 70, b.scale, lo, hi)
    keep = ~sees[:60]
    check_attention(out[:60][torch.from_numpy(keep)], None, [w[keep] for w in want], dt, 130, dt == BF16)
    assert torch.isfinite(lse).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_queries_and_keys_that_are_not_finite(dt):
    b = Batch([(40, 30)], 4, 2, 64, 16, dt, seed=4)
    b.q[3, 1, 5], b.k_new[20, 0, 2] = float("nan"), float("nan")
    out, _ = run(b, softcap=10.0)
    nan = np.isnan(f64(out)).any(-1)
    want = np.zeros((30, 4), bool)
    want[3, 1] = True
    want[20:, :2] = True
    assert np.array_equal(nan, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_large_scores_meet_the_cap(dt):
    """Scores far beyond the cap: probabilities of equal scores are equal."""
    b = Batch([(300, 2)], 2, 2, 64, 16, dt, seed=5)
    b.q = torch.full_like(b.q, 1e4)
    out, lse = run(b, softcap=1.0)
    K = b.K[0]
    want = ref.attention(f64(b.q), K, b.V[0], 300, b.scale, *limits(300, 2), cap=1.0)
    # tanh is +-1 but where a key's channels nearly cancel: the error of scores as in the plain check
    want = (want[0], want[1], want[2], np.full_like(want[3], 64 * 2.0 ** -24 * 4))
    x = b.scale * np.einsum("rhd,nhd->rhn", f64(b.q), K)
    if (np.abs(x) > 20).all():
        check_attention(out, lse, want, dt, 302, False)


@pytest.mark.gpu
def test_some_sequences_strided_queries_and_a_window_already_there():
    b = Batch(RAGGED, 4, 2, 64, 16, BF16, seed=9)
    some = torch.tensor([5, 2, 4], dtype=torch.int32).cuda()
    wide = torch.zeros(b.T, 8 * 64, dtype=BF16)
    wide[:, 128:384] = b.q.view(b.T, -1)
    q = wide.cuda()[:, 128:384].view(b.T, 4, 64)
    kc0, vc0 = b.kc.clone(), b.vc.clone()
    out, lse = torch.full((b.T, 4, 64), 7.0, dtype=BF16).cuda(), torch.full((b.T, 4), 7.0).cuda()
    ops.verify_attn_masked(q, b.k_new.cuda(), b.v_new.cuda(), b.kc, b.vc, *b.args, seq_ids=some, out=out, lse=lse)
    check(b, out, lse, seqs=[5, 2, 4])
    rest = [r for i in (0, 1, 3, 6) for r in range(b.cu[i], b.cu[i + 1])]
    assert (out[rest] == 7).all() and (lse[rest] == 7).all()
    # what the call wrote into the caches: the handled windows and nothing else
    kh, vh = b.kc.cpu(), b.vc.cpu()
    k0, v0 = kc0.cpu(), vc0.cpu()
    for i in (5, 2, 4):
        for p in range(b.ctx[i], b.ctx[i] + b.k[i]):
            page, slot = int(b.table[i, p // 16]), p % 16
            r = b.cu[i] + p - b.ctx[i]
            k0[page, :, :, slot, :], v0[page, :, :, slot] = b.k_new[r].view(2, 2, 32), b.v_new[r]
    bits = lambda t: t.view(torch.int16)  # noqa: E731
    assert torch.equal(bits(kh), bits(k0)) and torch.equal(bits(vh), bits(v0))
    again, lse2 = ops.verify_attn_masked(q, None, None, b.kc, b.vc, *b.args, seq_ids=some, lse=True)
    for i in (5, 2, 4):
        assert torch.equal(again[b.rows(i)], out[b.rows(i)]) and torch.equal(lse2[b.rows(i)], lse[b.rows(i)])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_without_modifiers_it_is_the_plain_attention(dt):
    """The same rows by verify_attn_paged: both within a rounding of the 64-bit form."""
    b = Batch([(400, 5), (0, 60), (33, 1)], 8, 2, 64, 32, dt, seed=1)
    kc, vc = torch.nan_to_num(b.kc), torch.nan_to_num(b.vc)
    out, lse = run(b)
    check(b, out, lse)
    plain = ops.verify_attn_paged(b.q.cuda(), b.k_new.cuda(), b.v_new.cuda(), kc, vc, *b.args)
    assert (plain.float() - out.float()).abs().max() < (0.05 if dt == BF16 else 1e-5)


@pytest.mark.gpu
def test_a_wide_table_and_a_loose_bound_of_windows():
    """Tables and max_q far above what the batch has give the same rows, to rounding."""
    b = Batch([(900, 2), (5, 9)], 8, 2, 128, 16, BF16, seed=3)
    pt, ctx, cu, _ = b.args
    wide = torch.full((2, 5000), -1, dtype=torch.int32).cuda()
    wide[:, : pt.shape[1]] = pt
    for max_q in (9, 200, 3000):
        b.args = (wide, ctx, cu, max_q)
        b.max_q = max_q
        check(b, *run(b, window=700), window=700)


@pytest.mark.gpu
def test_a_call_repeats_bit_for_bit_whatever_the_workspace_holds():
    b = Batch([(2000, 8), (700, 3)], 32, 4, 128, 16, BF16, seed=8)
    n = ops.attn_masked_workspace_size(2, 32, 4, 128, 8, b.table.shape[1], 16)
    outs = []
    for fill in (0, 255, 77):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        outs.append(run(b, softcap=50.0, workspace=ws))
    for o, l in outs[1:]:
        assert torch.equal(o, outs[0][0]) and torch.equal(l, outs[0][1])


@pytest.mark.gpu
def test_pages_behind_four_gigabytes():
    """Page offsets past 2^32 bytes."""
    Hkv, D, ps = 4, 128, 64
    P = (1 << 32) // (Hkv * D * ps * 2) + 40
    kc = torch.zeros(P, Hkv, D // 32, ps, 32, dtype=BF16, device="cuda")
    vc = torch.zeros(P, Hkv, D, ps, dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    L, k = 300, 9
    pages = torch.arange(P - 5, P, device="cuda", dtype=torch.int32)[None].flip(1).contiguous()
    for x in (kc, vc):
        x[P - 5:] = torch.randn(x[P - 5:].shape, generator=g, device="cuda").to(BF16)
    q = torch.randn(k, 32, D, generator=g, device="cuda").to(BF16)
    kn, vn = (torch.randn(k, Hkv, D, generator=g, device="cuda").to(BF16) for _ in range(2))
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    small = [kc[P - 5:].clone(), vc[P - 5:].clone()]
    want = ops.verify_attn_masked(q, kn, vn, *small, pages - (P - 5), dev([L]), dev([0, k]), k, softcap=30.0)
    got = ops.verify_attn_masked(q, kn, vn, kc, vc, pages, dev([L]), dev([0, k]), k, softcap=30.0)
    assert torch.equal(got, want)


@pytest.mark.gpu
def test_python_refusals():
    b = Batch([(5, 3)], 4, 2, 64, 16, BF16)
    good = dict(q=b.q.cuda(), k_new=b.k_new.cuda(), v_new=b.v_new.cuda(), k_cache=b.kc, v_cache=b.vc, page_table=b.args[0],
                ctx_lens=b.args[1], cu_q=b.args[2], max_q=3)
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    i = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.int32)  # noqa: E731
    for bad in (dict(slopes=f(3)), dict(slopes=i(4)), dict(first_key=i(2)), dict(first_key=f(3)), dict(end_key=i(4)),
                dict(lse=f(3, 3)), dict(out=f(3, 4, 64)), dict(k_cache=b.kc.float()), dict(v_cache=b.vc[:, :, :32].contiguous()),
                dict(page_table=i(2, 1)), dict(workspace=torch.zeros(1 << 20, dtype=torch.uint8)), dict(k_new=b.k_new),
                dict(k_new=b.k_new[:2].cuda()), dict(cu_q=i(3))):
        with pytest.raises(ValueError):
            ops.verify_attn_masked(**{**good, **bad})
    with pytest.raises(TypeError):
        ops.verify_attn_masked(**{**good, "v_new": None})
    for bad in (dict(softcap=-1.0), dict(softcap=float("nan")), dict(window=-2), dict(scale=0.0), dict(max_q=0)):
        with pytest.raises(ops.IpdvError):
            ops.verify_attn_masked(**{**good, **bad})
    with pytest.raises(ops.IpdvError, match="exceeds max_q"):
        ops.verify_attn_masked(**{**good, "max_q": 2}, validate=True)
    ops.verify_attn_masked(**good, validate=True)


# --- refusals (no GPU) ---

def c_attn(**kw):
    a = dict(cap=0.0, window=0, q=16, qs=256, kn=16, vn=16, kc=16, vc=16, pt=16, mp=4, ctx=16, cu=16, n=2, mq=3, out=16, lse=16, Hq=4, Hkv=2,
             D=64, ps=16, P=8, scale=0.125, dtype=1, ws=256, wsb=1 << 30)
    a.update(kw)
    return ops.lib().verify_attn_masked(
        a["q"], a["qs"], a["kn"], a["vn"], a["kc"], a["vc"], a["pt"], a["mp"], a["ctx"], a["cu"], None, a["n"], a["mq"],
        a["cap"], a["window"], None, None, None, a["out"], a["lse"], a["Hq"], a["Hkv"], a["D"], a["ps"], a["P"], a["scale"],
        a["dtype"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), -1), (dict(out=None), -1), (dict(kc=None), -1), (dict(vc=None), -1), (dict(kn=None), -1), (dict(vn=None), -1),
    (dict(Hq=5), -1), (dict(mq=0), -1), (dict(n=-1), -1), (dict(scale=0.0), -1), (dict(scale=float("inf")), -1),
    (dict(qs=255), -1), (dict(P=0), -1), (dict(mp=0), -1), (dict(D=96), -2), (dict(ps=128), -2), (dict(dtype=2), -2),
    (dict(q=8), -2), (dict(out=24), -2), (dict(kn=8, vn=16), -2), (dict(qs=260), -2), (dict(mq=1 << 28, Hq=2), -2),
    (dict(P=1 << 30), -2), (dict(n=40000), -2), (dict(ws=None), -3), (dict(wsb=4), -3), (dict(ws=264), -2),
    (dict(n=0, q=None), 0), (dict(cap=-1.0), -1), (dict(cap=float("inf")), -1),
    (dict(cap=float("nan")), -1), (dict(window=-1), -1)])
def test_attention_refusals(kw, status):
    assert c_attn(**kw) == status
    assert (ops.lib().ipdv_last_error() != b"") == (status != 0)


def test_workspace_query():
    size = ops.attn_masked_workspace_size
    assert size(64, 32, 4, 128, 8, 512, 16) > size(64, 32, 4, 128, 8, 512, 16, window=100) > 0
    assert size(64, 32, 4, 128, 8, 512, 16, window=100, has_end_key=True) == size(64, 32, 4, 128, 8, 512, 16)
    assert size(64, 32, 4, 96, 8, 512, 16) == 0 and size(64, 6, 4, 128, 8, 512, 16) == 0
    assert size(64, 32, 4, 128, 8, 512, 16, window=-1) == 0


def test_workspace_stays_small_for_long_prompts_and_wide_tables():
    size = ops.attn_masked_workspace_size
    assert size(8, 32, 4, 128, 1024, 64, 16) < 1 << 29
    assert size(16, 32, 4, 128, 512, 2048, 16) < 1 << 30
    assert size(1, 32, 4, 128, 1, 1 << 20, 16) < 1 << 29
