"""The verdict on drafts by probabilities against a 64-bit plain form: whole windows, both
kinds of drafts, filters, temperatures, rows that cannot be drawn from; its refusals."""
import math

import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests import masked_reference as ref
from tests import q8_reference as filters
from tests.masked_reference import BF16, F32, f64

NAMES = ("temperature", "top_k", "top_p", "min_p")


def rows(seed, T, V, dt, agree=0.6):
    g = torch.Generator().manual_seed(seed)
    t = 4 * torch.randn(T, V, generator=g)
    d = t + agree * torch.randn(T, V, generator=g)
    return t.to(dt), d.to(dt), g


def probs(l, f, m):
    """A row's probabilities; None where a cut lies too close to a border to be sure of."""
    l = f64(l)[m]
    T, k, p, mn = (None if f.get(n) is None else f[n][m].item() for n in NAMES)
    T = 1.0 if T is None else T
    ends = {filters.kept_prefix(l, T, k, p, mn, d)[1] for d in (-1e-6, 0.0, 1e-6)}
    order, n, _ = filters.kept_prefix(l, T, k, p, mn)
    return ref.softmax_kept(l, order[:n], T) if len(ends) == 1 else None


def check(target, draft, tf, df, x, cu, u, ud, got, eos=-1):
    """Every sequence whose decisions are farther than 1e-8 from a border; returns how many."""
    sure = 0
    for b in range(len(cu) - 1):
        r = range(int(cu[b]), int(cu[b + 1]))
        P = [probs(target, tf, m) for m in r]
        Q = None if draft is None else [probs(draft, df, m) if x[m] >= 0 else np.zeros(target.shape[1]) for m in r]
        if any(p is None for p in P) or (Q and any(q is None for q in Q)):
            continue
        sl = slice(int(cu[b]), int(cu[b + 1]))
        n, token, fin, ratio, logp, margin = ref.verdict(np.array(P), None if Q is None else np.array(Q), x[sl], u[sl], ud[b], eos)
        # a ratio: 1e-9 and its rounding to fp32
        assert np.allclose(f64(got["p_accept"][sl]), ratio, rtol=2.0 ** -24 + 2e-9, atol=1e-30)
        if margin < 1e-8:
            continue
        sure += 1
        assert (int(got["n_acc"][b]), int(got["token"][b]), int(got["finished"][b])) == (n, token, fin)
        if token >= 0:
            assert abs(float(got["logp"][b]) - logp) <= 2.0 ** -23 * abs(logp) + 1e-8
        else:
            assert math.isnan(float(got["logp"][b]))
    return sure


def call(target, draft, x, cu, u, ud, tf={}, df={}, eos=-1, **kw):
    c = lambda t, d: torch.as_tensor(np.asarray(t), dtype=d).cuda()  # noqa: E731
    f = {n: t.cuda() for n, t in tf.items()}
    f.update({"draft_" + n: t.cuda() for n, t in df.items()})
    return ops.verify_drafts(target.cuda(), None if draft is None else draft.cuda(), c(x, torch.int32), c(cu, torch.int32),
                             c(u, F32), c(ud, F32), eos_id=eos, **f, **kw)


def drafts(draft, f, g):
    """Tokens drawn from the draft's distribution."""
    out = []
    for m in range(draft.shape[0]):
        p = probs(draft, f, m)
        p = p if p is not None else ref.softmax_kept(f64(draft)[m], np.arange(draft.shape[1]), 1.0)
        out.append(int(np.searchsorted(np.cumsum(p), torch.rand(1, generator=g).item() * p.sum(), side="right")))
    return np.minimum(out, draft.shape[1] - 1)


RAGGED = [0, 1, 1, 6, 9, 26, 30]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("V", [1, 2, 57, 1000, 8192, 8193, 20000])
@pytest.mark.parametrize("kind", ["sampled", "certain"])
def test_windows(dt, V, kind):
    T = RAGGED[-1]
    t, d, g = rows(V, T, V, dt)
    x = drafts(d, {}, g)
    for b in (0, 3, 5):
        x[RAGGED[b + 1] - 1] = -1                    # a row behind the drafts
    u, ud = torch.rand(T, generator=g).numpy(), torch.rand(len(RAGGED) - 1, generator=g).numpy()
    d = d if kind == "sampled" else None
    got = call(t, d, x, RAGGED, u, ud)
    assert check(t, d, {}, {}, x, RAGGED, u, ud, got) >= len(RAGGED) - 3


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("which", ["temperature", "top_k", "top_p", "min_p", "all", "target only"])
def test_filters(dt, which):
    T, V, cu = 40, 5003, list(range(0, 41, 4))
    t, d, g = rows(3, T, V, dt)
    rng = np.random.default_rng(5)
    every = {"temperature": torch.tensor(rng.choice([0.0, 0.5, 1.0, 1.7], T), dtype=F32),
             "top_k": torch.tensor(rng.choice([0, 1, 5, 100], T), dtype=torch.int32),
             "top_p": torch.tensor(rng.choice([0.3, 0.9, 1.0], T), dtype=F32),
             "min_p": torch.tensor(rng.choice([0.0, 0.05, 0.5], T), dtype=F32)}
    tf = {which: every[which]} if which in every else every
    df = {} if which == "target only" else tf
    x = drafts(d, df, g)
    x[3::8] = -1
    u, ud = torch.rand(T, generator=g).numpy(), torch.rand(10, generator=g).numpy()
    got = call(t, d, x, cu, u, ud, tf, df)
    assert check(t, d, tf, df, x, cu, u, ud, got) >= 8


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_certain_drafts_and_filters(dt):
    T, V, cu = 24, 3001, [0, 6, 12, 18, 24]
    t, _, g = rows(8, T, V, dt)
    x = f64(t).argmax(1)
    x[5::6] = -1
    tf = {"top_k": torch.full((T,), 3, dtype=torch.int32), "temperature": torch.full((T,), 0.6)}
    u, ud = torch.rand(T, generator=g).numpy(), torch.rand(4, generator=g).numpy()
    check(t, None, tf, {}, x, cu, u, ud, call(t, None, x, cu, u, ud, tf))
    # a draft that the filter cuts is rejected whatever u is
    x[:] = f64(t).argmin(1)
    got = call(t, None, x, cu, 0 * u, ud, tf)
    assert (got["n_acc"] == 0).all() and (got["p_accept"] == 0).all()
    check(t, None, tf, {}, x, cu, 0 * u, ud, got)


@pytest.mark.gpu
def test_temperature_zero_takes_the_first_maximum():
    t = torch.zeros(4, 20000)
    t[0, [9000, 12345]] = 3.0
    t[1, 7] = 1.0
    t[2, 19999] = 2.0
    zero = {"temperature": torch.zeros(4)}
    for dt in (BF16, F32):
        got = call(t.to(dt), None, [9000, 7, 19999, -1], [0, 4], [0.99] * 4, [0.7], zero)
        assert int(got["n_acc"]) == 3 and int(got["token"]) == 0 and float(got["logp"]) == 0
        got = call(t.to(dt), None, [12345, 7, 19999, -1], [0, 4], [0.0] * 4, [0.7], zero)
        assert int(got["n_acc"]) == 0 and int(got["token"]) == 9000 and got["p_accept"].tolist() == [0, 1, 1, 0]
        both = call(t.to(dt), t.flip(0).to(dt), [9000, 7, 19999, -1], [0, 4], [0.99] * 4, [0.7], zero, zero)
        assert both["p_accept"].tolist() == [1, 1, 1, 0]          # q(x) = 0, p(x) = 1


@pytest.mark.gpu
def test_eos_ends_the_window():
    V = 100
    t = torch.full((5, V), -1e4)
    for r, v in enumerate([5, 9, 9, 5, 9]):
        t[r, v] = 0
    got = call(t, None, [5, 9, 9, 5, -1], [0, 3, 5], [0.5] * 5, [0.5, 0.5], eos=9)
    assert got["n_acc"].tolist() == [2, 1] and got["token"].tolist() == [-1, 9] and got["finished"].tolist() == [1, 1]
    got = call(t, None, [5, 9, 9, 5, -1], [0, 3, 5], [0.5] * 5, [0.5, 0.5])
    assert got["n_acc"].tolist() == [3, 1] and got["token"].tolist() == [-1, 9] and got["finished"].tolist() == [0, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("filtered", [False, True])
def test_rows_that_cannot_be_drawn_from(dt, filtered):
    """NaN, +inf, nothing finite, bad temperatures: the window ends, the others do not notice."""
    T, V = 14, 9001
    t, d, g = rows(1, T, V, dt)
    x = drafts(d, {}, g)
    x[13] = -1
    t[1, 17], t[3, 8999], t[5], d[7, 4] = float("nan"), float("inf"), -float("inf"), float("nan")
    temp = torch.ones(T)
    temp[9], temp[11] = -1.0, float("nan")
    tf = {"temperature": temp}
    if filtered:
        tf["top_k"] = torch.full((T,), 4000, dtype=torch.int32)
    cu = list(range(0, 15, 2))
    u, ud = np.zeros(T), torch.rand(7, generator=g).numpy()
    got = call(t, d, x, cu, u, ud, tf)
    n = got["n_acc"].tolist()
    assert n[:6] == [1] * 6 and got["token"].tolist()[:6] == [-1] * 6 and not got["finished"].any()
    bad = [1, 3, 5, 7, 9, 11]
    nan = np.isnan(f64(got["p_accept"]))
    assert nan[bad].all() and nan.sum() == len(bad)
    assert n[6] == 1 and int(got["token"][6]) >= 0                # the row without a draft, of a bad draft row or not
    d[13] = float("nan")
    again = call(t, d, x, cu, u, ud, tf)
    assert int(again["token"][6]) == int(got["token"][6])


@pytest.mark.gpu
def test_entries_of_no_mass_and_far_temperatures():
    V = 300
    t = torch.full((4, V), -float("inf"))
    t[:, 40], t[:, 41] = 1.0, 1.0
    d = t.clone()
    temp = {"temperature": torch.tensor([1.0, 1e-38, 3e38, float("inf")])}
    for r in range(4):
        for ud, want in ((0.0, 40), (0.4999, 40), (0.5001, 41), (0.99999, 41)):
            f = {"temperature": temp["temperature"][r: r + 1]}
            got = call(t[r: r + 1], None, [-1], [0, 1], [0.0], [ud], f)
            assert int(got["token"]) == want and abs(float(got["logp"]) + math.log(2)) < 1e-6
    # equal distributions: every draft is accepted, whatever u
    got = call(t, d, [40, 41, 40, 41], [0, 4], [1 - 2.0 ** -24] * 4, [0.5], temp, temp)
    assert int(got["n_acc"]) == 4 and (got["p_accept"] == 1).all() and int(got["token"]) == -1
    # drafts that have no mass in either, or lie outside the vocabulary
    got = call(t, d, [3, 299, 300, 2 ** 31 - 1], [0, 1, 2, 3, 4], [0.0] * 4, [0.2] * 4)
    assert (got["n_acc"] == 0).all() and (got["p_accept"] == 0).all() and got["token"].tolist() == [40] * 4


@pytest.mark.gpu
@pytest.mark.parametrize("V,at", [(20000, 17000), (9000, 8999), (40000, 2100)])
def test_whole_stretches_of_no_mass_are_not_drawn_from(V, at):
    t = torch.full((3, V), -float("inf"))
    t[:, at] = 2.0
    t[:, at - 1] = 1.0
    d = t.clone()
    d[:, at - 1] = 3.0
    for draft, df in ((None, {}), (d, {}), (d, {"top_k": torch.full((3,), 2, dtype=torch.int32)})):
        got = call(t, draft, [at - 1, -1, 0], [0, 1, 2, 3], [0.999] * 3, [0.0] * 3, {}, df)
        assert got["n_acc"].tolist() == [0, 0, 0]
        assert got["token"].tolist() == [at, at - 1, at - 1 if draft is None else at]


@pytest.mark.gpu
def test_emitted_tokens_follow_the_target():
    """Many windows of one draft over a small vocabulary: the first token emitted is
    distributed as the target (each frequency within five standard deviations)."""
    n, V = 20000, 6
    g = torch.Generator().manual_seed(0)
    t, d = torch.tensor([0.3, -1.0, 1.2, 0.0, 2.0, -3.0]), torch.tensor([1.5, 0.2, -0.5, 0.0, 1.0, 0.3])
    q, p = torch.softmax(d.double(), 0), torch.softmax(t.double(), 0).numpy()
    x = torch.multinomial(q, n, replacement=True, generator=g)
    u, ud = torch.rand(n, generator=g), torch.rand(n, generator=g)
    got = call(t.repeat(n, 1), d.repeat(n, 1), x, np.arange(n + 1), u, ud)
    out = torch.where(got["n_acc"].cpu() == 1, x, got["token"].cpu().long()).numpy()
    share = np.bincount(out, minlength=V) / n
    assert (np.abs(share - p) < 5 * np.sqrt(p * (1 - p) / n)).all()


@pytest.mark.gpu
def test_strides_and_unaligned_rows():
    T, V, cu = 12, 8200, [0, 4, 8, 12]
    t, d, g = rows(6, T, V, BF16)
    x = drafts(d, {}, g)
    u, ud = torch.rand(T, generator=g), torch.rand(3, generator=g)
    want = call(t, d, x, cu, u, ud)
    for pad, off in ((8, 0), (3, 0), (16, 1), (16, 8)):
        wide = torch.full((2, T, V + pad + off), float("nan"), dtype=BF16, device="cuda")
        wide[0, :, off: off + V], wide[1, :, off: off + V] = t.cuda(), d.cuda()
        got = call(wide[0][:, off: off + V], wide[1][:, off: off + V], x, cu, u, ud)
        assert all(torch.equal(got[n], want[n]) for n in ("n_acc", "token", "finished"))
        assert torch.allclose(got["p_accept"], want["p_accept"], rtol=1e-9, atol=0)


@pytest.mark.gpu
def test_many_rows_in_one_window_and_a_full_vocabulary():
    T, V = 600, 262144
    t = torch.zeros(1, V, dtype=BF16, device="cuda").expand(T, V).contiguous()
    t[:, 77] = 60.0                                       # everything at 77
    x = torch.full((T,), 77, dtype=torch.int32)
    x[599] = -1
    got = ops.verify_drafts(t, t, x.cuda(), torch.tensor([0, T], dtype=torch.int32).cuda(), torch.full((T,), 0.999).cuda(),
                            torch.tensor([0.3]).cuda())
    assert int(got["n_acc"]) == 599 and int(got["token"]) == 77
    x[400] = 262143
    got = ops.verify_drafts(t, t, x.cuda(), torch.tensor([0, T], dtype=torch.int32).cuda(), torch.full((T,), 1.0).cuda(),
                            torch.tensor([0.3]).cuda())
    assert int(got["n_acc"]) in (0, 400)                  # u of 1: equal probabilities are not passed
    assert int(got["n_acc"]) == 0


@pytest.mark.gpu
def test_rows_outside_every_window_and_empty_batches():
    t, d, g = rows(2, 6, 500, F32)
    x = drafts(d, {}, g)
    outs = {"p_accept": torch.full((6,), 7.0, device="cuda")}
    got = call(t, d, x, [0, 0, 2, 2], [0.0] * 6, [0.5] * 3, outs=outs)
    assert got["p_accept"] is outs["p_accept"] and (got["p_accept"][2:] == 7).all() and (got["p_accept"][:2] <= 1).all()
    assert got["n_acc"].tolist() == [0, 2, 0] and got["token"].tolist() == [-1] * 3
    got = call(t[:0], d[:0], x[:0], [0, 0], [], [0.5])
    assert got["n_acc"].tolist() == [0] and got["token"].tolist() == [-1]
    got = call(t, d, x, [0], [0.0] * 6, [])
    assert got["n_acc"].numel() == 0


@pytest.mark.gpu
def test_a_call_repeats_bit_for_bit_whatever_the_workspace_holds():
    T, V, cu = 20, 30000, [0, 5, 10, 15, 20]
    t, d, g = rows(4, T, V, BF16)
    x = drafts(d, {}, g)
    u, ud = torch.rand(T, generator=g), torch.rand(4, generator=g)
    f = {"top_k": torch.full((T,), 50, dtype=torch.int32), "top_p": torch.full((T,), 0.9)}
    size = ops.verify_drafts_workspace_size(T, V, 4, True, True)
    all_ = [call(t, d, x, cu, u, ud, f, f, workspace=torch.full((size,), fill, dtype=torch.uint8, device="cuda"))
            for fill in (0, 255, 91)]
    for got in all_[1:]:
        for n in got:
            assert torch.equal(torch.nan_to_num(got[n].float()), torch.nan_to_num(all_[0][n].float()))


@pytest.mark.gpu
def test_python_refusals():
    t, d, _ = rows(2, 6, 500, F32)
    f, i = (lambda *s: torch.zeros(*s, device="cuda")), (lambda *s: torch.zeros(*s, device="cuda", dtype=torch.int32))
    good = dict(target_logits=t.cuda(), draft_logits=d.cuda(), prop_tok=i(6), cu_q=i(3), u_accept=f(6), u_draw=f(2))
    for bad in (dict(draft_logits=d[:5].cuda()), dict(draft_logits=d.to(BF16).cuda()), dict(prop_tok=f(6)), dict(prop_tok=i(5)),
                dict(u_draw=f(3)), dict(u_accept=f(2)), dict(top_k=f(6)), dict(draft_top_p=f(5)), dict(cu_q=i(0)),
                dict(outs={"token": i(3)}), dict(outs={"finished": i(2)}), dict(draft_logits=None, draft_top_p=f(6)),
                dict(workspace=torch.zeros(10))):
        with pytest.raises(ValueError):
            ops.verify_drafts(**{**good, **bad})
    with pytest.raises(TypeError):
        ops.verify_drafts(**{**good, "u_draw": None})
    with pytest.raises(ops.IpdvError):
        ops.verify_drafts(**good, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))


# --- refusals (no GPU) ---

def c_drafts(**kw):
    a = dict(t=16, ts=500, d=16, ds=500, T=6, V=500, x=16, cu=16, B=2, ua=16, ud=16, n=16, tok=16, fin=16, pa=16, lp=16, dtype=0,
             ws=256, wsb=1 << 30)
    a.update(kw)
    return ops.lib().verify_drafts(a["t"], a["ts"], a["d"], a["ds"], a["T"], a["V"], a["x"], a["cu"], a["B"], a["ua"], a["ud"],
                                   *[None] * 8, -1, a["n"], a["tok"], a["fin"], a["pa"], a["lp"], a["dtype"], a["ws"], a["wsb"],
                                   None)


@pytest.mark.parametrize("kw,status", [
    (dict(t=None), -1), (dict(x=None), -1), (dict(cu=None), -1), (dict(ua=None), -1), (dict(ud=None), -1), (dict(n=None), -1),
    (dict(tok=None), -1), (dict(fin=None), -1), (dict(pa=None), -1), (dict(T=-1), -1), (dict(B=-1), -1), (dict(V=0), -1),
    (dict(ts=499), -1), (dict(ds=499), -1), (dict(V=262145, ts=1 << 20, ds=1 << 20), -2), (dict(T=1 << 22), -2),
    (dict(B=1 << 22), -2), (dict(dtype=4), -2), (dict(ws=264), -2), (dict(ws=None), -3), (dict(wsb=64), -3),
    (dict(B=0, t=None), 0)])
def test_drafts_refusals(kw, status):
    assert c_drafts(**kw) == status
    assert (ops.lib().ipdv_last_error() != b"") == (status != 0)


def test_workspace_query():
    size = ops.verify_drafts_workspace_size
    assert 0 < size(6, 500, 2) < size(6, 500, 2, True) and size(6, 262145, 2) == 0 and size(-1, 500, 2) == 0
