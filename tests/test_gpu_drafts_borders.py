"""Verdicts on drafts at the borders of the distributions: u of 0, drafts that a filter cuts
far below the maximum, vocabularies masked by a finite fill."""
import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests import masked_reference as ref
from tests import q8_reference as filters
from tests.masked_reference import BF16, F32, f64
from tests.test_gpu_drafts import c_drafts, call, check, rows


def at(f, name, m):
    return None if f.get(name) is None else f[name][m].item()


def kept(l, f, m):
    """Row m's kept entries, and its temperature."""
    T = at(f, "temperature", m)
    T = 1.0 if T is None else T
    order, n, _ = filters.kept_prefix(f64(l)[m], T, at(f, "top_k", m), at(f, "top_p", m), at(f, "min_p", m))
    return order[:n], T


def probs(l, f, m):
    return ref.softmax_kept(f64(l)[m], *kept(l, f, m))


def check_exactly(target, draft, tf, df, x, cu, u, ud, got):
    """Every decision as the 64-bit form has it: for u of 0, which asks only whether a
    probability is 0."""
    for b in range(len(cu) - 1):
        r = slice(int(cu[b]), int(cu[b + 1]))
        P = np.array([probs(target, tf, m) for m in range(r.start, r.stop)])
        Q = None if draft is None else np.array([probs(draft, df, m) for m in range(r.start, r.stop)])
        n, token, _, ratio, logp, _ = ref.verdict(P, Q, x[r], u[r], ud[b])
        # 1e-9, the rounding to fp32, and its least normal number
        assert np.allclose(f64(got["p_accept"][r]), ratio, rtol=2.0 ** -24 + 2e-9, atol=2.0 ** -126)
        assert (int(got["n_acc"][b]), int(got["token"][b])) == (n, token)
        if token >= 0:
            assert abs(float(got["logp"][b]) - logp) <= 2.0 ** -23 * abs(logp) + 1e-8


FILLS = [-1e4, -1e9, torch.finfo(BF16).min, -float("inf")]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("fill", FILLS)
@pytest.mark.parametrize("V,allowed", [(20000, [1500, 9000, 9001, 19999]), (300, [0, 299]), (40000, [8200])])
@pytest.mark.parametrize("temp", [None, 0.3, 2.0])
def test_a_vocabulary_masked_by_a_fill(dt, fill, V, allowed, temp):
    """A fill 700 T or more below the maximum has no probability: a u of 0 accepts none of it and
    draws none of it, with drafts of either kind."""
    t = torch.full((6, V), fill, dtype=F32)
    g = torch.Generator().manual_seed(V)
    t[:, allowed] = torch.randn(6, len(allowed), generator=g)
    d = t.clone()
    d[:, allowed] += torch.randn(6, len(allowed), generator=g)
    d[1] = torch.randn(V, generator=g)               # a draft model that does not know of the mask
    t, d = t.to(dt), d.to(dt)
    f = {} if temp is None else {"temperature": torch.full((6,), temp)}
    masked = next(v for v in range(1, V) if v not in allowed)
    x = np.array([masked, masked, -1, allowed[-1], masked, -1])
    cu, zero = [0, 1, 2, 3, 5, 6], np.zeros(6)
    for draft, df in ((None, {}), (d, f)):
        got = call(t, draft, x, cu, zero, zero[:5], f, df)
        check_exactly(t, draft, f, df, x, cu, zero, zero, got)
        assert got["n_acc"].tolist() == [0, 0, 0, 1, 0]
        assert set(got["token"].tolist()) <= set(allowed)


def every(T, **f):
    return {n: torch.full((T,), v, dtype=torch.int32 if n == "top_k" else F32) for n, v in f.items()}


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("V", [5003, 40000])
@pytest.mark.parametrize("temp,k", [(0.05, 20), (0.1, 50), (0.2, 200), (0.2, 3000)])
@pytest.mark.parametrize("certain", [False, True])
def test_top_k_far_below_the_maximum(dt, V, temp, k, certain):
    """The k-th entry lies more than 32 nats below the first.  Drafts inside, outside the
    target's and outside both top-ks, at u of 0."""
    T = 24
    t, d, g = rows(V + k, T, V, dt)
    f = every(T, temperature=temp, top_k=k)
    df = {} if certain else f
    d = None if certain else d
    # one row of each sequence is drafted from inside, so that the second decides
    x = np.zeros(T, np.int64)
    last = []
    for m in range(T):
        inside, _ = kept(t, f, m)
        other = kept(d, f, m)[0] if d is not None else np.zeros(0, np.int64)
        last.append((f64(t)[m].max() - f64(t)[m][inside[-1]]) / temp)
        only_draft = np.setdiff1d(other, inside)
        out = np.setdiff1d(np.arange(V), np.union1d(inside, other))
        x[m] = (inside[0], inside[-1], only_draft[0] if len(only_draft) else out[0], out[0], out[-1], -1)[m % 6]
    assert np.mean(np.array(last) > 32) > 0.5
    cu, u = [0, 2, 3, 4, 5, 6, 12, 13, 14, 15, 16, 17, 18, 24], np.zeros(T)
    for ud in (np.zeros(13), torch.rand(13, generator=g).numpy()):
        got = call(t, d, x, cu, u, ud, f, df)
        if not ud.any():
            check_exactly(t, d, f, df, x, cu, u, ud, got)
        else:
            check(t, d, f, df, x, cu, u, ud, got)
    cut = np.isin(np.arange(T) % 6, (3, 4))
    assert (f64(got["p_accept"])[cut] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_drafts_outside_both_top_ks(dt):
    t = torch.tensor([[0.0, -40.0, -41.0, -42.0]] * 4).to(dt)
    f = every(4, top_k=2)
    x, cu = np.array([3, 2, 1, 0]), [0, 1, 2, 4]
    got = call(t, t, x, cu, [0.0] * 4, [0.0] * 3, f, f)
    # nothing is left of max(0, p - q): drawn from p
    assert got["p_accept"].tolist() == [0, 0, 1, 1]
    assert got["n_acc"].tolist() == [0, 0, 2] and got["token"].tolist() == [0, 0, -1]
    got = call(t, None, x, cu, [0.0] * 4, [0.0] * 3, f)
    assert got["n_acc"].tolist() == [0, 0, 2] and got["token"].tolist() == [0, 0, -1]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("V", [300, 30000])
@pytest.mark.parametrize("k", [2, 70, 1000, 29000, 40000])
@pytest.mark.parametrize("ties", [False, True])
def test_a_row_whose_entries_all_lie_far_below_its_first(dt, V, k, ties):
    """One entry at 0, all others 40 to 100 nats below, in any order; with ties, of few values."""
    T = 6
    rng = np.random.default_rng(V + k)
    l = -40.0 - (rng.integers(0, 7, (T, V)) * 8.0 if ties else 60.0 * rng.random((T, V)))
    l[np.arange(T), rng.integers(0, V, T)] = 0.0
    t = torch.from_numpy(l).to(F32).to(dt)
    f = every(T, top_k=k)
    x = np.zeros(T, np.int64)
    for m in range(T):
        order, n, _ = filters.kept_prefix(f64(t)[m], 1.0, 0, None, None)
        x[m] = (order[min(k, V) - 1], order[k] if k < V else V, order[0], order[-1], -1, order[k // 2 % V])[m]
    cu, u, ud = list(range(T + 1)), np.zeros(T), np.zeros(T)
    check_exactly(t, None, f, {}, x, cu, u, ud, call(t, None, x, cu, u, ud, f))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("more", [{}, dict(top_k=3), dict(top_k=100), dict(temperature=0.5)])
def test_a_min_p_far_below_the_maximum(dt, more):
    """min-p of 1e-20: entries down to 46 nats are kept, others not."""
    V, T = 9000, 4
    t = torch.full((T, V), -60.0)
    t[:, 77], t[:, 8191], t[:, 3], t[:, 500] = 0.0, -20.0, -22.0, -45.0
    t[:, 40], t[:, 8999] = -47.0, -23.5
    t = t.to(dt)
    f = every(T, min_p=1e-20, **more)
    x = np.array([40, 500, 8999, 12])
    cu, u, ud = list(range(T + 1)), np.zeros(T), np.zeros(T)
    got = call(t, None, x, cu, u, ud, f)
    check_exactly(t, None, f, {}, x, cu, u, ud, got)
    assert got["n_acc"].tolist()[0] == 0 and got["n_acc"].tolist()[3] == 0


@pytest.mark.gpu
def test_log_probabilities_over_the_draws():
    """logp may be u_draw; other outputs over inputs are refused."""
    T, V, cu = 12, 20000, [0, 4, 8, 12]
    t, d, g = rows(6, T, V, F32)
    x = np.full(T, -1)
    x[::4] = f64(d).argmax(1)[::4]
    u, ud = torch.rand(T, generator=g).cuda(), torch.rand(3, generator=g).cuda()
    i32 = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()  # noqa: E731
    args = t.cuda(), d.cuda(), i32(x), i32(cu), u
    want = ops.verify_drafts(*args, ud)
    place = ud.clone()
    got = ops.verify_drafts(*args, place, outs={"logp": place})
    assert got["logp"] is place and torch.equal(torch.nan_to_num(place), torch.nan_to_num(want["logp"]))
    assert torch.equal(got["token"], want["token"]) and (got["token"] >= 0).all()
    with pytest.raises(ops.IpdvError, match="may not be inputs"):
        ops.verify_drafts(*args, ud, outs={"p_accept": u})


# --- refusals (no GPU) ---

@pytest.mark.parametrize("kw", [dict(pa=64), dict(n=32), dict(tok=32), dict(tok=48)])
def test_outputs_over_inputs_are_refused(kw):
    a = dict(x=32, cu=48, ua=64, ud=80, n=96, tok=112, fin=128, pa=144, lp=160)
    assert c_drafts(**{**a, **kw}) == -1
    assert b"may not be inputs" in ops.lib().ipdv_last_error()
