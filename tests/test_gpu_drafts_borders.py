"""Verdicts on drafts at the borders of the distributions: u of 0, drafts that a filter cuts
far below the maximum, vocabularies masked by a finite fill."""
import numpy as np
import pytest
import torch

from tests import masked_reference as ref
from tests import q8_reference as filters
from tests.masked_reference import BF16, F32, f64
from tests.test_gpu_drafts import call


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
