"""sample_logits against a 64-bit plain form, and its refusals."""
import math

import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests import q8_reference as ref

BF16, F32 = torch.bfloat16, torch.float32
INF = float("inf")


def call(l, u, T=None, k=None, p=None, m=None):
    M = l.shape[0]
    t = lambda x, d: None if x is None else torch.as_tensor(np.broadcast_to(np.asarray(x), (M,)).copy()).to(d).cuda()  # noqa: E731
    token, logp = ops.sample_logits(l.cuda(), t(u, F32), t(T, F32), t(k, torch.int32), t(p, F32), t(m, F32))
    return token.cpu().numpy(), logp.cpu().double().numpy()


def check(l, u, T=1.0, k=0, p=1.0, m=0.0):
    M = l.shape[0]
    b = lambda x, d=np.float32: np.broadcast_to(np.asarray(x, d), (M,))  # noqa: E731
    token, logp = call(l, u, T, k, p, m)
    lf = l.float().double().numpy()
    u, T, k, p, m = b(u), b(T), b(k, np.int32), b(p), b(m)
    for i in range(M):
        assert ref.draw_is_right(lf[i], float(T[i]), int(k[i]), float(p[i]), float(m[i]), float(u[i]), int(token[i]),
                                 float(logp[i])), (i, T[i], k[i], p[i], m[i], u[i], token[i], logp[i])
    return token


def gauss(M, V, dt, std=4.0, seed=0):
    return (std * torch.randn(M, V, generator=torch.Generator().manual_seed(seed))).to(dt)


def uniforms(M, seed=1):
    u = np.random.default_rng(seed).random(M).astype(np.float32)
    u[0] = 0.0
    u[-1] = 1 - 2.0 ** -24
    return u


FILTERS = [dict(), dict(T=0.6), dict(k=1), dict(k=50), dict(k=10 ** 6), dict(p=0.9), dict(p=0.999), dict(p=0.0), dict(m=0.05),
           dict(m=1.0), dict(m=2.0), dict(T=0.7, k=20, p=0.8, m=0.1), dict(T=1.3, k=400, p=0.95), dict(T=0.05, k=40, p=0.99),
           dict(T=5.0, p=0.9), dict(T=0.0), dict(k=3000 - 7, p=0.99)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("V", [1, 2, 63, 1000, 8191, 8192, 8193, 32003])
@pytest.mark.parametrize("f", FILTERS)
def test_draws_match_the_plain_form(dt, V, f):
    check(gauss(7, V, dt, seed=V), uniforms(7), **f)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("V", [151936, 262144])
def test_large_vocabularies_and_mixed_parameters(dt, V):
    M = 12
    r = np.random.default_rng(3)
    check(gauss(M, V, dt), uniforms(M), r.choice([0.0, 0.3, 0.7, 1.0, 1.5], M), r.choice([0, 1, 50, 3000], M),
          r.choice([0.3, 0.9, 1.0], M), r.choice([0.0, 0.02], M))


@pytest.mark.gpu
@pytest.mark.parametrize("f", [dict(), dict(k=1), dict(k=700), dict(k=20000), dict(p=0.5), dict(p=0.37, k=30000), dict(m=0.5)])
@pytest.mark.parametrize("few", [1, 3])
def test_equal_logits_go_by_index(f, few):
    """All logits equal, or of three values: ties by the thousand, the lowest indices stay."""
    V = 40001
    l = torch.zeros(5, V)
    if few == 3:
        l = torch.randint(0, 3, (5, V), generator=torch.Generator().manual_seed(0)).float() * 0.01
    check(l, uniforms(5), **f)
    if few == 1 and f.get("k"):
        assert call(l, uniforms(5), **f)[0].max() < f["k"]


@pytest.mark.gpu
def test_masked_rows():
    l = gauss(8, 20000, F32)
    l[0] = -INF                               # nothing left
    l[1, 1:] = -INF                           # one entry
    l[2, :-3] = -INF                          # the last three, in the last chunk
    l[3, 5] = float("nan")
    l[4, 19999] = INF
    l[5] = torch.where(torch.arange(20000) % 17 == 3, l[5], torch.tensor(-INF))
    l[6] = torch.finfo(F32).min               # a mask of the type's lowest value, two entries stay
    l[6, [77, 9000]] = torch.tensor([1.0, 1.5])
    l[7] = torch.finfo(F32).min               # and a row of nothing else: all alike
    for f in (dict(), dict(k=5), dict(p=0.9), dict(m=0.2), dict(T=0.0), dict(T=0.5, k=3, p=0.5)):
        token, logp = call(l, 0.6, **f)
        assert (token[[0, 3, 4]] == -1).all() and np.isnan(logp[[0, 3, 4]]).all()
        assert token[1] == 0 and logp[1] == 0.0
        check(l[[1, 2, 5, 6, 7]], 0.6, **f)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("many", [300, 2500, 5000])
def test_cuts_in_crowded_bins(dt, many):
    """A cut among `many` entries within a small step of one another, of which one
    part of the vocabulary holds a few, another most, and a third none."""
    V = 50000
    g = torch.Generator().manual_seed(many)
    l = torch.full((6, V), -20.0) + torch.randn(6, V, generator=g)
    crowd = torch.cat([torch.randperm(16000, generator=g)[:100], 32768 + torch.randperm(16000, generator=g)[: many - 100]])
    l[:, crowd] = 2.0 + 0.05 * torch.randn(6, many, generator=g)
    l[:, 40] = 6.0
    l = l.to(dt)
    for f in (dict(k=many // 2), dict(k=many), dict(k=many // 3, p=0.6), dict(p=0.5), dict(p=0.97), dict(p=0.6, m=0.0183),
              dict(k=many - 50, m=0.019), dict(k=many - 50, p=0.9, m=0.0178)):
        check(l, uniforms(6), **f)


@pytest.mark.gpu
def test_many_rows():
    """More rows than workgroups at once; rows of one logit set repeat as their uniforms do."""
    few = gauss(5, 300, F32)
    rows = np.random.default_rng(0).integers(0, 5, 20000)
    u = np.random.default_rng(1).integers(0, 50, 20000).astype(np.float32) / 50
    token, logp = call(few[rows], u, 0.9, 30, 0.8)
    for r in range(5):
        for x in range(50):
            same = (rows == r) & (u == np.float32(x) / np.float32(50))
            assert len(set(token[same])) <= 1
    some = np.arange(0, 20000, 97)
    for i in some:
        assert ref.draw_is_right(few[rows[i]].double().numpy(), float(np.float32(0.9)), 30, float(np.float32(0.8)), 0.0, float(u[i]),
                                 int(token[i]), float(logp[i]))


@pytest.mark.gpu
def test_odd_temperatures():
    l = gauss(6, 3001, F32)
    token, logp = call(l, 0.5, T=[-1.0, float("nan"), 0.0, INF, 1e-30, 1e30])
    assert (token[:2] == -1).all() and np.isnan(logp[:2]).all()
    assert token[2] == int(l[2].argmax()) and logp[2] == 0.0 and token[4] == int(l[4].argmax())
    for i in (3, 5):                          # uniform
        assert token[i] == 1500 and abs(logp[i] + math.log(3001)) < 1e-5
    # parameters that are no numbers filter nothing
    a = call(l, 0.5, p=float("nan"), m=float("nan"))
    b = call(l, 0.5)
    assert (a[0] == b[0]).all()


@pytest.mark.gpu
def test_far_apart_logits_and_low_temperatures():
    """Chunks whose entries all lie far below another's; a cut that falls below what can be drawn."""
    l = gauss(4, 30000, F32)
    l[:, 25000] = 500.0
    l[1, 100] = 499.0
    l[2, 29999] = 500.0
    for f in (dict(), dict(k=50), dict(p=0.99), dict(T=0.02, k=3), dict(m=0.3)):
        check(l, np.array([0.1, 0.2, 0.6, 0.99], np.float32), **f)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_strided_rows_and_given_outputs(dt):
    wide = gauss(6, 2050, dt)
    u = torch.from_numpy(uniforms(6)).cuda()
    view = wide.cuda()[:, 1: 2001]            # rows apart, and no row on 16 bytes
    token, logp = torch.full((6,), 9, dtype=torch.int32).cuda(), torch.zeros(6).cuda()
    ws = torch.full((ops.sample_logits_workspace_size(6, 2000),), 255, dtype=torch.uint8).cuda()
    out = ops.sample_logits(view, u, token=token, logp=logp, workspace=ws)
    assert out[0] is token and out[1] is logp
    again = ops.sample_logits(view.contiguous(), u)
    assert torch.equal(token, again[0]) and torch.equal(logp, again[1])


@pytest.mark.gpu
def test_draws_follow_the_distribution():
    """20000 evenly spaced uniforms count out every entry's probability."""
    l = gauss(1, 50, F32, 2.0).expand(20000, 50).contiguous()
    u = ((np.arange(20000) + 0.5) / 20000).astype(np.float32)
    token, _ = call(l, u, T=0.8, k=30)
    p = np.exp(l[0].double().numpy() / 0.8)
    p[np.argsort(-p, kind="stable")[30:]] = 0
    assert np.abs(np.bincount(token, minlength=50) / 20000 - p / p.sum()).max() <= 1.01 / 20000


def c_call(**kw):
    a = dict(l=16, s=1000, M=4, V=1000, u=16, token=16, dtype=0, ws=16, wsb=1 << 30)
    a.update(kw)
    return ops.lib().sample_logits(a["l"], a["s"], a["M"], a["V"], a["u"], None, None, None, None, a["token"], None, a["dtype"],
                                   a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(l=None), -1), (dict(u=None), -1), (dict(token=None), -1), (dict(M=-1), -1), (dict(V=0), -1), (dict(s=999), -1),
    (dict(V=262145, s=300000), -2), (dict(M=1 << 24), -2), (dict(dtype=2), -2), (dict(dtype=0x11), -2), (dict(ws=None), -3),
    (dict(wsb=100), -3), (dict(ws=24), -2), (dict(M=0, l=None), 0)])
def test_sample_refusals(kw, status):
    assert c_call(**kw) == status
    assert (ops.lib().ipdv_last_error() != b"") == (status != 0)


def test_workspace_query():
    assert ops.sample_logits_workspace_size(64, 151936) > 0
    assert ops.sample_logits_workspace_size(64, 262145) == 0 and ops.sample_logits_workspace_size(0, 100) == 0
