"""sample_logits where its arithmetic changes hands or rounds: far bins, the
least temperatures, needs and uniforms that fall between two prefix sums."""
import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests.test_gpu_sample_logits import BF16, F32, INF, call, check, gauss  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,l", [(float.fromhex(a), float.fromhex(b)) for a, b in (
    # 8 l / T just below 2^24, and fp32 rounds 8 / T up: the next logit's floor in 64 bits is one less than l's in 32
    ("0x1.eb94a4p-17", "0x1.eb94a0p+4"), ("0x1.dbdb7ep-15", "0x1.dbdb7ap+6"), ("0x1.f44f66p-11", "0x1.f44f62p+10"),
    ("0x1.deb6fap-19", "0x1.deb6f6p+2"), ("0x1.e1f30ap-23", "0x1.e1f306p-2"))])
@pytest.mark.parametrize("f", [dict(), dict(k=2), dict(k=9), dict(p=0.6), dict(m=0.3), dict(k=8, p=0.8, m=0.05)])
def test_bins_next_to_the_end_of_fp32_fractions(T, l, f):
    """Neighbouring logits on both sides of 8 l / T = 2^24, in one part of the vocabulary and in several."""
    near = (np.array(l, np.float32).view(np.uint32) + np.arange(-6, 7, dtype=np.int64)).astype(np.uint32).view(np.float32)
    rows = torch.full((4, 40000), float(l) - 1.0)
    rng = np.random.default_rng(1)
    for row, (lo, hi) in zip(rows, ((0, 16000), (16384, 32000), (0, 40000), (0, 40000))):
        at = rng.choice(np.arange(lo, hi), 13, replace=False)
        row[torch.from_numpy(at)] = torch.from_numpy(near)
    rows[3][rows[3] == float(near.max())] = float(l) - 1.0      # a maximum of its own
    check(rows, np.array([0.1, 0.5, 0.77, 0.999], np.float32), T=T, **f)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("T", [1e-45, 1e-39, 2.3e-38, 2.0 ** -124, 1e-37])
@pytest.mark.parametrize("f", [dict(), dict(k=5), dict(p=0.9), dict(m=0.2), dict(k=3, p=0.7, m=0.5)])
def test_least_temperatures_with_a_maximum_of_zero(dt, T, f):
    """Log-probs of a certain token, maxima subtracted, and rows of zeros: 8 / T passes the largest fp32 number below 2.35e-38."""
    l = -gauss(4, 40000, dt).abs() - 0.5
    l[0] = -INF
    l[0, 39000] = 0.0
    l[1, 20001] = -0.0
    l[2, [17000, 33000, 39999]] = 0.0
    l[3] = 0.0
    check(l, np.array([0.5, 0.0, 0.4, 0.7], np.float32), T=T, **f)


def test_a_need_between_two_sums():
    """One entry of logit 0, k of -0.1 and n of another, top-p a hair (2e-12) above
    the mass of the first k + 1: the next entry is kept too, and no more.  The mass
    before the last bin, got by taking that bin off the sum up to it, is as much
    above the sum up to the bin before."""
    cases = [(-0.24, 2, 257117, "0x1.d21f4cp-17"), (-0.13, 2, 226936, "0x1.d91a0cp-17"), (-0.2, 1, 171842, "0x1.c649e0p-17"),
             (-0.2, 1, 221202, "0x1.60eaecp-17"), (-0.2, 1, 117596, "0x1.4bec00p-16"), (-0.2, 1, 241385, "0x1.4368cap-17"),
             (-0.13, 2, 242759, "0x1.ba43f4p-17"), (-0.2, 1, 102910, "0x1.7b49d8p-16")]
    u = np.array([0.0, 0.3, 0.6, 0.95], np.float32)
    l = torch.full((len(cases), 262144), -INF)
    for row, (x, k, n, _) in zip(l, cases):
        row[200: 200 + n] = x
        row[50: 50 + k] = -0.1
        row[20] = 0.0
    p = np.array([float.fromhex(c[3]) for c in cases], np.float32)
    token, logp = call(l.repeat_interleave(4, 0), np.tile(u, len(cases)), p=p.repeat(4))
    for i, (x, k, _, _) in enumerate(cases):
        v = np.array([20, *range(50, 50 + k), 200])
        w = np.exp([0.0] + [-0.1] * k + [x])
        at = np.searchsorted(np.cumsum(w) / w.sum(), u, side="right")
        assert (token[4 * i: 4 * i + 4] == v[at]).all(), (i, token[4 * i: 4 * i + 4])
        assert np.abs(logp[4 * i: 4 * i + 4] - np.log(w / w.sum())[at]).max() < 1e-5


def test_a_uniform_between_two_sums():
    """A first entry of e^-27.7, nothing beside it, and zeros behind: uniforms next to
    its share fall on it or on the first zero, which is the next that holds mass."""
    V, M = 16384, 512
    l = torch.zeros(1, V)
    l[0, :32] = -INF
    l[0, 0] = -27.7
    share = np.exp(-27.7) / (V - 32 + np.exp(-27.7))
    u = (share * (1 + np.linspace(-0.02, 0.02, M))).astype(np.float32)
    token, _ = call(l.expand(M, V).contiguous(), u)
    assert set(token) == {0, 32}
    assert (np.diff(token) >= 0).all() and abs(u[np.argmax(token)] / share - 1) < 1e-4
