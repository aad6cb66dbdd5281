"""ipdv_rope_inv_freq's ramp over its whole range (host arithmetic, no GPU)."""
import math

import numpy as np
import pytest

from paper_2609_36546_amd import ops


@pytest.mark.parametrize("rot", [4, 16, 64, 128, 256])
@pytest.mark.parametrize("base", [30.0, 1e4, 5e5])
@pytest.mark.parametrize("length", [1, 5, 40, 2048, 8192, 65536, 131072, 1 << 24, 2 ** 31 - 1])
@pytest.mark.parametrize("fast,slow", [(32.0, 1.0), (8.0, 2.5)])
def test_ramp(rot, base, length, fast, slow):
    factor, n = 4.0, rot // 2
    f, _ = ops.rope_inv_freq(rot, base, ops.ROPE_YARN, factor, length, fast, slow)
    plain = np.array([base ** (-2.0 * p / rot) for p in range(n)])
    ratio = f.double().numpy() / plain
    turns = length * plain / (2 * math.pi)
    step = 2.0 ** -24 + 1e-9                               # one rounding to fp32
    pair = lambda t: rot * math.log(length / (2 * math.pi * t)) / (2 * math.log(base))  # noqa: E731
    hi, lo = min(math.ceil(pair(slow)), rot - 1), max(math.floor(pair(fast)), 0)
    for p in range(n):
        ramp = 1.0 if p >= hi else 0.0 if p <= lo else (p - lo) / (hi - lo)
        assert abs(ratio[p] - (1 - ramp + ramp / factor)) <= step, (p, turns[p])
    # what the header says: the whole factor only up to beta_slow turns, none of it from beta_fast on
    assert (ratio[turns > slow * (1 + 1e-9)] > 1 / factor + step).all()
    assert (np.abs(ratio[turns < slow * base ** (-2.0 / rot)] - 1 / factor) <= step).all()
    assert (np.abs(ratio[turns > fast * base ** (2.0 / rot)] - 1) <= step).all()
    assert (np.diff(ratio) <= 2 * step).all()


@pytest.mark.parametrize("rot", [64, 128])
def test_a_small_base_over_a_long_context(rot):
    """The last pair turns 2.4 (2.8) times over 131072 positions: it lies inside the ramp."""
    f, _ = ops.rope_inv_freq(rot, 1e4, ops.ROPE_YARN, 4.0, 131072)
    last = 1e4 ** (-(rot - 2) / rot)
    assert 131072 * last / (2 * math.pi) > 2.4
    assert 0.45 < float(f[-1]) / last < 0.50
