"""Plain forms, in 64 bits, of the operators around the 8-bit cache (numpy and
CPU torch; no code of the library)."""
import math

import numpy as np
import torch

E4M3 = torch.float8_e4m3fn


def rope(x, pos, inv_freq, layout, factor=1.0, inverse=False):
    """x [T, H, D] float64, pos [T], inv_freq [R/2]: pairs turned as complex numbers."""
    R = 2 * len(inv_freq)
    a = np.asarray(pos, np.float64)[:, None] * np.asarray(inv_freq, np.float64)
    w = factor * np.exp((-1j if inverse else 1j) * a)[:, None, :]
    y = x.astype(np.float64).copy()
    i, j = (slice(0, R // 2), slice(R // 2, R)) if layout == 0 else (slice(0, R, 2), slice(1, R, 2))
    z = (y[..., i] + 1j * y[..., j]) * w
    y[..., i], y[..., j] = z.real, z.imag
    return y


def quantise(x):
    """x [..., D] float64 -> (values that the cache stands for, scale bytes).  A row
    that is not finite becomes NaN with byte 255."""
    x = np.asarray(x, np.float64)
    amax = np.abs(x).max(-1)
    ok = np.isfinite(x).all(-1)
    a = np.where(ok & (amax > 0), amax, 1.0)
    e = np.ceil(np.log2(a / 448.0)).astype(np.int64)
    e += a > 448.0 * 2.0 ** e                       # rounding of the logarithm
    e -= a <= 448.0 * 2.0 ** (e - 1)
    e = np.where(amax > 0, np.maximum(e, -126), 0)
    y = np.where(ok[..., None], x, 0.0) * 2.0 ** -e[..., None].astype(np.float64)
    mag = np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6)))
    step = 2.0 ** (mag - 3)
    v = np.round(y / step) * step * 2.0 ** e[..., None].astype(np.float64)   # half to even
    return np.where(ok[..., None], v, np.nan), np.where(ok, e + 127, 255).astype(np.uint8)


def slots(page_table, ctx, cu, seqs, page_size):
    """(row, sequence, position, page, slot) of every window row of `seqs`."""
    for b in seqs:
        for r in range(cu[b], cu[b + 1]):
            pos = int(ctx[b]) + r - int(cu[b])
            yield r, b, pos, int(page_table[b, pos // page_size]), pos % page_size


def cached(k, v, scale, page, slot):
    """Keys and values of one slot, float64 [Hkv, D], from CPU copies of the cache."""
    kk = k[page, :, :, slot, :].float().reshape(k.shape[1], -1).double().numpy()
    vv = v[page, :, :, slot].float().double().numpy()
    e = scale[page, :, :, slot].numpy().astype(np.float64) - 127.0
    f = np.where(e == 128.0, np.nan, 2.0 ** np.where(e == 128.0, 0.0, e))
    return kk * f[:, :1], vv * f[:, 1:]


def attention(q, K, V, L, scale):
    """q [k, Hq, D], K and V [n, Hkv, D] float64: row i sees positions 0 .. L + i."""
    k, Hq, D = q.shape
    G = Hq // K.shape[1]
    out = np.zeros((k, Hq, D))
    for h in range(Hq):
        s = scale * (q[:, h] @ K[:, h // G].T)
        for i in range(k):
            w = np.exp(s[i, : L + i + 1] - s[i, : L + i + 1].max())
            out[i, h] = (w / w.sum()) @ V[: L + i + 1, h // G]
    return out


def kept_prefix(l, T, k, p, m, nudge=0.0):
    """The row's order and the length of the kept prefix; `nudge` moves the
    masses that borders are compared with."""
    l = np.asarray(l, np.float64)
    order = np.argsort(-l, kind="stable")
    order = order[np.isfinite(l[order])]
    if T == 0:
        return order, 1, np.ones(len(order))
    x = (l[order] - l[order[0]]) / T
    w = np.exp(x)
    n = len(order)
    if k and k > 0:
        n = min(n, k)
    if p is not None and p < 1:
        before = np.concatenate([[0.0], np.cumsum(w[:n])[:-1]]) / w[:n].sum()
        n = min(n, max(1, int((before < p + nudge).sum())))
    if m is not None and m > 0:
        n = min(n, max(1, int((x >= math.log(m)).sum())))
    return order, n, w


def draw_is_right(l, T, k, p, m, u, token, logp, slack=1e-6):
    """Whether a draw is the inverse of the filtered distribution, give or take
    `slack` of the mass at a border."""
    ends = {kept_prefix(l, T, k, p, m, d)[1] for d in (-slack, 0.0, slack)}
    order, _, w = kept_prefix(l, T, k, p, m)
    for n in range(min(ends), max(ends) + 1):
        idx = np.sort(order[:n])
        mass = np.zeros(len(l))
        mass[order[:n]] = w[:n]
        c = np.cumsum(mass[idx]) / mass[idx].sum()
        at = np.searchsorted(idx, token)
        if at == len(idx) or idx[at] != token or mass[token] == 0:
            continue
        lo = c[at - 1] if at else 0.0
        if lo - slack <= u <= c[at] + slack and abs(logp - math.log(mass[token] / mass[idx].sum())) < 1e-5:
            return True
    return False
