"""Plain forms, in 64 bits, of attention with modified scores, the weights that it
gives, eviction by them and the verdict on drafts by probabilities (numpy; no code
of the library), and batches to run them on."""
import math

import numpy as np
import torch

BF16, F32 = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().float().cpu().double().numpy()


def limits(L, k, window=0, first=None, end=None):
    """First and end key of every row of a window of k over L cached tokens."""
    p = L + np.arange(k)
    lo = np.maximum(first if first is not None else 0, 0) + np.zeros(k, np.int64)
    hi = np.minimum(end if end is not None else p + 1, L + k)
    if window:
        lo = np.maximum(lo, p - window + 1)
    return lo, hi


def scores(q, K, L, scale, cap, slopes, h):
    """Modified scores [k, n] of head h, and a bound of what fp32 sums of them are off by."""
    G = q.shape[1] // K.shape[1]
    k, n, D = q.shape[0], K.shape[0], q.shape[2]
    with np.errstate(invalid="ignore"):
        x = scale * (q[:, h] @ K[:, h // G].T)
        size = scale * (np.abs(q[:, h]) @ np.abs(K[:, h // G]).T)
        if cap:
            x = cap * np.tanh(x / cap)
        if slopes is not None:
            x = x - slopes[h] * np.abs((L + np.arange(k))[:, None] - np.arange(n))
    # D products summed, then a few roundings of the score or the cap
    return x, (D + 8) * 2.0 ** -24 * size + 16 * 2.0 ** -24 * (np.abs(x) + cap)


def attention(q, K, V, L, scale, lo, hi, cap=0.0, slopes=None):
    """q [k, Hq, D], K and V [n, Hkv, D]: outputs, lse, and per output what its
    probabilities' errors are measured in: sum p |V|, and the largest error of a score."""
    k, Hq, D = q.shape
    G = Hq // K.shape[1]
    out, size = np.zeros((k, Hq, D)), np.zeros((k, Hq, D))
    lse, err = np.full((k, Hq), -np.inf), np.zeros((k, Hq))
    for h in range(Hq):
        x, e = scores(q, K, L, scale, cap, slopes, h)
        for i in range(k):
            if lo[i] >= hi[i]:
                continue
            s = x[i, lo[i]: hi[i]]
            m = s.max()
            w = np.exp(s - m)
            V_i = V[lo[i]: hi[i], h // G]
            out[i, h], size[i, h] = (w / w.sum()) @ V_i, (w / w.sum()) @ np.abs(V_i)
            lse[i, h], err[i, h] = m + math.log(w.sum()), e[i, lo[i]: hi[i]].max()
    return out, lse, size, err


def check_attention(out, lse, want, dt, n, rounded):
    """`rounded`: probabilities are rounded to bf16 once."""
    ref, ref_lse, size, err = want
    half = torch.finfo(dt).eps / 2
    # a probability is off by e^(2 err) - 1 with its normalisation; sums of n terms in fp32; 2^-16: two
    # bf16 terms; the output's own rounding
    p = (2 * err + n * 2.0 ** -23 + (2.0 ** -8 if rounded else 2.0 ** -16 if dt == BF16 else 2.0 ** -22))[..., None]
    got = f64(out)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    ok = ~np.isnan(ref)
    bad = np.abs(got - ref) > p * size + half * np.abs(ref) * (1 + p) + 1e-30
    assert not bad[ok].any(), (np.abs(got - ref) / (p * size + half * np.abs(ref) + 1e-30))[ok].max()
    if lse is not None:
        g = f64(lse)
        live = np.isfinite(ref_lse)
        assert np.array_equal(np.isneginf(g), np.isneginf(ref_lse))
        tol = 2 * err + n * 2.0 ** -23 + 2.0 ** -22 * (1 + np.abs(np.where(live, ref_lse, 0)))
        assert (np.abs(g - ref_lse)[live] <= tol[live]).all()


def weights(q, K, lse, L, scale, lo, hi, cap=0.0, slopes=None):
    """What every key gathers [n, Hkv], and a bound of what fp32 is off by."""
    k, Hq, _ = q.shape
    n, Hkv = K.shape[:2]
    out, err = np.zeros((n, Hkv)), np.zeros((n, Hkv))
    for h in range(Hq):
        x, e = scores(q, K, L, scale, cap, slopes, h)
        for i in range(k):
            s = slice(lo[i], hi[i])
            if lo[i] >= hi[i]:
                continue
            w = np.exp(x[i, s] - lse[i, h])
            out[s, h * Hkv // Hq] += w
            # 2^-126: a weight below the least normal fp32 number may be 0
            err[s, h * Hkv // Hq] += w * (e[i, s] + 4 * 2.0 ** -24 * (np.abs(lse[i, h]) + 4 + k * Hq // Hkv)) + 2.0 ** -126
    return out, err


class Batch:
    """Ragged windows over a paged cache whose slots hold NaN where nothing was written."""

    def __init__(self, windows, Hq, Hkv, D, ps, dt, seed=0, extra=3, spread=1.0):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.dt, self.ps, self.Hkv, self.D, self.Hq = dt, ps, Hkv, D, Hq
        self.ctx = np.array([w[0] for w in windows], np.int32)
        self.k = np.array([w[1] for w in windows], np.int32)
        self.cu = np.concatenate([[0], np.cumsum(self.k)]).astype(np.int32)
        self.T, self.max_q = int(self.cu[-1]), max(1, int(self.k.max()))
        need = -(-(self.ctx + self.k) // ps)
        P = int(need.sum()) + extra
        ids = rng.permutation(P)
        self.table = np.full((len(windows), max(1, int(need.max()))), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at: at + n]
            at += n
        self.free = ids[at:].astype(np.int32)
        kc = torch.full((P, Hkv, D // 32, ps, 32), float("nan"), dtype=dt)
        vc = torch.full((P, Hkv, D, ps), float("nan"), dtype=dt)
        self.K, self.V = [], []
        rand = lambda *s: (spread * torch.randn(*s, generator=g)).to(dt)  # noqa: E731
        self.q, self.k_new, self.v_new = rand(self.T, Hq, D), rand(self.T, Hkv, D), rand(self.T, Hkv, D)
        for b, L in enumerate(self.ctx):
            k, v = rand(int(L), Hkv, D), rand(int(L), Hkv, D)
            for p in range(int(L)):
                kc[self.table[b, p // ps], :, :, p % ps, :] = k[p].view(Hkv, -1, 32)
                vc[self.table[b, p // ps], :, :, p % ps] = v[p]
            r = slice(int(self.cu[b]), int(self.cu[b + 1]))
            self.K.append(np.concatenate([f64(k), f64(self.k_new[r])]))
            self.V.append(np.concatenate([f64(v), f64(self.v_new[r])]))
        self.kc, self.vc = kc.cuda(), vc.cuda()
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()  # noqa: E731
        self.args = (dev(self.table), dev(self.ctx), dev(self.cu), self.max_q)
        self.scale = 1.0 / math.sqrt(D)

    def rows(self, b):
        return slice(int(self.cu[b]), int(self.cu[b + 1]))

    def read(self, kc, vc, table, b, p):
        """Key and value of a position, from host copies of the caches."""
        page, slot = int(table[b, p // self.ps]), p % self.ps
        return f64(kc[page, :, :, slot, :].reshape(self.Hkv, self.D)), f64(vc[page, :, :, slot])


def softmax_kept(l, kept, T):
    """Probabilities of a row over the kept indices."""
    p = np.zeros(len(l))
    kept = np.asarray(kept)
    if T == 0:
        p[kept[0]] = 1.0
        return p
    x = (l[kept] - l[kept].max()) / T
    p[kept] = np.exp(x) / np.exp(x).sum()
    return p


def verdict(P, Q, x, u, u_draw, eos=-1):
    """P, Q [k, V] (Q None: certain drafts): n_acc, token, finished, ratios, ln p(token),
    and how far the decisions were from going the other way."""
    k = len(x)
    ratio, margin = np.zeros(k), np.inf
    for i in range(k):
        if x[i] >= 0 and x[i] < P.shape[1]:
            q = 1.0 if Q is None else Q[i, x[i]]
            ratio[i] = min(1.0, P[i, x[i]] / q) if q > 0 else float(P[i, x[i]] > 0)
    n = 0
    for i in range(k):
        if x[i] < 0:
            w = P[i]
            break
        inside = x[i] < P.shape[1]
        p, q = (P[i, x[i]] if inside else 0.0), (1.0 if Q is None else Q[i, x[i]] if inside else 0.0)
        margin = min(margin, abs(u[i] * q - p) / max(p, q, 1e-300))
        if not u[i] * q < p:
            w = np.maximum(P[i] - (Q[i] if Q is not None else (np.arange(P.shape[1]) == x[i]) * 2.0), 0.0)
            if not w.sum() > 0:
                w = P[i]
            break
        n += 1
        if x[i] == eos:
            return n, -1, 1, ratio, np.nan, margin
    else:
        return n, -1, 0, ratio, np.nan, margin
    c = np.cumsum(w) / w.sum()
    token = int(np.argmax(c > u_draw)) if (c > u_draw).any() else int(np.nonzero(w)[0][-1])
    margin = min(margin, np.abs(c - u_draw).min())
    return n, token, int(token == eos), ratio, math.log(P[n, token]), margin
