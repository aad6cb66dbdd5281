"""Attention with modified scores, the weights that it gives, the verdict on drafts and
eviction, together as a serving loop calls them: step after step over one cache, on a
stream of its own, and from captured graphs."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests import masked_reference as ref
from tests.masked_reference import BF16, F32, Batch, check_attention, f64, limits
from tests.test_gpu_drafts import call, check, rows
from tests.test_gpu_mass_evict import appended, check_evict, check_mass, dev, evicted, masses


def bits(t):
    return t.cpu().view(torch.int16 if t.element_size() == 2 else torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("ps", [16, 64])
@pytest.mark.parametrize("longest", [1, 16, 17])
@pytest.mark.parametrize("ranged", [False, True])
def test_the_window_is_appended_whoever_sees_it(dt, ps, longest, ranged):
    """Every window row's key and value lie in its slot afterwards, all other slots are as they
    were: windows that cross pages, and ranges that leave out the window or all keys."""
    k = lambda n: min(n, longest)  # noqa: E731
    b = Batch([(0, k(16)), (15, k(17)), (31, k(2)), (63, k(17)), (7, 0), (1500, k(9))], 8, 2, 64, ps, dt, seed=longest)
    kw = {}
    if ranged:
        p = np.concatenate([b.ctx[i] + np.arange(n) for i, n in enumerate(b.k)])
        end = np.minimum(p + 1, 5 * (np.arange(b.T) % 3))           # 0, 5 or 10 keys
        kw = dict(end_key=dev(end))
    kx, vx = b.kc.cpu(), b.vc.cpu()
    for i, L in enumerate(b.ctx):
        for j in range(int(b.k[i])):
            page, slot, r = int(b.table[i, (L + j) // ps]), (L + j) % ps, int(b.cu[i]) + j
            kx[page, :, :, slot, :] = b.k_new[r].view(2, -1, 32)
            vx[page, :, :, slot] = b.v_new[r]
    ops.verify_attn_masked(b.q.cuda(), b.k_new.cuda(), b.v_new.cuda(), b.kc, b.vc, *b.args, **kw)
    assert torch.equal(bits(b.kc), bits(kx)) and torch.equal(bits(b.vc), bits(vx))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mod", [dict(), dict(window=70, softcap=9.0), dict(slopes=True), dict(first=True)])
def test_masses_of_many_rows(dt, D, mod):
    """Rows enough for workgroups that share a block of keys."""
    b = Batch([(0, 170), (90, 131), (31, 3), (400, 1), (5, 0)], 16, 2, D, 16, dt, seed=D)
    mod, first = dict(mod), None
    if mod.pop("slopes", False):
        mod["slopes"] = dev(2.0 ** -np.arange(1.0, 17), np.float32)
    if mod.pop("first", False):
        first = np.concatenate([b.ctx[i] + np.arange(n) for i, n in enumerate(b.k)]) // 50 * 50
    kw = dict(mod, first_key=dev(first))
    lse = appended(b, **kw)
    m = masses(b)
    got = ops.attn_mass(b.q.cuda(), b.kc, lse, *b.args, mass=m.cuda(), decay=0.75, **kw)
    check_mass(b, got, lse, m, 0.75, mod, first=first)


@pytest.mark.gpu
@pytest.mark.parametrize("D,ps,Hq,Hkv", [(64, 16, 8, 1), (128, 64, 8, 4), (128, 16, 3, 3)])
@pytest.mark.parametrize("k", [1, 2])
@pytest.mark.parametrize("mod", [dict(), dict(window=77), dict(softcap=6.0, first=True)])
def test_few_rows_over_short_contexts(D, ps, Hq, Hkv, k, mod):
    """Walks left whole by eight waves: lengths around their blocks, and a value that is not finite
    among the keys, which the rows that see it get and no others."""
    b = Batch([(n, k) for n in (0, 1, 31, 32, 33, 255, 257, 700, 1016)], Hq, Hkv, D, ps, BF16, seed=D + k)
    p = np.concatenate([b.ctx[i] + np.arange(k) for i in range(len(b.ctx))])
    mod, first = dict(mod), None
    if mod.pop("first", False):
        first = p // 300 * 300
    lo = np.broadcast_to(limits(p, 1, mod.get("window", 0), first, p + 1)[0], p.shape)
    out, lse = ops.verify_attn_masked(b.q.cuda(), b.k_new.cuda(), b.v_new.cuda(), b.kc, b.vc, *b.args, lse=True,
                                      first_key=dev(first), **mod)
    for bad in (False, True):
        if bad:                                  # of the last two sequences
            for i, at in ((7, 600), (8, 950)):
                b.vc[int(b.table[i, at // ps]), 0, 5, at % ps] = float("nan")
            out, lse = ops.verify_attn_masked(b.q.cuda(), None, None, b.kc, b.vc, *b.args, lse=True, first_key=dev(first), **mod)
        for i, L in enumerate(b.ctx):
            r, V = b.rows(i), b.V[i].copy()
            if bad and i >= 7:
                at = 600 if i == 7 else 950
                V[at, 0, 5] = 0.0                # in place of it, in rows that do not see it
                seen = lo[r] <= at
                G = Hq // Hkv
                got = f64(out[r])
                assert np.isnan(got[seen][:, :G, 5]).all()
                got[seen, :G, 5] = 0.0
                assert np.isfinite(got).all()
                if seen.any():
                    continue
            f = None if first is None else first[r]
            want = ref.attention(f64(b.q[r]), b.K[i], V, int(L), b.scale, *limits(int(L), k, mod.get("window", 0), f),
                                 mod.get("softcap", 0.0))
            check_attention(out[r], lse[r], want, BF16, int(L) + k, k * Hq // Hkv > 16)


class Loop:
    """Four sequences of a cache whose pages hold NaN until they are written."""
    CAP, SINK, RECENT = 15.0, 2, 6

    def __init__(self, dt, Hq=8, Hkv=2, D=64, ps=16, seed=0):
        self.dt, self.Hq, self.Hkv, self.D, self.ps, self.B, self.width = dt, Hq, Hkv, D, ps, 4, 6
        self.rng, self.g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        pages = self.rng.permutation(2 * self.B * self.width + 3).astype(np.int32)
        self.tables = [pages[i * self.B * self.width:][: self.B * self.width].reshape(self.B, -1) for i in (0, 1)]
        P, nan = len(pages), float("nan")
        self.kc = torch.full((P, Hkv, D // 32, ps, 32), nan, dtype=dt).cuda()
        self.vc = torch.full((P, Hkv, D, ps), nan, dtype=dt).cuda()
        self.mass = torch.zeros(P, Hkv, ps).cuda()
        self.side = np.zeros(self.B, np.int64)              # which of its two tables a sequence lives in
        self.ctx = np.array([0, 7, 40, 70], np.int32)
        self.limit, self.keep = 72, 33
        rand = lambda *s: torch.randn(*s, generator=self.g).to(dt)  # noqa: E731
        for b, L in enumerate(self.ctx):
            k, v = rand(int(L), Hkv, D), rand(int(L), Hkv, D)
            for p in range(int(L)):
                page = self.tables[0][b, p // ps]
                self.kc[page, :, :, p % ps, :] = k[p].view(Hkv, -1, 32).cuda()
                self.vc[page, :, :, p % ps] = v[p].cuda()

    def table(self):
        return np.stack([self.tables[s][b] for b, s in enumerate(self.side)])

    def window(self, T):
        rand = lambda *s: torch.randn(*s, generator=self.g).to(self.dt)  # noqa: E731
        return rand(T, self.Hq, self.D), rand(T, self.Hkv, self.D), rand(T, self.Hkv, self.D)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_a_serving_loop(dt):
    """Windows of drafts, their weights into the masses, the verdict, and eviction of what has
    grown too long into the sequence's other pages; each call against the plain form of the
    state that it was given."""
    s, evictions, V = Loop(dt, seed=3), 0, 211
    for step in range(60):
        if step > 8 and evictions > 1:
            break
        k = s.rng.integers(0, 6, s.B)
        cu = np.concatenate([[0], np.cumsum(k)]).astype(np.int32)
        T, table = int(cu[-1]), s.table()
        if T == 0:
            continue
        q, kn, vn = s.window(T)
        args = dev(table), dev(s.ctx), dev(cu), int(k.max())
        out, lse = ops.verify_attn_masked(q.cuda(), kn.cuda(), vn.cuda(), s.kc, s.vc, *args, lse=True, softcap=s.CAP, validate=True)
        before = s.mass.cpu()
        ops.attn_mass(q.cuda(), s.kc, lse, *args, mass=s.mass, decay=0.9, softcap=s.CAP)
        kh, vh, mh = s.kc.cpu(), s.vc.cpu(), f64(s.mass)
        want_mass, err = f64(before), np.zeros(mh.shape)
        for b, L in enumerate(s.ctx):
            r, n = slice(int(cu[b]), int(cu[b + 1])), int(L + k[b])
            if k[b] == 0:
                continue
            p = np.arange(n)
            K, W = (f64(x) for x in (kh[table[b, p // s.ps], :, :, p % s.ps, :].flatten(2), vh[table[b, p // s.ps], :, :, p % s.ps]))
            assert np.array_equal(K[L:], f64(kn[r])) and np.array_equal(W[L:], f64(vn[r]))
            lo, hi = limits(int(L), int(k[b]))
            want = ref.attention(f64(q[r]), K, W, int(L), s.D ** -0.5, lo, hi, s.CAP)
            check_attention(out[r], lse[r], want, dt, n, dt == BF16 and int(k.max()) * 4 > 16)
            w, e = ref.weights(f64(q[r]), K, f64(lse[r]), int(L), s.D ** -0.5, lo, hi, s.CAP)
            for j in range(n):
                at = int(table[b, j // s.ps]), slice(None), j % s.ps
                want_mass[at] = (0.9 * want_mass[at] if j < L else 0.0) + w[j]
                err[at] = e[j] + 2.0 ** -23 * want_mass[at]
        # a sequence without rows keeps its masses times the decay
        for b in np.nonzero(k == 0)[0]:
            for j in range(int(s.ctx[b])):
                at = int(table[b, j // s.ps]), slice(None), j % s.ps
                want_mass[at] *= 0.9
                err[at] = 2.0 ** -23 * want_mass[at]
        assert (np.abs(mh - want_mass) <= err).all()
        t, d, g = rows(step, T, V, dt)
        x = np.array([int(i) for i in f64(d).argmax(1)])
        x[cu[1:][k > 0] - 1] = -1                    # the row behind the drafts
        u, ud = torch.rand(T, generator=g).numpy(), torch.rand(s.B, generator=g).numpy()
        got = call(t, d, x, cu, u, ud)
        assert check(t, d, {}, {}, x, cu, u, ud, got) >= s.B - 1
        s.ctx = (s.ctx + np.where(k > 0, got["n_acc"].cpu().numpy() + 1, 0)).astype(np.int32)
        long = np.nonzero(s.ctx > s.limit)[0].astype(np.int32)
        if len(long) == 0:
            continue
        other = np.stack([s.tables[1 - i][b] for b, i in enumerate(s.side)])
        keep = np.full(s.B, s.keep)
        state = s.kc.cpu(), s.vc.cpu(), s.mass.cpu()
        new, kept = ops.kv_evict(s.kc, s.vc, s.mass, dev(table), dev(other), dev(s.ctx), dev(keep), s.SINK, s.RECENT,
                                 seq_ids=dev(long), validate=True)
        view = SimpleNamespace(kc=s.kc, vc=s.vc, ps=s.ps, ctx=s.ctx, Hkv=s.Hkv, table=table)
        check_evict(view, other, state, keep, s.SINK, s.RECENT, new, kept, s.mass, seqs=long)
        s.ctx[long], s.side[long] = new.cpu().numpy()[long], 1 - s.side[long]
        evictions += len(long)
    assert evictions >= 2


class Step:
    """One window of every operator, its inputs and outputs in tensors that stay."""

    def __init__(self, dt, seed, windows, mod):
        b = self.b = Batch(windows, 8, 2, 64, 16, dt, seed=seed, extra=40)
        self.mod = dict(mod)
        V, T, B = 3001, b.T, len(windows)
        t, d, g = rows(seed, T, V, dt)
        self.t, self.d = t.cuda(), d.cuda()
        self.x, self.u = dev(f64(d).argmax(1)), torch.rand(T, generator=g).cuda()
        self.ud, self.f = torch.rand(B, generator=g).cuda(), dict(top_p=torch.full((T,), 0.9).cuda())
        self.q, self.kn, self.vn = b.q.cuda(), b.k_new.cuda(), b.v_new.cuda()
        self.mass0, self.mass = masses(b, seed).cuda(), torch.empty(b.kc.shape[0], 2, 16, device="cuda")
        self.dst = dev(b.free[: 8 * B].reshape(B, 8)) if len(b.free) >= 8 * B else None
        self.keep = dev(np.full(B, 30))
        self.ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (
            ops.attn_masked_workspace_size(B, 8, 2, 64, b.max_q, b.table.shape[1], 16),
            ops.verify_drafts_workspace_size(T, V, B, True, False))]
        self.k0, self.v0 = b.kc.clone(), b.vc.clone()

    def run(self):
        b = self.b
        b.kc.copy_(self.k0)
        b.vc.copy_(self.v0)
        self.mass.copy_(self.mass0)
        self.out, self.lse = ops.verify_attn_masked(self.q, self.kn, self.vn, b.kc, b.vc, *b.args, lse=True, workspace=self.ws[0],
                                                    **self.mod)
        ops.attn_mass(self.q, b.kc, self.lse, *b.args, mass=self.mass, decay=0.5, **self.mod)
        self.v = ops.verify_drafts(self.t, self.d, self.x, b.args[2], self.u, self.ud, workspace=self.ws[1], **self.f)
        self.e = ops.kv_evict(b.kc, b.vc, self.mass, b.args[0], self.dst, b.args[1], self.keep, 1, 4)

    def state(self):
        return [t.clone() for t in (self.out, self.lse, self.mass, self.b.kc, self.b.vc, *self.v.values(), *self.e)]


def same(got, want):
    return all(torch.equal(bits(x) if x.dtype in (BF16, F32) else x.cpu(), bits(y) if y.dtype in (BF16, F32) else y.cpu())
               for x, y in zip(got, want))


STEPS = [(BF16, 1, [(700, 4), (90, 1), (0, 3)], dict(softcap=20.0)), (F32, 2, [(33, 20), (1200, 2), (64, 1)], dict(window=90))]


@pytest.mark.gpu
def test_two_captured_steps_in_turn():
    """Each replay gives the bits of the eager call, with the other graph's replays, eager calls of
    either and synchronizations in between."""
    steps = [Step(*a) for a in STEPS]
    want = []
    for s in steps:
        s.run()
        want.append(s.state())
    assert all(int((w[2] != s.mass0).sum()) for s, w in zip(steps, want))
    side = torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph() for _ in steps]
    for s, g in zip(steps, graphs):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.run()
        torch.cuda.current_stream().wait_stream(side)
        with torch.cuda.graph(g):
            s.run()
    held = [(s.out, s.lse, s.mass, s.b.kc, s.b.vc, *s.v.values(), *s.e) for s in steps]

    def replay(i):
        for t in (*held[i][:3], *held[i][5:]):
            t.fill_(0)
        graphs[i].replay()

    for _ in range(3):
        for i in (0, 1):
            replay(i)
            torch.cuda.synchronize()
            assert same(held[i], want[i])
        replay(1)
        replay(0)
        assert same(held[0], want[0]) and same(held[1], want[1])
        other = Step(*STEPS[0])
        other.run()
        assert same(other.state(), want[0])


@pytest.mark.gpu
def test_a_stream_of_its_own():
    """All four on a stream that is not the default one, behind inputs that it writes itself."""
    s = Step(*STEPS[0])
    s.run()
    want, q = s.state(), s.q.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s.q.zero_()
        torch.empty(1 << 28, dtype=torch.uint8, device="cuda").fill_(1)
        s.q.copy_(q)
        s.run()
        got = s.state()
    side.synchronize()
    assert same(got, want)


@pytest.mark.gpu
def test_a_shared_workspace_holds_nothing_between_calls():
    """Two steps of different sizes, one workspace each call kind: what the other left is not read."""
    a, c = Step(*STEPS[0]), Step(*STEPS[1])
    a.run(), c.run()
    want = a.state(), c.state()
    ws = [torch.empty(max(x.numel(), y.numel()), dtype=torch.uint8, device="cuda") for x, y in zip(a.ws, c.ws)]
    a.ws = c.ws = ws
    for fill in (0, 255):
        for w in ws:
            w.fill_(fill)
        for s, state in ((a, want[0]), (c, want[1]), (a, want[0])):
            s.run()
            assert same(s.state(), state)


# --- the largest tables and bounds ---

@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("max_q", [9, 200])
def test_masses_under_a_table_of_the_largest_width(dt, max_q):
    """2^22 positions: more blocks of keys than a grid's second dimension holds."""
    b = Batch([(900, 9), (5, 3)], 16, 2, 64, 64, dt, seed=6)
    lse = appended(b)
    m = masses(b)
    pt, ctx, cu, _ = b.args
    wide = torch.full((2, (1 << 22) // 64 - 4), -1, dtype=torch.int32).cuda()
    wide[:, : pt.shape[1]] = pt
    got = ops.attn_mass(b.q.cuda(), b.kc, lse, wide, ctx, cu, max_q, mass=m.cuda(), decay=0.5)
    check_mass(b, got, lse, m, 0.5, {})


@pytest.mark.gpu
def test_attention_under_a_loose_bound_of_windows():
    """A max_q of 2^17, 2^20 rows per KV head: half of what a call may have."""
    b = Batch([(900, 2), (5, 9)], 8, 1, 64, 16, BF16, seed=3)
    want, lse0 = ops.verify_attn_masked(b.q.cuda(), b.k_new.cuda(), b.v_new.cuda(), b.kc, b.vc, *b.args, lse=True, window=700)
    pt, ctx, cu, _ = b.args
    wide = torch.full((2, 5000), -1, dtype=torch.int32).cuda()
    wide[:, : pt.shape[1]] = pt
    out, lse = ops.verify_attn_masked(b.q.cuda(), None, None, b.kc, b.vc, wide, ctx, cu, 1 << 17, lse=True, window=700,
                                      seq_ids=torch.tensor([1, 0], dtype=torch.int32).cuda())
    for i, L in enumerate(b.ctx):
        r, n = b.rows(i), int(b.k[i])
        x = ref.attention(f64(b.q[r]), b.K[i], b.V[i], int(L), b.scale, *limits(int(L), n, 700))
        check_attention(out[r], lse[r], x, BF16, int(L) + n, True)
        check_attention(want[r], lse0[r], x, BF16, int(L) + n, b.max_q * 8 > 16)


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,ps", [(8, 16), (8, 32), (16, 16), (16, 64)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [False, True])
def test_windows_under_tables_of_more_than_the_caches_hold(Hq, ps, D, bad):
    """Windows of one tile, whose keys are loaded as a stream, the window's own among them; a value that
    is not finite stays with the rows that see it."""
    b = Batch([(900, 2), (5, 9), (3000, 8), (31, 1)], Hq, 2, D, ps, BF16, seed=Hq + D)
    if bad:
        b.v_new[3, 0, 7] = float("nan")          # of the second window, seen from its second row on
        b.V[1][5 + 1, 0, 7] = 0.0
    pt, ctx, cu, _ = b.args
    wide = torch.full((4, 1200000 // ps), -1, dtype=torch.int32).cuda()
    wide[:, : pt.shape[1]] = pt
    out, lse = ops.verify_attn_masked(b.q.cuda(), b.k_new.cuda(), b.v_new.cuda(), b.kc, b.vc, wide, ctx, cu, 9, lse=True, softcap=20.0)
    for i, L in enumerate(b.ctx):
        r, n = b.rows(i), int(b.k[i])
        if bad and i == 1:
            got = f64(out[r])
            assert np.isnan(got[1:, : Hq // 2, 7]).all() and np.isfinite(got[0]).all()
            got[1:, : Hq // 2, 7] = 0.0
            assert np.isfinite(got).all()
            continue
        want = ref.attention(f64(b.q[r]), b.K[i], b.V[i], int(L), b.scale, *limits(int(L), n), 20.0)
        check_attention(out[r], lse[r], want, BF16, int(L) + n, True)


@pytest.mark.gpu
def test_eviction_under_tables_of_the_largest_width():
    b, table, dst, dkeep = evicted([300], [130], 2, 64, 64, BF16, 3, [130])
    m = masses(b, 5)
    before = b.kc.cpu(), b.vc.cpu(), m.clone()
    mass = m.cuda()
    wide = lambda t: torch.cat([t, torch.full((1, (1 << 22) // 64 - t.shape[1]), -1, dtype=torch.int32).cuda()], 1)  # noqa: E731
    new, kept = ops.kv_evict(b.kc, b.vc, mass, wide(b.args[0]), wide(dst), b.args[1], dkeep, 4, 64)
    assert (kept[0, :, 130:] == -1).all()
    slots = table.shape[1] * 64
    check_evict(b, table, before, [130], 4, 64, new, kept[:, :, :slots], mass)


def test_batches_too_large_for_a_launch_are_refused():
    size = ops.verify_drafts_workspace_size
    assert size(0, 262144, 1 << 16) > 0 and size(0, 262144, 1 << 17) == 0
