"""The 8-bit cache: append, read-back and attention against 64-bit plain forms,
and their refusals."""
import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests import q8_reference as ref

BF16, F32 = torch.bfloat16, torch.float32


def f64(t):
    return t.detach().float().cpu().double().numpy()


def pool(windows, Hkv, D, ps, seed=0, extra=3, total=0, fill=None):
    """A cache whose slots hold NaN bytes and NaN scales until written, and the batch's arrays.  `total`: pages at least."""
    rng = np.random.default_rng(seed)
    ctx = np.array([w[0] for w in windows], np.int32)
    cu = np.concatenate([[0], np.cumsum([w[1] for w in windows])]).astype(np.int32)
    need = -(-(ctx + np.diff(cu)) // ps)
    P = max(int(need.sum()) + extra, total)
    ids = rng.permutation(int(need.sum()) + extra) + (P - int(need.sum()) - extra)     # the pool's last pages
    table = np.full((len(windows), max(1, int(need.max()))), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at: at + n]
        at += n
    c = ops.Q8Cache.empty(P, Hkv, D, ps)
    c.k.view(torch.uint8).fill_(0x7F)
    c.v.view(torch.uint8).fill_(0xFF)
    c.scale.fill_(255)
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    return c, table, ctx, cu, dev(table), dev(ctx), dev(cu)


def rows_of(windows, H, D, dt, seed):
    T = sum(w[1] for w in windows)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, H, D, generator=g) * torch.exp(3 * torch.randn(T, H, 1, generator=g))
    return x.to(dt)


def host(c):
    return c.k.cpu(), c.v.cpu(), c.scale.cpu()


def fill(c, table, ctx, cu, page_table, seed, dt=BF16, spread=1.0):
    """Writes every position of every sequence, as one window over an empty cache; returns the float64 values per sequence."""
    n = (ctx + np.diff(cu)).astype(np.int32)
    cu_all = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    g = torch.Generator().manual_seed(seed)
    T = int(cu_all[-1])
    k = (spread * torch.randn(T, c.Hkv, c.D, generator=g)).to(dt)
    v = torch.randn(T, c.Hkv, c.D, generator=g).to(dt)
    ops.kv_append_q8(k.cuda(), v.cuda(), c, page_table, torch.zeros(len(n), dtype=torch.int32).cuda(),
                     torch.from_numpy(cu_all).cuda(), int(max(1, n.max())))
    kq, vq = ref.quantise(f64(k))[0], ref.quantise(f64(v))[0]
    return [(kq[a:b], vq[a:b]) for a, b in zip(cu_all[:-1], cu_all[1:])]


RAGGED = [(0, 1), (5, 0), (15, 2), (16, 16), (3, 40), (100, 13), (31, 33)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("Hkv,D,ps", [(1, 64, 16), (3, 128, 32), (2, 128, 16), (5, 64, 64)])
def test_append_writes_the_rows_and_nothing_else(dt, Hkv, D, ps):
    c, table, ctx, cu, pt, dctx, dcu = pool(RAGGED, Hkv, D, ps)
    k, v = rows_of(RAGGED, Hkv, D, dt, 1), rows_of(RAGGED, Hkv, D, dt, 2)
    k[0] = 0.0                                              # a row of zeros
    v[1, 0] = torch.arange(D) % 2 * 1e-39                   # subnormal: the least exponent
    k[2, 0, 3], v[3, 0, 5], k[4, 0, 0] = float("inf"), float("nan"), -float("inf")
    k[5, 0] = 448.0                                         # the largest that needs no scale
    v[5, 0] = 450.0
    before = [t.view(torch.uint8).clone() for t in (c.k, c.v, c.scale)]
    ops.kv_append_q8(k.cuda(), v.cuda(), c, pt, dctx, dcu, 40)
    kh, vh, sh = host(c)
    (kq, ke), (vq, ve) = ref.quantise(f64(k)), ref.quantise(f64(v))
    b_k, b_v, b_s = (t.cpu() for t in before)
    for r, b, pos, page, slot in ref.slots(table, ctx, cu, range(len(ctx)), ps):
        gk, gv = ref.cached(kh, vh, sh, page, slot)
        assert np.array_equal(gk, kq[r], equal_nan=True) and np.array_equal(gv, vq[r], equal_nan=True)
        assert np.array_equal(sh[page, :, 0, slot].numpy(), ke[r]) and np.array_equal(sh[page, :, 1, slot].numpy(), ve[r])
        b_k[page, :, :, slot, :] = kh.view(torch.uint8)[page, :, :, slot, :]
        b_v[page, :, :, slot] = vh.view(torch.uint8)[page, :, :, slot]
        b_s[page, :, :, slot] = sh[page, :, :, slot]
    assert torch.equal(b_k, kh.view(torch.uint8)) and torch.equal(b_v, vh.view(torch.uint8)) and torch.equal(b_s, sh)
    # read back: exact, in either type
    for t in (BF16, F32):
        rk, rv = ops.kv_read_q8(c, pt, dctx, dcu, 40, k.shape[0], dtype=t)
        tiny = np.abs(vq) < 2.0 ** -126                     # below bf16's normal range a value is rounded
        assert np.array_equal(f64(rk), kq, equal_nan=True)
        assert np.array_equal(np.where(tiny, 0, f64(rv)), np.where(tiny, 0, vq), equal_nan=True)


@pytest.mark.gpu
def test_append_and_read_of_some_sequences_and_strided_rows():
    c, table, ctx, cu, pt, dctx, dcu = pool(RAGGED, 2, 64, 16)
    T = int(cu[-1])
    wide = torch.randn(T + 3, 8 * 64, generator=torch.Generator().manual_seed(4)).cuda()
    k, v = wide[:, 128:256].view(-1, 2, 64), wide[:, 256:384].view(-1, 2, 64)
    some = torch.tensor([5, 2, 3], dtype=torch.int32).cuda()
    ops.kv_append_q8(k, v, c, pt, dctx, dcu, 16, seq_ids=some)
    kh, vh, sh = host(c)
    kq, vq = ref.quantise(f64(k))[0], ref.quantise(f64(v))[0]
    for r, b, pos, page, slot in ref.slots(table, ctx, cu, range(len(ctx)), 16):
        gk, gv = ref.cached(kh, vh, sh, page, slot)
        if b in (5, 2, 3):
            assert np.array_equal(gk, kq[r]) and np.array_equal(gv, vq[r])
        else:
            assert (sh[page, :, :, slot] == 255).all()
    ko = torch.full((T + 3, 2, 64), 7.0, device="cuda")
    vo = ko.clone()
    ops.kv_read_q8(c, pt, dctx, dcu, 16, T + 3, seq_ids=some, dtype=F32, k_out=ko, v_out=vo)
    live = np.zeros(T + 3, bool)
    for b in (5, 2, 3):
        live[cu[b]: cu[b + 1]] = True
    assert np.array_equal(f64(ko)[live], kq[live]) and np.array_equal(f64(vo)[live], vq[live])
    assert (f64(ko)[~live] == 7).all() and (f64(vo)[~live] == 7).all()


def check_rows(got, want, dt):
    """bf16: half a step of the result, and the probabilities' rounding, half
    a step each: an error of at most 2^-8 of sum p |V|, whose size over a row is
    taken as three times the row's rms (it is below one rms where many keys share
    the mass).  fp32: products exact, sums of at most 2^14 terms in fp32."""
    rms = np.sqrt((want ** 2).mean(-1, keepdims=True))
    half = torch.finfo(dt).eps / 2
    tol = half * np.abs(want) + (3 * half if dt == BF16 else 2.0 ** -17) * rms
    off = np.abs(f64(got) - want)
    print("worst", (off / tol).max(), flush=True)
    assert (off <= tol).all()
    if dt == BF16:
        assert (np.linalg.norm(f64(got) - want, axis=-1) <= 1e-2 * np.linalg.norm(want, axis=-1)).all()


ATTN = [
    # heads, D, page, windows (context, rows)
    (4, 2, 64, 16, [(0, 1), (1, 1), (63, 1), (64, 1), (65, 1), (300, 1)]),          # one 16-row tile
    (16, 8, 128, 16, [(0, 1), (5, 0), (2000, 1), (17, 1)]),
    (32, 4, 128, 32, [(100, 4), (0, 3), (777, 4)]),                                 # two tiles
    (32, 4, 128, 16, [(1000, 8), (3, 5), (0, 8), (129, 1), (40, 0)]),               # four
    (16, 4, 64, 64, [(500, 30), (0, 17), (77, 32)]),                                # two row groups
    (32, 4, 128, 16, [(0, 150), (33, 64), (0, 1)]),                                 # four row groups, two items
    (3, 3, 64, 16, [(0, 200), (10, 129)]),                                          # one head per KV head
    (5, 1, 128, 64, [(700, 7)]),
    (32, 1, 64, 16, [(250, 3), (0, 4)]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("Hq,Hkv,D,ps,windows", ATTN)
def test_attention_matches_the_plain_form(dt, Hq, Hkv, D, ps, windows):
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, Hkv, D, ps)
    kv = fill(c, table, ctx, cu, pt, 5)
    g = torch.Generator().manual_seed(6)
    q = (2 * torch.randn(int(cu[-1]), Hq, D, generator=g)).to(dt)
    out = torch.full_like(q, float("nan"), device="cuda")
    ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, int(np.diff(cu).max()), out=out, scale=0.3 / D ** 0.5)
    for b, (K, V) in enumerate(kv):
        if cu[b + 1] > cu[b]:
            want = ref.attention(f64(q[cu[b]: cu[b + 1]]), K, V, int(ctx[b]), 0.3 / D ** 0.5)
            check_rows(out[cu[b]: cu[b + 1]], want, dt)
    # the same call repeats bit for bit, and a window bound above the need changes no more than the order of sums
    again = ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, int(np.diff(cu).max()), scale=0.3 / D ** 0.5)
    assert torch.equal(out, again)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_attention_of_large_scores_and_values(dt):
    """Scores of hundreds (one key takes the mass) and values of 1e30."""
    windows = [(400, 3), (0, 2)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, 2, 64, 16)
    n = (ctx + np.diff(cu)).astype(np.int32)
    g = torch.Generator().manual_seed(8)
    k = (8 * torch.randn(int(n.sum()), 2, 64, generator=g)).to(dt)
    v = (1e30 * torch.randn(int(n.sum()), 2, 64, generator=g)).to(dt)
    cu_all = torch.tensor([0, n[0], n.sum()], dtype=torch.int32).cuda()
    ops.kv_append_q8(k.cuda(), v.cuda(), c, pt, torch.zeros(2, dtype=torch.int32).cuda(), cu_all, int(n.max()))
    kq, vq = ref.quantise(f64(k))[0], ref.quantise(f64(v))[0]
    q = (8 * torch.randn(5, 4, 64, generator=g)).to(dt)
    out = ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, 3)
    want = ref.attention(f64(q[:3]), kq[: n[0]], vq[: n[0]], 400, 0.125)
    # a score of 500 is off by 500 * 2^-22 in fp32, a probability by as much of itself
    off = np.abs(f64(out[:3]) - want) / np.sqrt((want ** 2).mean(-1, keepdims=True))
    assert off.max() < (4 * 2.0 ** -9 * 3 if dt == BF16 else 2e-3)


@pytest.mark.gpu
def test_nan_rows_reach_only_the_rows_that_see_them():
    """A window token with a NaN value, another with an infinite key: rows before
    them are as without, rows that see them are NaN; the slots behind stay NaN."""
    windows = [(70, 6), (20, 3)]
    for key in (False, True):
        c, table, ctx, cu, pt, dctx, dcu = pool(windows, 2, 64, 16)
        kv = fill(c, table, ctx, cu, pt, 9)
        k, v = rows_of(windows, 2, 64, BF16, 3), rows_of(windows, 2, 64, BF16, 4)
        (k if key else v)[3, 1, 7] = float("inf") if key else float("nan")
        ops.kv_append_q8(k.cuda(), v.cuda(), c, pt, dctx, dcu, 6)
        q = torch.randn(9, 4, 64, generator=torch.Generator().manual_seed(2)).to(BF16)
        out = f64(ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, 6))
        nan = np.isnan(out)
        assert nan[3:6, 2:].all() and not nan[:3].any() and not nan[:6, :2].any() and not nan[6:].any()
        K, V = kv[0][0].copy(), kv[0][1].copy()
        K[70:76], V[70:76] = ref.quantise(f64(k[:6]))[0], ref.quantise(f64(v[:6]))[0]
        want = ref.attention(f64(q[:3]), K[:73], V[:73], 70, 0.125)
        check_rows(torch.from_numpy(out[:3]), want, BF16)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """Pages whose bytes lie beyond 2^32 of the pool's start."""
    windows = [(90, 2), (0, 20)]
    Hkv, D, ps = 8, 128, 64
    total = (1 << 32) // (Hkv * D * ps) + 40
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, Hkv, D, ps, total=total)
    assert (table[table >= 0].astype(np.int64) * Hkv * D * ps > 2 ** 32).all()
    kv = fill(c, table, ctx, cu, pt, 5)
    q = torch.randn(22, 8, D, generator=torch.Generator().manual_seed(6)).to(BF16)
    out = ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, 20)
    for b, (K, V) in enumerate(kv):
        check_rows(out[cu[b]: cu[b + 1]], ref.attention(f64(q[cu[b]: cu[b + 1]]), K, V, int(ctx[b]), D ** -0.5), BF16)
    rk, _ = ops.kv_read_q8(c, pt, dctx, dcu, 20, 22, dtype=F32)
    assert np.array_equal(f64(rk[:2]), kv[0][0][90:])


@pytest.mark.gpu
def test_many_sequences_some_handled_strided_queries():
    """More sequences than threads of a workgroup; every third is handled."""
    rng = np.random.default_rng(0)
    windows = [(int(rng.integers(0, 90)), int(rng.integers(0, 4))) for _ in range(700)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, 1, 64, 16)
    kv = fill(c, table, ctx, cu, pt, 5)
    ids = rng.permutation(700)[:233].astype(np.int32)
    wide = torch.randn(int(cu[-1]), 3, 2, 64, generator=torch.Generator().manual_seed(6)).to(BF16)
    q = wide.cuda()[:, 1]
    out = torch.full((int(cu[-1]), 2, 64), 7.0, dtype=BF16, device="cuda")
    ops.verify_attn_q8(q, c, pt, dctx, dcu, 3, seq_ids=torch.from_numpy(ids).cuda(), out=out)
    handled = set(ids.tolist())
    for b, (K, V) in enumerate(kv):
        o = out[cu[b]: cu[b + 1]]
        if b in handled:
            if len(o):
                check_rows(o, ref.attention(f64(wide[cu[b]: cu[b + 1], 1]), K, V, int(ctx[b]), 0.125), BF16)
        else:
            assert (o == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("heads,longest", [((16, 4), 320), ((16, 16), 200), ((15, 5), 260)])
def test_prompts_of_many_lengths(dt, heads, longest):
    """Enough work for every workgroup, in row groups of very different lengths; every second prompt in another order."""
    rng = np.random.default_rng(longest)
    windows = [(0, int(n)) for n in rng.integers(1, longest, 36)] + [(0, 0), (0, longest), (17, 3), (0, longest)]
    Hq, Hkv = heads
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, Hkv, 64, 16)
    kv = fill(c, table, ctx, cu, pt, 5)
    q = torch.randn(int(cu[-1]), Hq, 64, generator=torch.Generator().manual_seed(6)).to(dt)
    ids = rng.permutation(len(windows)).astype(np.int32)
    for some in (ids, ids[:29]):
        out = torch.full((int(cu[-1]), Hq, 64), 7.0, dtype=dt, device="cuda")
        ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, longest, seq_ids=torch.from_numpy(some).cuda(), out=out)
        for b, (K, V) in enumerate(kv):
            o = out[cu[b]: cu[b + 1]]
            if b not in some:
                assert (o == 7).all()
            elif len(o) and (some is ids or b % 4 == 0):
                check_rows(o, ref.attention(f64(q[cu[b]: cu[b + 1]]), K, V, int(ctx[b]), 0.125), dt)


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,most", [(1, 1, 5), (8, 1, 7), (16, 1, 11)])
def test_more_sequences_than_are_kept_in_lds(Hq, Hkv, most):
    rng = np.random.default_rng(most)
    windows = [(int(rng.integers(0, 60)), int(rng.integers(0, most))) for _ in range(1500)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, Hkv, 64, 16)
    kv = fill(c, table, ctx, cu, pt, 5)
    q = torch.randn(int(cu[-1]), Hq, 64, generator=torch.Generator().manual_seed(6)).to(BF16)
    out = torch.full_like(q, float("nan"), device="cuda")
    ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, most, out=out)
    want = [ref.attention(f64(q[a:b]), K, V, int(L), 0.125) for a, b, (K, V), L in zip(cu[:-1], cu[1:], kv, ctx) if b > a]
    check_rows(out, np.concatenate(want), BF16)


@pytest.mark.gpu
@pytest.mark.parametrize("bound", [1, 3, 40, 5000])
def test_a_window_bound_above_the_need(bound):
    windows = [(200, 1), (0, 1), (33, 0), (700, 1)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, 2, 128, 16)
    kv = fill(c, table, ctx, cu, pt, 5)
    q = torch.randn(3, 8, 128, generator=torch.Generator().manual_seed(6)).to(BF16)
    out = ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, bound)
    for b, (K, V) in enumerate(kv):
        if cu[b + 1] > cu[b]:
            check_rows(out[cu[b]: cu[b + 1]], ref.attention(f64(q[cu[b]: cu[b + 1]]), K, V, int(ctx[b]), 128 ** -0.5), BF16)


@pytest.mark.gpu
def test_a_captured_call_follows_its_lengths():
    """One captured call over windows that change between replays: prompts, a few
    rows over long contexts, nothing at all, and prompts again."""
    B, T, Hq, Hkv, D, ps = 40, 6000, 16, 4, 64, 16
    rng = np.random.default_rng(0)
    prompts = [(0, int(n)) for n in rng.integers(1, 240, B)]
    few = [(int(rng.integers(100, 600)), int(rng.integers(0, 9))) for _ in range(B)]
    roomy = [(max(a[0], b[0]), max(a[1], b[1])) for a, b in zip(prompts, few)]
    c, table, _, _, pt, _, _ = pool(roomy, Hkv, D, ps)
    c.k.view(torch.uint8).fill_(0x30)
    g = torch.Generator().manual_seed(1)
    c.v.copy_(torch.randn(c.v.shape, generator=g).to(torch.float8_e4m3fn))
    c.k.copy_(torch.randn(c.k.shape, generator=g).to(torch.float8_e4m3fn))
    c.scale.fill_(127)
    ctx, cu = torch.zeros(B, dtype=torch.int32).cuda(), torch.zeros(B + 1, dtype=torch.int32).cuda()
    q = torch.randn(T, Hq, D, generator=g).to(BF16).cuda()
    out = torch.zeros_like(q)
    ws = torch.full((ops.attn_q8_workspace_size(B, Hq, Hkv, D, 240),), 255, dtype=torch.uint8, device="cuda")
    call = lambda o, w: ops.verify_attn_q8(q, c, pt, ctx, cu, 240, out=o, workspace=w)  # noqa: E731

    def set_windows(w):
        ctx.copy_(torch.tensor([x[0] for x in w], dtype=torch.int32))
        cu.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum([x[1] for x in w])]).astype(np.int32)))

    set_windows(few)
    call(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    for w in (prompts, few, [(5, 0)] * B, prompts, few):
        set_windows(w)
        out.fill_(7.0)
        want = call(torch.full_like(out, 7.0), None)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        n = sum(x[1] for x in w)
        assert torch.isfinite(out).all() and (out[n:] == 7).all() and not (out[:n] == 7).all(-1).any()


@pytest.mark.gpu
def test_two_calls_at_once():
    """Calls on two streams over one cache, each with a workspace of its own."""
    windows = [(900, 8), (0, 64), (300, 1), (40, 30)]
    c, table, ctx, cu, pt, dctx, dcu = pool(windows, 2, 128, 16)
    fill(c, table, ctx, cu, pt, 5)
    qs = [torch.randn(int(cu[-1]), 16, 128, generator=torch.Generator().manual_seed(i)).to(BF16).cuda() for i in range(2)]
    want = [ops.verify_attn_q8(q, c, pt, dctx, dcu, 64) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(ops.verify_attn_q8(qs[i], c, pt, dctx, dcu, 64))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


@pytest.mark.gpu
def test_long_contexts_of_shared_pages():
    """512 sequences that share one long prefix's pages, of many lengths: items of more than 256 steps."""
    B, k, Hq, Hkv, D, ps = 512, 5, 32, 2, 64, 64
    n = 16800
    c, table, ctx, cu, pt, _, _ = pool([(n - 1, 1)], Hkv, D, ps)
    (K, V), = fill(c, table, ctx, cu, pt, 5)
    L = np.random.default_rng(1).integers(16300, n - k, B).astype(np.int32)
    g = torch.Generator().manual_seed(6)
    q = (2 * torch.randn(B * k, Hq, D, generator=g)).to(BF16).cuda()
    out = ops.verify_attn_q8(q, c, pt.expand(B, -1).contiguous(), torch.from_numpy(L).cuda(),
                             torch.arange(0, B * k + 1, k, dtype=torch.int32).cuda(), k)
    Kd, Vd = torch.from_numpy(K).cuda(), torch.from_numpy(V).cuda()
    pos = torch.arange(n, device="cuda")
    for b in range(0, B, 5):
        for h in range(Hkv):
            rows = q[b * k: (b + 1) * k, h * 16: (h + 1) * 16].double().reshape(k * 16, D)
            s = rows @ Kd[:, h].T.contiguous() * D ** -0.5
            s[pos[None] > int(L[b]) + torch.arange(k, device="cuda").repeat_interleave(16)[:, None]] = -float("inf")
            want = torch.softmax(s, 1) @ Vd[:, h].contiguous()
            check_rows(out[b * k: (b + 1) * k, h * 16: (h + 1) * 16], want.view(k, 16, D).cpu().numpy(), BF16)


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,D", [(8, 64), (2, 128)])
def test_nan_rows_inside_a_tile(Hq, D):
    """A value row that is not a number between rows of one tile, before and behind a block's end."""
    for at in (5, 33, 59):
        windows = [(70, 60), (20, 3)]
        c, table, ctx, cu, pt, dctx, dcu = pool(windows, 2, D, 16)
        kv = fill(c, table, ctx, cu, pt, 9)
        k, v = rows_of(windows, 2, D, BF16, 3), rows_of(windows, 2, D, BF16, 4)
        v[at, 1, 7] = float("nan")
        ops.kv_append_q8(k.cuda(), v.cuda(), c, pt, dctx, dcu, 60)
        q = torch.randn(63, Hq, D, generator=torch.Generator().manual_seed(2)).to(BF16)
        out = f64(ops.verify_attn_q8(q.cuda(), c, pt, dctx, dcu, 60))
        nan = np.isnan(out)
        assert nan[at:60, Hq // 2:].all() and not nan[:at].any() and not nan[:60, : Hq // 2].any() and not nan[60:].any()
        K, V = kv[0][0].copy(), kv[0][1].copy()
        K[70:130], V[70:130] = ref.quantise(f64(k[:60]))[0], ref.quantise(f64(v[:60]))[0]
        want = ref.attention(f64(q[:at]), K[: 70 + at], V[: 70 + at], 70, D ** -0.5)
        check_rows(torch.from_numpy(out[:at]), want, BF16)


# --- refusals (no GPU) ---

def c_kv(read=False, **kw):
    a = dict(k=16, ks=128, v=32, vs=128, kp=16, vp=16, sc=16, pt=16, mp=4, ctx=16, cu=16, n=2, mq=3, Hkv=2, D=64, ps=16, P=8,
             dtype=1)
    a.update(kw)
    L = ops.lib()
    if read:
        return L.kv_read_q8(a["kp"], a["vp"], a["sc"], a["pt"], a["mp"], a["ctx"], a["cu"], None, a["n"], a["mq"], a["k"],
                            a["v"], a["Hkv"], a["D"], a["ps"], a["P"], a["dtype"], None)
    return L.kv_append_q8(a["k"], a["ks"], a["v"], a["vs"], a["kp"], a["vp"], a["sc"], a["pt"], a["mp"], a["ctx"], a["cu"],
                          None, a["n"], a["mq"], a["Hkv"], a["D"], a["ps"], a["P"], a["dtype"], None)


@pytest.mark.parametrize("read", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(k=None), -1), (dict(sc=None), -1), (dict(pt=None), -1), (dict(n=-1), -1), (dict(mq=0), -1), (dict(Hkv=0), -1),
    (dict(mp=0), -1), (dict(P=0), -1), (dict(D=96), -2), (dict(ps=8), -2), (dict(ps=48), -2), (dict(dtype=3), -2),
    (dict(n=40000), -2), (dict(k=24), -2), (dict(vp=8), -2), (dict(sc=17), -2), (dict(n=0, k=None), 0)])
def test_cache_refusals(read, kw, status):
    assert c_kv(read, **kw) == status
    assert (ops.lib().ipdv_last_error() != b"") == (status != 0)


@pytest.mark.parametrize("kw,status", [(dict(ks=127), -1), (dict(vs=0), -1), (dict(ks=132), -2)])
def test_append_stride_refusals(kw, status):
    assert c_kv(**kw) == status


def c_attn(**kw):
    a = dict(q=16, qs=256, kp=16, vp=16, sc=16, pt=16, mp=4, ctx=16, cu=16, n=2, mq=3, out=16, Hq=4, Hkv=2, D=64, ps=16, P=8,
             scale=0.125, dtype=1, ws=256, wsb=1 << 30)
    a.update(kw)
    return ops.lib().verify_attn_q8(a["q"], a["qs"], a["kp"], a["vp"], a["sc"], a["pt"], a["mp"], a["ctx"], a["cu"], None,
                                    a["n"], a["mq"], a["out"], a["Hq"], a["Hkv"], a["D"], a["ps"], a["P"], a["scale"],
                                    a["dtype"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), -1), (dict(out=None), -1), (dict(kp=None), -1), (dict(Hq=5), -1), (dict(mq=0), -1), (dict(n=-1), -1),
    (dict(scale=0.0), -1), (dict(scale=float("inf")), -1), (dict(qs=255), -1), (dict(D=96), -2), (dict(ps=128), -2),
    (dict(dtype=2), -2), (dict(q=8), -2), (dict(out=24), -2), (dict(qs=260), -2), (dict(ws=None), -3), (dict(wsb=100), -3),
    (dict(ws=264), -2), (dict(n=0, q=None), 0)])
def test_attention_refusals(kw, status):
    assert c_attn(**kw) == status
    assert (ops.lib().ipdv_last_error() != b"") == (status != 0)


def test_workspace_query():
    assert ops.attn_q8_workspace_size(64, 32, 4, 128, 8) > 0
    assert ops.attn_q8_workspace_size(64, 32, 4, 96, 8) == 0
    assert ops.attn_q8_workspace_size(64, 6, 4, 128, 8) == 0


def test_cache_object_checks_its_tensors():
    with pytest.raises(ValueError):
        ops.Q8Cache.empty(2, 1, 64, 16, device="cpu")


@pytest.mark.gpu
def test_a_workspace_elsewhere_is_refused():
    c, _, _, cu, pt, dctx, dcu = pool([(3, 2)], 2, 64, 16)
    q = torch.zeros(2, 4, 64, dtype=BF16, device="cuda")
    ws = torch.empty(2 * ops.attn_q8_workspace_size(1, 4, 2, 64, 2), dtype=torch.uint8)
    for bad in (ws, ws.cuda()[::2]):
        with pytest.raises(ValueError):
            ops.verify_attn_q8(q, c, pt, dctx, dcu, 2, workspace=bad)
        with pytest.raises(ValueError):
            ops.sample_logits(torch.zeros(1, 50, device="cuda"), torch.zeros(1, device="cuda"), workspace=bad)
