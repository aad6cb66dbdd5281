"""The operators around the 8-bit cache as a rollout engine runs them: rotary
positions, the quantised append, attention over the pages and the filtered
draw, several steps on one cache; eager, on a stream of their own, and captured."""
import numpy as np
import pytest
import torch

from paper_2609_36546_amd import ops
from tests import q8_reference as ref
from tests.test_gpu_q8 import check_rows, f64, pool

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
HQ, HKV, D, PS, V = 8, 2, 64, 16, 5003


class Engine:
    """A batch whose sequences grow by a window per step; buffers kept between steps, as an engine does."""

    def __init__(self, windows, seed, roomy=64):
        grown = [(c, n + roomy) for c, n in windows]
        self.cache, self.table, _, _, self.pt, _, _ = pool(grown, HKV, D, PS, seed)
        self.k = np.array([n for _, n in windows])
        self.cu_h = np.concatenate([[0], np.cumsum(self.k)]).astype(np.int32)
        self.ctx_h = np.array([c for c, _ in windows], np.int32)
        self.T, self.max_q, B = int(self.cu_h[-1]), int(self.k.max()), len(windows)
        self.cu = torch.from_numpy(self.cu_h).cuda()
        self.ctx = torch.from_numpy(self.ctx_h).cuda()
        self.inv, self.factor = ops.rope_inv_freq(D, 1e4, ops.ROPE_YARN, 4.0, 64)
        self.inv_d = self.inv.cuda()
        self.qkv = torch.zeros(self.T, (HQ + 2 * HKV) * D, dtype=BF16, device="cuda")
        self.q = torch.zeros(self.T, HQ, D, dtype=BF16, device="cuda")
        self.kr = torch.zeros(self.T, HKV, D, dtype=BF16, device="cuda")
        self.out = torch.zeros_like(self.q)
        self.logits = torch.zeros(self.T, V, device="cuda")
        self.u = torch.zeros(self.T, device="cuda")
        self.temp = torch.full((self.T,), 0.8, device="cuda")
        self.top_k = torch.full((self.T,), 40, dtype=torch.int32, device="cuda")
        self.top_p = torch.full((self.T,), 0.9, device="cuda")
        self.token = torch.zeros(self.T, dtype=torch.int32, device="cuda")
        self.logp = torch.zeros(self.T, device="cuda")
        self.ws = torch.full((ops.attn_q8_workspace_size(B, HQ, HKV, D, self.max_q),), 255, dtype=torch.uint8, device="cuda")
        self.sws = torch.full((ops.sample_logits_workspace_size(self.T, V),), 255, dtype=torch.uint8, device="cuda")

    def set_inputs(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=g))
        self.logits.copy_(4 * torch.randn(self.logits.shape, generator=g))
        self.u.copy_(torch.rand(self.T, generator=g))

    def step(self):
        q = self.qkv[:, : HQ * D].view(self.T, HQ, D)
        k = self.qkv[:, HQ * D: (HQ + HKV) * D].view(self.T, HKV, D)
        v = self.qkv[:, (HQ + HKV) * D:].view(self.T, HKV, D)
        ops.rope_window(q, k, self.inv_d, self.ctx, self.cu, self.max_q, factor=self.factor, q_out=self.q, k_out=self.kr)
        ops.kv_append_q8(self.kr, v, self.cache, self.pt, self.ctx, self.cu, self.max_q)
        ops.verify_attn_q8(self.q, self.cache, self.pt, self.ctx, self.cu, self.max_q, out=self.out, workspace=self.ws)
        ops.sample_logits(self.logits, self.u, self.temp, self.top_k, self.top_p, token=self.token, logp=self.logp,
                          workspace=self.sws)
        return self.out.clone(), self.token.clone(), self.logp.clone()


def test_steps_match_the_plain_form():
    e = Engine([(0, 3), (0, 1), (0, 0), (0, 8)], 1)
    K = [np.zeros((0, HKV, D)) for _ in e.k]
    W = [np.zeros((0, HKV, D)) for _ in e.k]
    for step in range(6):
        e.set_inputs(step)
        out, token, logp = e.step()
        x = e.qkv
        pos = np.concatenate([e.ctx_h[b] + np.arange(n) for b, n in enumerate(e.k)])
        q = ref.rope(f64(x[:, : HQ * D].reshape(e.T, HQ, D)), pos, e.inv.numpy(), 0, e.factor)
        # the turned rows, rounded to bf16: within a rounding of the plain form's, and what the rest goes by
        assert (np.abs(f64(e.q) - q) <= 2.0 ** -8 * np.abs(q) + 1e-5).all()
        kq = ref.quantise(f64(e.kr))[0]
        vq = ref.quantise(f64(x[:, (HQ + HKV) * D:].reshape(e.T, HKV, D)))[0]
        for b, n in enumerate(e.k):
            r0, r1 = e.cu_h[b], e.cu_h[b + 1]
            K[b], W[b] = np.concatenate([K[b], kq[r0:r1]]), np.concatenate([W[b], vq[r0:r1]])
            if n:
                check_rows(out[r0:r1], ref.attention(f64(e.q[r0:r1]), K[b], W[b], int(e.ctx_h[b]), D ** -0.5), BF16)
        for i in range(e.T):
            assert ref.draw_is_right(f64(e.logits)[i], float(e.temp[i]), 40, float(e.top_p[i]), 0.0, float(e.u[i]),
                                     int(token[i]), float(logp[i]))
        e.ctx_h = e.ctx_h + e.k.astype(np.int32)
        e.ctx.copy_(torch.from_numpy(e.ctx_h))


def test_another_stream_gives_the_same():
    a, b = (Engine([(20, 4), (7, 1), (0, 9)], 2) for _ in range(2))
    for e in (a, b):
        e.cache.k.view(torch.uint8).zero_()
        e.cache.v.view(torch.uint8).zero_()
        e.cache.scale.fill_(127)
        e.set_inputs(5)
    want = a.step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = b.step()
    torch.cuda.current_stream().wait_stream(s)
    for x, y in zip(want, got):
        assert torch.equal(x, y)


def test_two_captured_steps_replay_like_eager_ones():
    """Two engines' steps as two graphs, replayed in turn with eager work and
    synchronisations between; every replay equals the eager step."""
    shapes = [[(33, 2), (90, 1)], [(5, 7), (0, 4), (61, 1)]]
    eager, graphed, graphs = [], [], []
    for i, w in enumerate(shapes):
        pair = [Engine(w, 10 + i) for _ in range(2)]
        for e in pair:
            e.cache.k.view(torch.uint8).zero_()
            e.cache.v.view(torch.uint8).zero_()
            e.cache.scale.fill_(127)
            e.set_inputs(100)
        eager.append(pair[0])
        graphed.append(pair[1])
    s = torch.cuda.Stream()
    for e in graphed:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            e.step()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = e.step()
        graphs.append((g, res))
    for e in eager:
        e.step()
    for round_ in range(4):
        for i, (g, res) in enumerate(graphs):
            for e in (eager[i], graphed[i]):
                e.set_inputs(200 + 10 * round_ + i)
                e.ctx.add_(1)
            want = eager[i].step()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip(want, res):
                assert torch.equal(x, y)
            assert torch.equal(eager[i].cache.k.view(torch.uint8), graphed[i].cache.k.view(torch.uint8))
            assert torch.equal(eager[i].cache.scale, graphed[i].cache.scale)
