"""residual_norm, qk_norm_rope_axes with its page write and shaped_attention together, as a served layer runs them:
against the same layer in plain float32, prompts cut into chunks and single tokens against one call, captured and
replayed, on two streams, and two graphs that share a workspace."""
import numpy as np
import pytest
import torch

import paper_2606_16824_amd as cwlib
from gpu_util import to_gpu
from shaped_util import call, inputs, shape_of

pytestmark = pytest.mark.gpu

HQ, HKV, D, PAGE, WIDTH, EPS = 8, 2, 64, 16, 512, 1e-5
AXES = [0] * 12 + [1] * 10 + [2] * 10
CAP, WINDOW = 20.0, 60


class Layer:
    """Weights, pools and block tables of one layer over two sequences."""

    def __init__(self, seed=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        bf = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[0] ** -0.5).to(torch.bfloat16)
        self.qkv, self.proj = bf(WIDTH, (HQ + 2 * HKV) * D), bf(HQ * D, WIDTH)
        w = lambda n: torch.rand(n, generator=g, device="cuda") + 0.5
        self.wq, self.wk, self.post, self.pre, self.first = w(D), w(D), w(WIDTH), w(WIDTH), w(WIDTH)
        a = torch.arange(400, dtype=torch.float64, device="cuda")[:, None] * 100.0 ** (-torch.arange(0, D, 2, device="cuda") / D)
        self.angles = torch.cat([a.cos(), a.sin()], 1).float()
        self.slopes = torch.exp2(-torch.arange(1, HQ + 1, device="cuda").float())
        self.pools = [torch.full((64, HKV, PAGE, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        self.table = torch.randperm(64, generator=g, device="cuda").to(torch.int32).view(2, 32).contiguous()

    def step(self, x, pos, lp, ls, full=None, lse=None):
        """x bf16 [T, WIDTH] is the residual stream; returns it after the layer, and the next block's input."""
        seq = torch.repeat_interleave(torch.arange(2, device="cuda"), torch.tensor(ls, device="cuda"))
        at = torch.cat([torch.arange(a, a + n, device="cuda") for a, n in zip(lp, ls)])
        slots = self.table[seq, at // PAGE].long() * PAGE + at % PAGE
        _, y = cwlib.residual_norm(torch.zeros_like(x), x, pre_weight=self.first, eps=EPS)
        z = torch.matmul(y, self.qkv).view(-1, HQ + 2 * HKV, D)
        q, k, v = cwlib.qk_norm_rope_axes(z[:, :HQ], z[:, HQ:HQ + HKV], self.angles, pos, AXES, q_weight=self.wq, k_weight=self.wk,
                                          eps=EPS, v=z[:, HQ + HKV:], k_pool=self.pools[0], v_pool=self.pools[1], slots=slots)
        o = cwlib.shaped_attention(q, k, v, self.pools[0], self.pools[1], self.table, lp, ls, HQ // HKV, D ** -0.5, score_cap=CAP,
                                   slopes=self.slopes, window=WINDOW, full_lens=full, lse=lse)
        return cwlib.residual_norm(torch.matmul(o.view(-1, HQ * D), self.proj), x, post_weight=self.post, pre_weight=self.pre, eps=EPS)

    def plain(self, x, pos, n, full):
        """The layer over one whole sequence in float32 (rounded nowhere)."""
        rms = lambda t, w: t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * w
        x = x.float()
        z = (rms(x, self.first) @ self.qkv.float()).view(n, HQ + 2 * HKV, D)
        half = torch.arange(D // 2, device="cuda")
        row = pos[torch.tensor(AXES, device="cuda")].long().t()
        cos, sin = self.angles[row, half][:, None], self.angles[row, D // 2 + half][:, None]
        turn = lambda t: torch.cat([t[..., :D // 2] * cos - t[..., D // 2:] * sin, t[..., D // 2:] * cos + t[..., :D // 2] * sin], -1)
        q, k, v = turn(rms(z[:, :HQ], self.wq)), turn(rms(z[:, HQ:HQ + HKV], self.wk)), z[:, HQ + HKV:]
        k, v = (t.repeat_interleave(HQ // HKV, 1).transpose(0, 1).contiguous() for t in (k, v))
        s = torch.stack([q[:, h] @ k[h].t() for h in range(HQ)]) * D ** -0.5
        s = torch.tanh(s / CAP) * CAP
        p, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None, :]
        s = s - self.slopes[:, None, None] * (p - j).abs()
        seen = ((j <= p) | (j < full)) & (j > p - WINDOW)
        w = torch.softmax(s.masked_fill(~seen, -torch.inf), -1)
        o = torch.stack([w[h] @ v[h] for h in range(HQ)], 1).reshape(n, HQ * D)
        r = x + rms(o @ self.proj.float(), self.post)
        return r, rms(r, self.pre)


def _stream(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(sum(n), WIDTH, generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, 400, (3, sum(n)), generator=g, device="cuda", dtype=torch.int32)
    return x, pos


def test_layer_against_plain_and_cut_into_steps():
    """Relative 2-norm of the outputs' error: seven roundings to bf16 lie on the way (input of the projections, their
    outputs, rotated heads, weights, attention, residual, y), each at most 2^-8 and those before the scores
    taken through exponents of at most some 6 (2 * 6 * 2^-8 for a weight): below 0.1 in any case, and two runs that
    cut the prompts otherwise (other tiles, the streaming kernel) below twice that of each other."""
    print("\n[case] layer", flush=True)
    n = [150, 97]
    x, pos = _stream(n, 1)
    full = [40, 0]
    one = Layer()
    res, y = one.step(x, pos, [0, 0], n, full=full)
    a = 0
    for b in range(2):
        want, want_y = one.plain(x[a:a + n[b]], pos[:, a:a + n[b]], n[b], full[b])
        for got, ref in ((res, want), (y, want_y)):
            e = (got[a:a + n[b]].float() - ref).norm() / ref.norm()
            print(f"[layer] relative {e.item():.2e}", flush=True)
            assert e.item() < 0.1
        a += n[b]
    # the same in steps: chunks and single tokens mixed, the prefix mask's tokens in the first one
    cut = Layer()
    done, out = [0, 0], [[], []]
    for step in ([40, 33], [1, 20], [1, 1], [60, 0], [1, 1], [0, 42], [47, 0]):
        rows, take = [], []
        for b in range(2):
            lo = done[b] + (0 if b == 0 else n[0])
            rows.append(torch.arange(lo, lo + step[b], device="cuda"))
        rows = torch.cat(rows)
        got, _ = cut.step(x[rows].contiguous(), pos[:, rows].contiguous(), list(done), step, full=full)
        out[0].append(got[:step[0]])
        out[1].append(got[step[0]:])
        done = [done[b] + step[b] for b in range(2)]
    torch.cuda.synchronize()
    assert done == n
    for b, part in ((0, res[:150]), (1, res[150:])):
        e = (torch.cat(out[b]).float() - part.float()).norm() / part.float().norm()
        print(f"[layer] cut against whole {e.item():.2e}", flush=True)
        assert e.item() < 0.2


def test_layer_captured_and_replayed():
    """A step of single tokens in a graph, replayed on other tokens between eager calls."""
    print("\n[case] layer graph", flush=True)
    n, lp = [1, 1], [149, 77]
    layer = Layer()
    x0, pos0 = _stream(lp, 5)
    layer.step(x0, pos0, [0, 0], lp)
    cwlib.init()
    x, pos = (t.clone() for t in _stream(n, 6))
    at = torch.tensor(lp, device="cuda")
    slots = layer.table[torch.arange(2, device="cuda"), at // PAGE].long() * PAGE + at % PAGE
    ws = torch.empty(cwlib.shaped_workspace_bytes(lp, n, HKV, HQ // HKV, D, PAGE, window=WINDOW), dtype=torch.uint8, device="cuda")
    out = torch.empty(2, HQ, D, dtype=torch.bfloat16, device="cuda")

    def step():
        _, y = cwlib.residual_norm(x, x, pre_weight=layer.first, eps=EPS)
        z = y[:, :HQ * D].view(2, HQ, D)  # (no projection: library products stay out of this graph)
        kv = y[:, :HKV * D].view(2, HKV, D)
        q, k, v = cwlib.qk_norm_rope_axes(z, kv, layer.angles, pos, AXES, q_weight=layer.wq, k_weight=layer.wk, v=kv,
                                          k_pool=layer.pools[0], v_pool=layer.pools[1], slots=slots)
        cwlib.shaped_attention(q, k, v, layer.pools[0], layer.pools[1], layer.table, lp, n, HQ // HKV, D ** -0.5, score_cap=CAP,
                               slopes=layer.slopes, window=WINDOW, out=out, workspace=ws)
        return cwlib.residual_norm(out.view(2, HQ * D), x, post_weight=layer.post, pre_weight=layer.pre, eps=EPS)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r, y = step()
    for seed in (11, 12, 13):
        nx, npos = _stream(n, seed)
        x.copy_(nx)
        pos.copy_(npos)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (r, y, out)]
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], out)


@pytest.mark.parametrize("dt", ["bf16", "fp8"])
def test_captured_mixed_step_and_a_shared_workspace(dt):
    """Two graphs of different batches on one workspace, replayed in turn; every replay writes its own plan."""
    print(f"\n[case] shaped graphs {dt}", flush=True)
    cwlib.init()
    cases = []
    for lp, ls, seed in (([300, 0, 17, 500], [1, 70, 1, 129], 3), ([64, 900], [200, 1], 4)):
        w = inputs(lp, ls, 2, 4, 64, 16, dt, seed=seed)
        n = w.spec.prefix_lens + w.spec.suffix_lens
        kw = shape_of(w, cap=20.0, slopes=True, window=100, docs=3, full=n // 2, seed=seed)
        cases.append((to_gpu(w), kw))
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    wants = [call(dw, kw, workspace=ws).clone() for dw, kw in cases]
    dev = [{k: torch.from_numpy(kw[k]).cuda() for k in ("slopes", "key_begins")} for _, kw in cases]
    graphs, outs = [], []
    torch.cuda.synchronize()
    for (dw, kw), d in zip(cases, dev):
        s = dw.spec
        out = torch.zeros_like(dw.q)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cwlib.shaped_attention(dw.q, dw.k_new, dw.v_new, dw.k_pool, dw.v_pool, dw.block_table, s.prefix_lens, s.suffix_lens,
                                   s.gqa_group, s.softmax_scale, k_scale=dw.k_scale, v_scale=dw.v_scale, out=out, workspace=ws,
                                   **{**kw, **d})
        graphs.append(g)
        outs.append(out)
    for _ in range(3):
        for i in (0, 1, 1, 0):
            outs[i].zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], wants[i])
        call(*cases[0], workspace=ws)


def test_two_streams_at_once():
    print("\n[case] shaped streams", flush=True)
    jobs = []
    for seed, dt in ((5, "bf16"), (6, "fp8")):
        w = inputs([700, 40, 1500], [90, 1, 33], 2, 4, 128, 16, dt, seed=seed)
        kw = shape_of(w, cap=30.0, window=333, seed=seed)
        dw = to_gpu(w)
        jobs.append((dw, kw, call(dw, kw).clone(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for i, (dw, kw, _, stream) in enumerate(jobs):
            with torch.cuda.stream(stream):
                got[i].append(call(dw, kw))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, jobs[i][2]) for x in got[i])


def test_offsets_past_32_bits():
    """Pages beyond 4 GiB of each pool: the same bits as with the pages at the pools' start."""
    print("\n[case] shaped large pools", flush=True)
    w = inputs([300, 40], [1, 60], 8, 2, 128, 64, "bf16", seed=8)
    kw = shape_of(w, cap=20.0, window=200)
    dw = to_gpu(w)
    want = call(dw, kw)
    small, num = dw.k_pool.shape[0], 40000  # 5.2 GB a pool
    for name in ("k_pool", "v_pool"):
        big = torch.empty(num, 8, 64, 128, dtype=torch.bfloat16, device="cuda")
        big[num - small:] = getattr(dw, name)
        setattr(dw, name, big)
    table = dw.block_table
    dw.block_table = torch.where(table < small, table + (num - small), table)
    got = call(dw, kw)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
