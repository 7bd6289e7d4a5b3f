"""The layer operators together, as a serving loop uses them: tables from lengths on the GPU,
norm, rotation and page write, differential attention over the pages; and captured into
graphs."""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_16824_amd as cwlib

pytestmark = pytest.mark.gpu
PAIRS, G, EPS, AFTER = 2, 3, 1e-5, 0.7


class _Model:
    """One layer's weights and pools, and the requests it serves."""

    def __init__(self, d, page, pages, seqs, stride, dtype, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.gen, self.d, self.page = g, d, page
        self.hq, self.hkv = 2 * PAIRS * G, 2 * PAIRS
        self.wq, self.wk = (torch.rand(d, generator=g, device="cuda") + 0.5 for _ in "qk")
        self.weight = torch.rand(2 * d, generator=g, device="cuda") + 0.5
        self.lam = torch.rand(PAIRS * G, generator=g, device="cuda") * 0.6 + 0.2
        a = torch.arange(4000, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
        self.cos_sin = torch.cat([a.cos(), a.sin()], 1).float().cuda()
        self.k_scale = self.v_scale = None
        if dtype == "fp8":
            self.k_pool, self.v_pool = (torch.full((pages, self.hkv, page, d), 0x7F, dtype=torch.uint8, device="cuda") for _ in "kv")
            self.k_scale, self.v_scale = (torch.rand(pages, self.hkv, generator=g, device="cuda") * 0.01 + 0.008 for _ in "kv")
        else:
            self.k_pool, self.v_pool = (torch.full((pages, self.hkv, page, d), float("nan"), dtype=torch.bfloat16, device="cuda")
                                        for _ in "kv")
        self.table = torch.full((seqs, stride), 1 << 30, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)

    def qkv(self, t):
        x = torch.randn(t, self.hq + 2 * self.hkv, self.d, generator=self.gen, device="cuda", dtype=torch.bfloat16)
        return x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:]

    def rotate_and_write(self, qkv, tables, **kw):
        q, k, v = qkv
        return cwlib.qk_norm_rope(q, k, self.cos_sin, tables.positions, q_weight=self.wq, k_weight=self.wk, v=v,
                                  k_pool=self.k_pool, v_pool=self.v_pool, slots=tables.slots, k_scale=self.k_scale,
                                  v_scale=self.v_scale, **kw)

    def attend(self, q, k, v, lp, ls, **kw):
        return cwlib.diff_attention(q, k, v, self.k_pool, self.v_pool, self.table, lp, ls, G, self.d ** -0.5, self.lam,
                                    k_scale=self.k_scale, v_scale=self.v_scale, norm_weight=self.weight, norm_eps=EPS,
                                    out_scale=AFTER, **kw)


def _bits(t):
    return t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


STEPS = [[37, 5, 64], [1, 1, 40], [20, 1, 1], [1, 1, 1], [1, 100, 1]]


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
def test_serving_loop(d, page):
    """Five steps of three requests; every row against the oracle's attention over the whole
    sequences' keys and values, which never saw a page.

    The rows: tolerance of the attention's own tests (bf16 weights: r = 2 2^-8 + 2^-10 of the
    mass), its norm and its rounding."""
    print(f"\n[case] serving loop d={d} page={page}", flush=True)
    m = _Model(d, page, 64, 3, 24, "bf16", seed=d)
    lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    host = np.zeros(3, dtype=np.int64)
    free = m.free
    per = [[[], [], [], []] for _ in range(3)]  # q, k, v, out rows of each request
    for step in STEPS:
        new = torch.tensor(step, dtype=torch.int32, device="cuda")
        t = sum(step)
        tables = cwlib.build_step_tables(lens, new, free, m.table, page, t + 3)
        short = tables._replace(positions=tables.positions[:t], slots=tables.slots[:t])
        q, k, v = m.rotate_and_write(m.qkv(t), short)
        out = m.attend(q, k, v, host, step)
        taken, total, over = tables.info.tolist()
        assert total == t and over == 0 and tables.slots[t:].tolist() == [-1] * 3
        free = free[taken:]
        lens += new
        at = 0
        for b, n in enumerate(step):
            for i, x in enumerate((q, k, v, out)):
                per[b][i].append(x[at:at + n])
            at += n
        host += step
    torch.cuda.synchronize()
    assert len(free) == 64 - sum(-(-int(n) // page) for n in host)
    cat = [[torch.cat(x) for x in p] for p in per]
    q, k, v, out = (torch.cat([c[i] for c in cat]) for i in range(4))
    inp = oracle.PagedInputs(q=_bits(q), k_new=_bits(k), v_new=_bits(v), k_pool=_bits(m.k_pool), v_pool=_bits(m.v_pool),
                             block_table=m.table.cpu().numpy(), prefix_lens=np.zeros(3, dtype=np.int64), suffix_lens=host,
                             gqa_group=G, softmax_scale=d ** -0.5)
    w, lam = m.weight.cpu().double().numpy(), m.lam.cpu().double().numpy()
    ref, terms = oracle.diff_attention(inp, lam, w, EPS, AFTER)
    x, dx = terms["x"], (2 * 2.0 ** -8 + 2.0 ** -10) * terms["mass"]
    root = np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
    rms = np.sqrt((dx * dx).mean(-1, keepdims=True))
    tol = 1.1 * np.abs(AFTER * w) / root * (dx + np.abs(x) * rms / root) + 2.0 ** -8 * np.abs(ref)
    over = np.abs(out.cpu().double().numpy() - ref) / tol
    print(f"[serving loop] worst {over.max():.3f} of the tolerance over {len(ref)} rows", flush=True)
    assert over.max() <= 1.0


def test_block_manager_serves_the_loop():
    """The step's pages are the ones the framework's own check reads without complaint."""
    print("\n[case] tables through check_block_table", flush=True)
    m = _Model(64, 16, 40, 4, 12, "bf16", seed=5)
    lp, ls = [0, 0, 0, 0], [17, 0, 90, 1]
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    assert cwlib.check_block_table(m.table, lp, ls, 40, 16).sum() == 2 + 6 + 1
    cwlib.build_step_tables(dev(lp), dev(ls), m.free, m.table, 16, 108)
    assert cwlib.check_block_table(m.table, lp, ls, 40, 16).tolist() == [0, 0, 0, 0]


def _capture(fn):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fn()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fn()
    torch.cuda.synchronize()
    return g


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_captured_tables_and_rotation_follow_new_lengths(dtype):
    """One captured graph serves steps of other lengths: they lie on the GPU."""
    print(f"\n[case] captured tables and page write {dtype}", flush=True)
    m = _Model(64, 16, 300, 5, 40, dtype, seed=9)
    tokens = 200
    lens, new = (torch.zeros(5, dtype=torch.int32, device="cuda") for _ in "ab")
    new += 7
    x = torch.empty(tokens, m.hq + 2 * m.hkv, 64, dtype=torch.bfloat16, device="cuda")
    qkv = (x[:, :m.hq], x[:, m.hq:m.hq + m.hkv], x[:, m.hq + m.hkv:])
    new_t = lambda n, dt: torch.empty(n, dtype=dt, device="cuda")
    bufs = dict(cu_rows=new_t(6, torch.int32), seq_ids=new_t(tokens, torch.int32), positions=new_t(tokens, torch.int32),
                slots=new_t(tokens, torch.int64), info=new_t(3, torch.int64))
    outs = dict(q_out=torch.empty(tokens, m.hq, 64, dtype=torch.bfloat16, device="cuda"),
                k_out=torch.empty(tokens, m.hkv, 64, dtype=torch.bfloat16, device="cuda"),
                v_out=torch.empty(tokens, m.hkv, 64, dtype=torch.bfloat16, device="cuda"))

    def work():
        m.rotate_and_write(qkv, cwlib.build_step_tables(lens, new, m.free, m.table, 16, tokens, **bufs), **outs)

    state = lambda: [t.clone() for t in (m.table, m.k_pool, m.v_pool, *bufs.values(), *outs.values())]
    fresh = [t.clone() for t in (m.table, m.k_pool, m.v_pool)]

    def reset():
        for t, f in zip((m.table, m.k_pool, m.v_pool), fresh):
            t.copy_(f)
        for t in outs.values():
            t.fill_(0)

    m.free = m.free[m.free < 200].contiguous()  # pages 200 on are those held already
    g = _capture(work)
    for rep, (a, b) in enumerate((([0, 0, 0, 0, 0], [7, 1, 60, 0, 99]), ([0, 0, 16, 0, 0], [1, 1, 1, 1, 1]),
                                  ([0, 16, 0, 0, 32], [0, 64, 2, 100, 30]))):
        lens.copy_(torch.tensor(a, dtype=torch.int32))
        new.copy_(torch.tensor(b, dtype=torch.int32))
        x.copy_(torch.randn(x.shape, generator=m.gen, device="cuda"))
        for i in range(5):
            fresh[0][i, :a[i] // 16] = torch.arange(200 + 10 * i, 200 + 10 * i + a[i] // 16, dtype=torch.int32)
        reset()
        work()
        torch.cuda.synchronize()
        want = state()
        reset()
        g.replay()
        torch.cuda.synchronize()
        for i, (p, w) in enumerate(zip(state(), want)):
            assert torch.equal(p.view(torch.uint8), w.view(torch.uint8)), (rep, i)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("ls", [[1, 1, 1, 1], [70, 33, 2, 129], [1, 70, 1, 129]])
def test_captured_attention_replays(dtype, ls):
    """Two captured calls that share a workspace, between eager calls of other shapes."""
    print(f"\n[case] captured diff attention {dtype} {ls}", flush=True)
    cwlib.init()
    m = _Model(128, 16, 400, 4, 80, dtype, seed=11)
    m.k_pool.copy_(torch.randint(0, 120, m.k_pool.shape, generator=m.gen, device="cuda").to(m.k_pool.dtype))
    m.v_pool.copy_(torch.randint(0, 120, m.v_pool.shape, generator=m.gen, device="cuda").to(m.v_pool.dtype))
    if dtype == "bf16":
        m.k_pool.div_(100)
        m.v_pool.div_(100)
    m.table.copy_(torch.randperm(400, generator=m.gen, device="cuda")[:320].view(4, 80).to(torch.int32))
    lp = [300, 1000, 17, 500]
    t = sum(ls)
    q, k, v = (x.contiguous() for x in m.qkv(t))
    nb = cwlib.diff_workspace_bytes(lp, ls, PAIRS, G, 128, 16, dtype)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    outs = [torch.empty(t, PAIRS * G, 256, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    want = m.attend(q, k, v, lp, ls, workspace=ws).clone()
    small = tuple(x.contiguous() for x in m.qkv(5))
    other = m.attend(*small, [40, 7], [4, 1])

    def work():
        for o in outs:
            m.attend(q, k, v, lp, ls, out=o, workspace=ws)

    g = _capture(work)
    for rep in range(3):
        for o in outs:
            o.fill_(float("nan"))
        for _ in range(10):
            again = m.attend(*small, [40, 7], [4, 1])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, other)
        assert all(torch.equal(o, want) for o in outs), rep


def test_two_streams_at_once():
    """Calls that may overlap, each with its own workspace and outputs."""
    print("\n[case] two streams at once", flush=True)
    m = _Model(128, 16, 400, 4, 80, "bf16", seed=13)
    m.k_pool.copy_(torch.randn(m.k_pool.shape, generator=m.gen, device="cuda"))
    m.v_pool.copy_(torch.randn(m.v_pool.shape, generator=m.gen, device="cuda"))
    m.table.copy_(torch.randperm(400, generator=m.gen, device="cuda")[:320].view(4, 80).to(torch.int32))
    calls = [([900, 40, 333, 0], [40, 200, 3, 1]), ([1200, 1000, 5, 77], [1, 1, 1, 1])]
    data = [tuple(x.contiguous() for x in m.qkv(sum(ls))) for _, ls in calls]
    want = [m.attend(*d, *c) for d, c in zip(data, calls)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = [[], []]
    for _ in range(6):
        for i, (d, c) in enumerate(zip(data, calls)):
            with torch.cuda.stream(streams[i]):
                got[i].append(m.attend(*d, *c))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, w) for x in g)
