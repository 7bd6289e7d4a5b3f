"""residual_norm against the oracle, element by element.

Tolerance, from the kernel's arithmetic, mag = |s r| + |gate u|:
  r': 2^-16 mag: a row's sum of squares adds up to 64 products per lane, then over 256 lanes (relative error below
      80 * 2^-24), its root halves that, and some six more fp32 roundings follow; stored: + 2^-8 |r'| (bf16), 2^-24 |r'|
  y: |w| / root (d + |r'| rms(d) / root) with d = 2^-16 mag, root = sqrt(mean r'^2 + eps), + 2^-16 |y| for the same
      arithmetic once more; stored: + 2^-8 |y|"""
import numpy as np
import pytest
import torch

import oracle
import paper_2606_16824_amd as cwlib

pytestmark = pytest.mark.gpu

WIDTHS = [8, 64, 72, 512, 520, 1000, 1024, 1536, 2048, 2056, 4096, 5120, 6152, 8192, 10000, 16384]


def _data(tokens, width, wide, gate, seed, stride=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(tokens, width + stride, generator=g).to(torch.bfloat16)
    r = torch.randn(tokens, width, generator=g) * torch.where(torch.rand(width, generator=g) < 0.02, 60.0, 2.0)
    r = r if wide else r.to(torch.bfloat16)
    gt = {"": None, "row": torch.randn(width, generator=g).to(torch.bfloat16),
          "token": torch.randn(tokens, width + stride, generator=g).to(torch.bfloat16)}[gate]
    a, b = torch.rand(width, generator=g) + 0.5, torch.rand(width, generator=g) + 0.5
    return x, r, gt, a, b


def _check(x, r, gate, post, pre, scale, eps, got, what):
    f = lambda t: None if t is None else t.double().numpy()
    res, y = oracle.residual_norm(f(x), f(r), f(post), f(gate), scale, f(pre), eps)
    u, _ = oracle.residual_norm(f(x), np.zeros(x.shape), f(post), f(gate), 0.0, None, eps)
    mag = np.abs(scale * f(r)) + np.abs(u)
    d = 2.0 ** -16 * mag
    tol = d + (2.0 ** -24 if r.dtype is torch.float32 else 2.0 ** -8) * np.abs(res) + 1e-38
    over = (np.abs(f(got[0].cpu()) - res) / tol).max()
    over_y = 0.0
    if pre is not None:
        root = np.sqrt((res * res).mean(-1, keepdims=True) + eps)
        tol = np.abs(f(pre)) / root * (d + np.abs(res) * np.sqrt((d * d).mean(-1, keepdims=True)) / root) + (2.0 ** -16 + 2.0 ** -8) * np.abs(y)
        over_y = (np.abs(f(got[1].cpu()) - y) / (tol + 1e-38)).max()
    else:
        assert got[1] is None
    print(f"[{what}] worst {over:.3f}, y {over_y:.3f} of the tolerance", flush=True)
    assert over <= 1.0 and over_y <= 1.0, what


@pytest.mark.parametrize("tokens", [1, 5, 9000])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("wide", [False, True])
def test_widths(tokens, width, wide):
    if tokens == 9000 and width > 1100:
        tokens = 2300  # (more rows than workgroups)
    gate = ["", "row", "token"][(width // 8 + tokens) % 3]
    print(f"\n[case] residual {tokens} {width} {wide} {gate}", flush=True)
    x, r, gt, a, b = _data(tokens, width, wide, gate, width + tokens)
    got = cwlib.residual_norm(x.cuda(), r.cuda(), post_weight=a.cuda(), gate=None if gt is None else gt.cuda(), residual_scale=0.7,
                              pre_weight=b.cuda(), eps=1e-5)
    torch.cuda.synchronize()
    assert got[0].dtype == r.dtype and got[1].dtype == torch.bfloat16
    _check(x, r, gt, a, b, 0.7, 1e-5, got, f"residual {tokens} {width} {wide} {gate}")


@pytest.mark.parametrize("width", [72, 2048, 4096, 16384])
@pytest.mark.parametrize("post,pre,gate", [(False, False, ""), (True, False, "row"), (False, True, "token"), (False, False, "token"),
                                           (False, True, ""), (True, False, "")])
def test_parts(width, post, pre, gate):
    """Every part left out: plain residual sums, no second norm; more rows than workgroups."""
    print(f"\n[case] residual parts {width} {post} {pre} {gate}", flush=True)
    for tokens in (3, 2100):
        x, r, gt, a, b = _data(tokens, width, False, gate, 5)
        got = cwlib.residual_norm(x.cuda(), r.cuda(), post_weight=a.cuda() if post else None, gate=None if gt is None else gt.cuda(),
                                  pre_weight=b.cuda() if pre else None, eps=0.0)
        torch.cuda.synchronize()
        _check(x, r, gt, a if post else None, b if pre else None, 1.0, 0.0, got, f"parts {tokens} {width} {post} {pre} {gate}")


@pytest.mark.parametrize("wide", [False, True])
def test_in_place_strided_and_out(wide):
    """x and gate columns of a wider projection, the residual updated where it lies, no element behind the rows."""
    print(f"\n[case] residual in place {wide}", flush=True)
    x, r, gt, a, b = _data(37, 1000, wide, "token", 8, stride=24)
    rg = torch.full((38, 1000), 7.0, dtype=r.dtype, device="cuda")
    rg[:37] = r.cuda()
    y = torch.full((38, 1000), 7.0, dtype=torch.bfloat16, device="cuda")
    got = cwlib.residual_norm(x.cuda()[:, 8:1008], rg[:37], post_weight=a.cuda(), gate=gt.cuda()[:, 16:1016], pre_weight=b.cuda(),
                              eps=1e-6, residual_out=rg[:37], y_out=y[:37])
    torch.cuda.synchronize()
    assert got[0].data_ptr() == rg.data_ptr() and (rg[37] == 7.0).all() and (y[37] == 7.0).all()
    _check(x[:, 8:1008], r, gt[:, 16:1016], a, b, 1.0, 1e-6, got, "in place")


def test_large_small_and_none():
    """Values near the header's limit, a row of zeros, and no token."""
    print("\n[case] residual extremes", flush=True)
    x, r, _, a, b = _data(4, 2048, False, "", 9)
    x[0] *= 2.0 ** 54
    r[1] *= 2.0 ** 50
    x[2], r[2] = 0.0, 0.0
    x[3] *= 2.0 ** -60
    got = cwlib.residual_norm(x.cuda(), r.cuda(), post_weight=a.cuda(), pre_weight=b.cuda(), eps=1e-6)
    torch.cuda.synchronize()
    _check(x, r, None, a, b, 1.0, 1e-6, got, "extremes")
    empty = cwlib.residual_norm(x.cuda()[:0], r.cuda()[:0], pre_weight=b.cuda())
    assert empty[0].shape == empty[1].shape == (0, 2048)


def test_replayed_capture():
    print("\n[case] residual graph", flush=True)
    x, r, gt, a, b = _data(300, 4096, False, "row", 10)
    xg, rg, gg, ag, bg = x.cuda(), r.cuda(), gt.cuda(), a.cuda(), b.cuda()
    out, y = torch.empty_like(rg), torch.empty_like(xg)
    call = lambda: cwlib.residual_norm(xg, rg, post_weight=ag, gate=gg, pre_weight=bg, residual_out=out, y_out=y)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (1, 2, 3):
        xg.copy_(torch.randn(300, 4096, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), y.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], y)
