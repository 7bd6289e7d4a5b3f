"""shaped_attention over fp8 pools whose values are so small that fp16, which chunks hold them in, has
only some of its bits left for them: page scales that are no powers of two.

A code times its scale is rounded once there: to 2^-25, half a step of fp16 below 2^-14, beside the
scale's own rounding to 11 bits (the bound of shaped_util has both).  The weights are fp16 too, in chunks and
for single tokens, and it may drop those below 2^-33 of a row's largest one (half a step below 2^-14, against 2^8).
Here the other keys' weights are below e^-38 < 2^-54 of the ruling key's, so all that they add, and no more,
may be missing: 60 * 2^-54 of the largest value, also in an element where the ruling key's value is 0."""
import numpy as np
import pytest
import torch

from gpu_util import to_gpu
from shaped_util import bounds, call, inputs, reference, shape_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scales", [[1.9375 * 2.0 ** -29], [1.9375 * 2.0 ** -29, 1.0625 * 2.0 ** -27, 1.5 * 2.0 ** -24],
                                    [1.99 * 2.0 ** -20, 1.37 * 2.0 ** -15, 1.21 * 2.0 ** -12], [1.7 * 2.0 ** -33, 1.3 * 2.0 ** -60],
                                    [1.9375 * 2.0 ** -14, 1.3 * 2.0 ** -9, 1.6, 33.7]])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_page_scales_of_any_significand(d, page, scales):
    """A slope of -50 makes a row return the visible value that is farthest from it: scores lie within 6 of 0, so
    the next key's weight is below e^-38."""
    print(f"\n[case] shaped small values {d} {page} {scales}", flush=True)
    w = inputs([900, 200, 333, 64], [40, 70, 1, 130], 2, 4, d, page, "fp8", seed=11, sharp=1.0)
    rng = np.random.default_rng(5)
    codes = rng.integers(0, 256, size=tuple(w.v_pool.shape))
    codes = np.where(codes % 128 == 127, 7, codes).astype(np.uint8)  # (0x7F and 0xFF are NaN)
    w.v_pool.copy_(torch.from_numpy(codes))
    w.v_scale.copy_(torch.from_numpy(rng.choice(scales, size=tuple(w.v_scale.shape)).astype(np.float32)))
    kw = shape_of(w, window=60)
    kw["slopes"] = np.full(8, -50.0, dtype=np.float32)
    dw = to_gpu(w)
    out = torch.full(dw.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    call(dw, kw, out=out)
    torch.cuda.synchronize()
    got = out.cpu().double().numpy()
    ref, lse, terms = reference(w, kw)
    assert terms["scores"].max() < 20.0  # (sums of magnitudes: the scores themselves reach 5.5)
    largest = max(448.0 * max(scales), w.v_new.abs().max().item())
    tol = bounds(w, kw, ref, lse, terms)[0] + 60 * 2.0 ** -54 * largest
    over = np.abs(got - ref) / tol
    print(f"[shaped small values {d} {page} {scales}] worst {over.max():.3f} of the tolerance", flush=True)
    assert np.isfinite(got).all() and over.max() <= 1.0
