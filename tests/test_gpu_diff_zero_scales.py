"""Differential attention of single new tokens over fp8 pages: pages whose V scale is 0 hold the large
weights, so the output is what far smaller weights of the other pages leave.

Tolerance as in test_gpu_diff_value_scales.py."""
import pytest

from test_gpu_diff_fp8_scores import _peaked
from test_gpu_diff_value_scales import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("halves", [[0, 1], [0], [1]])
@pytest.mark.parametrize("d,page", [(128, 16), (64, 16), (128, 64), (64, 64)])
def test_a_page_of_zeros_with_all_the_weight(d, page, halves):
    """Scores on one page some 22 above the others': the others' weights are e^-22 = 2^-32 of its."""
    print(f"\n[case] diff zero value scale under the weight, halves {halves} d={d} page={page}", flush=True)
    lp = [700, 333, 1500, 70]
    w, lam = _peaked(lp, [1] * 4, 2, 3, d, page, seed=23 + d, size=60.0)
    for b in range(4):
        pg = int(w.block_table[b, (lp[b] // page) // 2])
        w.k_scale[pg] *= 1.37
        for pair in range(2):
            for m in halves:
                w.v_scale[pg, 2 * pair + m] = 0.0
    _check(w, lam, f"zero under the weight {halves} {d} {page}")
