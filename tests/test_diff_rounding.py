"""What the limit of test_gpu_diff_precision.py tells apart, in 64 bits on the CPU: results whose only
errors are the weights' rounding and the output's."""
import numpy as np
import pytest
import torch

import cw_workloads as cw
import oracle
from conftest import paged_inputs
from diff_rounding import singles_with_rounded_weights
from test_gpu_diff_precision import CASES, LIMIT


@pytest.mark.parametrize("dtype,terms,passes", [(torch.bfloat16, 1, False), (torch.bfloat16, 2, True), (torch.float16, 1, True)])
def test_the_limit_tells_one_bf16_weight_from_better_ones(dtype, terms, passes):
    lp, pairs, g, d, page = CASES[0]
    w = cw.materialize(cw.custom_spec(lp, [1] * len(lp), num_kv_heads=2 * pairs, gqa_group=g, head_dim=d, page_size=page, seed=8))
    lam = np.random.default_rng(8).uniform(0.2, 0.8, size=pairs * g).astype(np.float32)
    inp = paged_inputs(w)
    ref, _ = oracle.diff_attention(inp, lam)
    got = singles_with_rounded_weights(inp, lam, dtype, terms)
    relative = np.linalg.norm(got - ref) / np.linalg.norm(ref)
    print(dtype, terms, relative)
    assert (relative <= LIMIT) == passes
    assert relative <= 1.75e-3 or relative >= 2.1e-3  # not by a hair
