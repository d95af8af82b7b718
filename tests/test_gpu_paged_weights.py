"""The weights of the bf16 attention: what they are divided by, and how many bits of them reach the values."""
import math

import numpy as np
import pytest
import torch

from gpu_util import to_f64_host
from paged_util import attention_problem, call_attention, oracle_outputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K,Hq", [(1, 2), (17, 2), (40, 2), (70, 2), (100, 4), (300, 2), (530, 2)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_the_mean_of_ones_is_one(gpu_lib, K, Hq, D, splits):
    """Values of one under any weights: numerator and divisor are the same sum of the rounded weights, so that their ratio is 1 within a few
    2^-24, which is 1 in bf16 (its neighbours are 2^-8 and 2^-7 away).  The first keys set the reference; the others' weights are
    2^m (1 + 2^-8) and a little less, which bf16 rounds down by nearly half a step: divided by the sum of the unrounded weights
    the result would be a step below 1."""
    s = attention_problem(61, "bf16", 2, Hq, 2, D, K, 16, [K + 900, K + 177], None, False)
    s["vp"].fill_(1.0)
    s["q"].zero_()
    s["q"][..., 0] = 1.0
    s["kp"].zero_()
    for b in range(2):
        held = s["table"][b, 128 // 16:-(-int(s["lens"][b]) // 16)].tolist()
        s["kp"][held, :, :, 0] = 1.0
    for m in (0, 3, 7):
        scale = (m + math.log2(1.0 + 0.97 * 2.0 ** -8)) / math.log2(math.e)
        for mask in (dict(), dict(causal=True), dict(causal=True, window=700, sinks=5)):
            assert (call_attention(gpu_lib, s, kv_splits=splits, scale=scale, **mask) == 1.0).all()


@pytest.mark.parametrize("Hq,K,lens", [(4, 1, [700, 33, 5]), (16, 1, [90, 2000]), (64, 1, [40, 700]), (8, 8, [19, 333]), (2, 30, [31, 50])])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("splits", [0, 3])
def test_up_to_32_rows_lose_only_the_rounding_of_the_output(gpu_lib, Hq, K, lens, D, splits):
    """With A = sum_j p_j |v_jd| / sum_j p_j: a weight is two bf16 numbers, the second off by half a step (2^-8) of what the first one, below it
    by up to a step (2^-7), leaves: 2^-15 of each; scores, exponentials and sums in fp32 1e-5 of each, as in the fp32 kernel (paged_util); the output half a step
    of bf16, 2^-8 |o|.  Weights of one bf16 number would be off by up to 2^-8 A."""
    s = attention_problem(62 + K, "bf16", len(lens), Hq, 2, D, K, 16, lens, None, False)
    for mask in (dict(), dict(causal=True, window=300, sinks=2)):
        got = to_f64_host(call_attention(gpu_lib, s, kv_splits=splits, **mask))
        want, want_abs = oracle_outputs(s, **mask)
        bound = 2.0 ** -8 * np.abs(want) + 2.0 * (2.0 ** -15 + 1e-5) * want_abs + 1e-6
        assert (np.abs(got - want) <= bound).all()


@pytest.mark.parametrize("Hq,K,n", [(4, 1, 700), (16, 1, 90), (8, 8, 333), (2, 30, 192)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_infinite_values_keep_their_sign(gpu_lib, Hq, K, n, D, splits):
    """Among keys that every row sees, where the weights are what they are and where they are powers of two."""
    s = attention_problem(63, "bf16", 1, Hq, 2, D, K, 16, [n], None, False)
    for j, value in ((0, float("inf")), (5, float("-inf")), (15, float("inf"))):
        t = dict(s, vp=s["vp"].clone())
        t["vp"][int(s["table"][0, 0]), :, j, j] = value
        for scale in (0.0, 1e-30):                           # 1e-30: all weights are one
            got = to_f64_host(call_attention(gpu_lib, t, kv_splits=splits, scale=scale))
            clean = to_f64_host(call_attention(gpu_lib, s, kv_splits=splits, scale=scale))
            assert (got[..., j] == value).all()
            got[..., j] = clean[..., j]
            assert np.array_equal(got, clean)
