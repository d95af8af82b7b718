"""What the weights of the bf16 attention are divided by."""
import math

import pytest
import torch

from paged_util import attention_problem, call_attention

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
