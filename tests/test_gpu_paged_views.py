"""GPU parity of paged attention on block tensors that are views with rows in unusual places."""
import pytest
import torch

from paged_util import attention_problem, call_attention, dtype_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,K,Hq", [("bf16", 5, 2), ("bf16", 130, 1), ("bf16", 70, 4), ("bf16", 200, 4), ("fp32", 40, 2)])
@pytest.mark.parametrize("D,steps", [(64, (16, 16)), (128, (8, 8)), (128, (120, 56)), (128, (128, 24)), (64, (8, 256))])
def test_block_rows_that_overlap(gpu_lib, dtype, K, Hq, D, steps):
    """Rows of a sliding view (each begins inside the one before), in keys, values or both: the same bits as of a dense copy."""
    s = attention_problem(41, dtype, 2, Hq, 1, D, K, 16, [75, 64], None, True)
    g = torch.Generator(device="cuda")
    g.manual_seed(41)
    for x, step in zip(("kb", "vb"), steps):
        line = torch.randn((2, K * step + D), generator=g, device="cuda").to(dtype_of(dtype))
        s[x] = torch.as_strided(line, (2, 1, K, D), (line.stride(0), line.stride(0), step, 1))
    dense = dict(s, kb=s["kb"].contiguous(), vb=s["vb"].contiguous())
    for mask in (dict(), dict(causal=True), dict(causal=True, window=50)):
        assert torch.equal(call_attention(gpu_lib, s, **mask), call_attention(gpu_lib, dense, **mask))
