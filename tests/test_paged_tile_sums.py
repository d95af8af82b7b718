"""The kernels add up the key tiles of 64 sequences (or row tiles of sequences) at a time in 32 bits.  Where that many could have more, keys
are not shared out: no workspace.  No GPU: the plan is a function of the parameters."""
import ctypes

import pytest

import paper_2601_17917_amd as sd

BASE = dict(Hq=1, Hkv=1, D=64, K=1, page_size=1024, n_pages=1 << 20)


def need(**change):
    p = sd.PagedAttnParams(**dict(BASE, max_pages=change["max_kv_len"] // 1024 + 1, **change))
    n = sd.load_library().sdllm_paged_attention_workspace_bytes(ctypes.byref(p), 0)
    assert n != ctypes.c_size_t(-1).value, sd.load_library().sdllm_last_error()
    return n


# 16 keys in a tile (fp32), 32 (bf16, 128 wide) or 64; entries: sequences, or in fp32 the 16-row tiles of sequences.  (max_kv_len + K reaches 2^30.)
TOO_MANY = [dict(dtype=sd.FP32, B=1, K=1024, max_kv_len=1 << 29), dict(dtype=sd.FP32, B=1, K=700, max_kv_len=(1 << 30) - 700),
            dict(dtype=sd.FP32, B=1, K=3000, max_kv_len=1 << 29, D=128), dict(dtype=sd.FP32, B=64, max_kv_len=1 << 29),
            dict(dtype=sd.FP32, B=33, max_kv_len=(1 << 30) - 1), dict(dtype=sd.FP32, B=2, K=500, max_kv_len=1 << 29),
            dict(dtype=sd.BF16, B=64, D=128, max_kv_len=(1 << 30) - 1), dict(dtype=sd.BF16, B=90, D=128, max_kv_len=(1 << 30) - 1)]
FEW_ENOUGH = [dict(dtype=sd.FP32, B=1, K=1008, max_kv_len=(1 << 29) - 1008), dict(dtype=sd.FP32, B=1, K=1024, max_kv_len=1 << 28),
              dict(dtype=sd.FP32, B=1, K=1024, max_kv_len=1 << 29, causal=1, window=4096, sinks=4), dict(dtype=sd.FP32, B=1, max_kv_len=(1 << 30) - 1),
              dict(dtype=sd.FP32, B=31, max_kv_len=(1 << 30) - 1), dict(dtype=sd.BF16, B=63, D=128, max_kv_len=(1 << 30) - 1),
              dict(dtype=sd.BF16, B=64, D=128, max_kv_len=(1 << 30) - 33), dict(dtype=sd.BF16, B=64, max_kv_len=(1 << 30) - 1),
              dict(dtype=sd.BF16, B=64, K=40, max_kv_len=(1 << 30) - 40)]


@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("change", TOO_MANY, ids=str)
def test_sums_that_32_bits_do_not_hold_are_not_formed(change, splits):
    assert need(kv_splits=splits, **change) == 0


@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("change", FEW_ENOUGH, ids=str)
def test_keys_are_shared_out_up_to_there(change, splits):
    assert need(kv_splits=splits, **change) > 0
