"""Sizes at the limits of the paged attention: what is refused, and that the plans' workspaces stay within bounds.  No GPU: parameters
are checked before anything is launched."""
import ctypes

import pytest

import paper_2601_17917_amd as sd

INVALID = ctypes.c_size_t(-1).value
BASE = dict(dtype=sd.BF16, B=1, Hq=1, Hkv=1, D=64, K=1, page_size=16, n_pages=1 << 20, max_pages=1 << 12, max_kv_len=1 << 16)


def need(with_block=0, **change):
    p = sd.PagedAttnParams(**dict(BASE, **change))
    return sd.load_library().sdllm_paged_attention_workspace_bytes(ctypes.byref(p), with_block)


@pytest.mark.parametrize("change", [
    dict(B=1 << 22), dict(B=1 << 21, Hq=2, Hkv=2), dict(B=1 << 10, Hq=1 << 10, K=1 << 8), dict(K=1 << 28), dict(Hq=1 << 14, K=1 << 14),
    dict(K=(1 << 30) - (1 << 16) + 1),
])
def test_too_large(change):
    assert need(**change) == INVALID
    assert b"too large" in sd.load_library().sdllm_last_error()


@pytest.mark.parametrize("dtype", [sd.BF16, sd.FP32])
@pytest.mark.parametrize("change", [
    dict(B=(1 << 22) - 1, max_pages=1, max_kv_len=16), dict(B=1 << 10, Hq=1 << 10, Hkv=1, K=255), dict(B=4, Hq=8, Hkv=8, K=1 << 20),
    dict(max_pages=1 << 25, max_kv_len=1 << 29, n_pages=1 << 26), dict(B=60, Hq=64, Hkv=8, K=2048, max_pages=1 << 20, max_kv_len=1 << 24),
])
@pytest.mark.parametrize("splits", [0, 1, 5, 2 ** 31 - 1])
def test_workspaces_at_the_limits(dtype, change, splits):
    """At most a partial result of D + 2 floats for every row that 2^20 workgroups of 256 rows can have, nothing where keys are not shared out."""
    n = need(dtype=dtype, kv_splits=splits, **change)
    assert n != INVALID and n <= (1 << 28) * (64 + 2) * 4
    if splits == 1:
        assert n == 0


@pytest.mark.parametrize("scale", [1.01e38, 3.4e38])
def test_scales_whose_product_with_log2_e_is_no_number(scale):
    assert need(scale=scale) == INVALID
    assert b"scale" in sd.load_library().sdllm_last_error()
    assert need(scale=0.99e38) != INVALID
