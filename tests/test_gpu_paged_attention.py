"""GPU parity: sdllm_paged_attention against the fp64 oracle.  Rows that no sequence holds are NaN and table entries that no
sequence uses are invalid ids in every case, so that a read of either shows."""
import numpy as np
import pytest
import torch

from gpu_util import to_f64_host
from paged_util import attention_problem, call_attention, check_attention, oracle_outputs, SENTINEL

pytestmark = pytest.mark.gpu

SHAPES = [
    # B, Hq, Hkv, D, K, page, lens, q_lens, block
    (1, 4, 4, 128, 1, 16, [1], None, False),
    (1, 8, 2, 128, 1, 16, [700], None, False),
    (4, 8, 2, 64, 1, 16, [1, 15, 16, 17], None, False),
    (5, 8, 1, 128, 1, 32, [31, 32, 33, 500, 64], None, False),
    (3, 16, 1, 128, 1, 64, [0, 63, 1025], None, False),                  # an empty sequence
    (2, 32, 1, 64, 1, 128, [129, 127], None, False),
    (2, 6, 2, 128, 3, 16, [40, 3], [3, 2], False),                       # a few rows, the cache holds them
    (3, 4, 2, 128, 5, 16, [0, 33, 100], [5, 0, 1], True),                # a sequence without queries
    (2, 4, 4, 128, 32, 32, [96, 145], None, True),                       # blocks
    (2, 7, 1, 64, 27, 16, [7, 301], [27, 13], True),
    (1, 28, 4, 128, 32, 64, [450], None, True),
    (2, 2, 1, 128, 131, 16, [50, 260], [131, 77], True),                 # a prompt's piece
    (1, 3, 3, 64, 70, 256, [70], None, False),
]
MASKS = [dict(), dict(causal=True), dict(causal=True, window=20), dict(causal=True, window=33, sinks=4), dict(window=40, sinks=70),
         dict(causal=True, window=1)]


@pytest.mark.parametrize("mask", MASKS, ids=lambda m: "-".join(f"{k}{int(v)}" for k, v in m.items()) or "all")
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "B%d_%d_%d_D%d_K%d_page%d" % s[:6])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_shapes_and_masks(gpu_lib, dtype, shape, mask):
    B, Hq, Hkv, D, K, page, lens, q_lens, block = shape
    s = attention_problem(len(lens) + K, dtype, B, Hq, Hkv, D, K, page, lens, q_lens, block)
    check_attention(gpu_lib, s, dtype, **mask)


@pytest.mark.parametrize("splits", [1, 2, 3, 7, 64])
@pytest.mark.parametrize("dtype,K,Hq", [("bf16", 1, 4), ("bf16", 1, 40), ("bf16", 50, 4), ("fp32", 1, 4), ("fp32", 9, 4)])
def test_any_number_of_parts(gpu_lib, dtype, K, Hq, splits):
    s = attention_problem(11, dtype, 3, Hq, 2, 128, K, 16, [1000, 30 + K, 401], None, False)
    for mask in (dict(causal=True), dict(causal=True, window=300, sinks=17)):
        check_attention(gpu_lib, s, dtype, kv_splits=splits, **mask)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K,block", [(1, False), (1, True), (40, True)])
def test_plan_for_longer_sequences_than_there_are(gpu_lib, dtype, K, block):
    """The plan is made for max_kv_len; the lengths are device data and may be far below it.  Lengths above it are cut."""
    s = attention_problem(12, dtype, 4, 8, 2, 128, K, 64, [90, 64, 512, 41], None, block)
    s["table"] = np.pad(s["table"], ((0, 0), (0, 600)), constant_values=-1)
    check_attention(gpu_lib, s, dtype, max_kv_len=30000, causal=True)
    cut = dict(s, lens=np.minimum(s["lens"], 70))
    got = to_f64_host(call_attention(gpu_lib, s, max_kv_len=70))
    assert np.array_equal(got, to_f64_host(call_attention(gpu_lib, cut, max_kv_len=70)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K,Hq", [(1, 4), (1, 2), (33, 4)])
def test_pages_that_are_not_there_are_hidden(gpu_lib, dtype, K, Hq):
    """Entries outside the pool hide their keys: given back behind the window, or wrong."""
    s = attention_problem(13, dtype, 3, Hq, 2, 128, K, 16, [200, 100, 50], None, True)
    for e in (0, 3, 4, 5, 12):
        s["table"][0, e] = -1
    s["table"][1, 2] = s["kp"].shape[0]
    s["table"][2, :] = 2 ** 31 - 1
    for mask in (dict(), dict(causal=True, window=70)):
        check_attention(gpu_lib, s, dtype, **mask)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K,Hq", [(1, 4), (48, 4)])
def test_rows_that_see_nothing_are_zero(gpu_lib, dtype, K, Hq):
    s = attention_problem(14, dtype, 2, Hq, 2, 64, K, 16, [0, 0], None, False)
    assert (call_attention(gpu_lib, s) == 0).all()
    assert (call_attention(gpu_lib, s, max_kv_len=16) == 0).all()
    s = attention_problem(14, dtype, 2, Hq, 2, 64, K, 16, [30, 40], None, False)      # K = 48: the first rows lie before the first key
    check_attention(gpu_lib, s, dtype, causal=True)
    s["table"][:] = -1
    assert (call_attention(gpu_lib, s) == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K", [4, 16, 70])
def test_what_hidden_rows_hold_does_not_matter(gpu_lib, dtype, K):
    """Infinities and NaN in keys and values that only later rows see, or none."""
    s = attention_problem(15, dtype, 1, 4, 2, 128, K, 16, [100], None, True)
    clean = to_f64_host(call_attention(gpu_lib, s, causal=True, window=50))
    for x, bad in (("kb", float("nan")), ("vb", float("nan")), ("vb", float("inf")), ("kb", float("-inf"))):
        t = dict(s, **{x: s[x].clone()})
        t[x][0, :, K - 2] = bad
        got = to_f64_host(call_attention(gpu_lib, t, causal=True, window=50))
        assert np.array_equal(got[:, :, :K - 2], clean[:, :, :K - 2])
        assert not np.isfinite(got[:, :, K - 2]).all() or bad == float("-inf")
    t = dict(s, kp=s["kp"].clone(), vp=s["vp"].clone())
    page, row = s["table"][0, 20 // 16], 20 % 16                                       # key 20: outside every row's window
    t["kp"][page, :, row] = float("nan")
    t["vp"][page, :, row] = float("inf")
    assert np.array_equal(to_f64_host(call_attention(gpu_lib, t, causal=True, window=50)), clean)


def test_large_scores_and_scales(gpu_lib):
    for dtype in ("bf16", "fp32"):
        for K, lens in ((1, [300, 20]), (40, [300, 60])):
            s = attention_problem(16, dtype, 2, 4, 2, 128, K, 16, lens, None, False)
            check_attention(gpu_lib, s, dtype, scale=0.01)
            # keys of equal rows: the mean of the values, whatever the score
            s["kp"][:] = 3.0e4
            s["q"][:] = 1.0e4
            got = to_f64_host(call_attention(gpu_lib, s))
            want, want_abs = oracle_outputs(s)
            assert (np.abs(got - want) <= (2.0 ** -7 if dtype == "bf16" else 1e-5) * (want_abs + 1e-3)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K", [1, 6, 50])
def test_strided_queries_blocks_and_outputs(gpu_lib, dtype, K):
    """q, k, v as one projection leaves them (row per token, heads side by side), the output in the same order."""
    s = attention_problem(17, dtype, 2, 6, 2, 64, K, 16, [80, 33], None, True)
    want = call_attention(gpu_lib, s, causal=True)
    rows = torch.cat([s["q"], s["kb"], s["vb"]], 1).transpose(1, 2).contiguous()       # [B, K, heads, D]
    q, kb, vb = (x.transpose(1, 2) for x in rows.split([6, 2, 2], 2))
    out = torch.full((2, K, 6, 64), SENTINEL, dtype=q.dtype, device="cuda").transpose(1, 2)
    got = call_attention(gpu_lib, dict(s, q=q, kb=kb, vb=vb), out=out, causal=True)
    assert torch.equal(got, want)


def test_same_results_every_time(gpu_lib):
    s = attention_problem(18, "bf16", 5, 16, 2, 128, 1, 16, [3000, 17, 800, 1, 2100], None, False)
    first = call_attention(gpu_lib, s)
    for _ in range(3):
        assert torch.equal(call_attention(gpu_lib, s), first)


def test_offsets_beyond_32_bits(gpu_lib):
    """A pool of 8 GB per tensor whose last pages are in use: byte and element offsets pass 2^32 and 2^31."""
    Hkv, D, page = 8, 128, 256
    n_pages = (1 << 32) // (Hkv * page * D) + 40
    lens, K = [300, 700], 1
    kp = torch.zeros((n_pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    table = np.array([[n_pages - 1, n_pages - 3, 0], [n_pages - 2, 5, n_pages - 9]], dtype=np.int32)
    small = attention_problem(19, "bf16", 2, 16, Hkv, D, K, page, lens, None, False)
    for b in range(2):
        for e in range(-(-lens[b] // page)):
            kp[int(table[b, e])] = small["kp"][int(small["table"][b, e])]
            vp[int(table[b, e])] = small["vp"][int(small["table"][b, e])]
    got = call_attention(gpu_lib, dict(small, kp=kp, vp=vp, table=table), causal=True)
    assert torch.equal(got, call_attention(gpu_lib, small, causal=True))
