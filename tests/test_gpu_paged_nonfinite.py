"""Infinities and NaN among the values: which elements of the output they reach, with which sign, and that nothing else changes."""
import time

import numpy as np
import pytest
import torch

from gpu_util import to_f64_host
from paged_util import attention_problem, call_attention, oracle_outputs

pytestmark = pytest.mark.gpu


def reached(s, bad, causal=False, window=0, sinks=0):
    """The sum of the values that are not finite over the keys that each row sees (NaN where they cancel), zero where it sees none.
    bad: [B,Hkv,N,D] of the cached rows and, behind them, the block's."""
    B, Hq, K, D = s["q"].shape
    n_pages, Hkv, page = s["kp"].shape[:3]
    out = np.zeros((B, Hq, K, D))
    for b in range(B):
        n, q = int(s["lens"][b]), K if s["q_lens"] is None else int(s["q_lens"][b])
        total = n + (q if s["kb"] is not None else 0)
        j = np.arange(total)
        here = np.array([x >= n or 0 <= s["table"][b, x // page] < n_pages for x in j])
        for r in range(q):
            p = total - q + r
            seen = here & ((j <= p) | (not causal))
            if window:
                seen &= (p - j < window) | (j < sinks)
            with np.errstate(invalid="ignore"):
                add = bad[b][:, :total][:, seen].sum(1)
            out[b, :, r] = np.repeat(add, Hq // Hkv, 0)
    return out


CASES = [("bf16", 4, 4), ("bf16", 9, 4), ("bf16", 40, 2), ("bf16", 60, 4), ("bf16", 150, 4), ("fp32", 3, 4), ("fp32", 40, 4)]


@pytest.mark.parametrize("dtype,K,Hq", CASES)
@pytest.mark.parametrize("mask", [dict(causal=True), dict(causal=True, window=40, sinks=9), dict(window=30), dict()],
                         ids=lambda m: "-".join(f"{k}{int(v)}" for k, v in m.items()) or "all")
@pytest.mark.parametrize("share", [0.0005, 0.02])
@pytest.mark.parametrize("block", [False, True])
def test_where_they_arrive(gpu_lib, dtype, K, Hq, mask, share, block):
    """Draws of +inf, -inf and NaN over the cached rows and the block, holes in the table; keys shared out or not."""
    s = attention_problem(71 + K, dtype, 2, Hq, 2, 64, K, 16, [K + 300, K + 17], [K, K - K // 3], block)
    s["table"][0, 3] = -1
    s["table"][1, 1] = s["kp"].shape[0]
    rng = np.random.default_rng(71)
    n_pages, Hkv, page, D = s["vp"].shape
    kinds = np.array([np.inf, -np.inf, np.nan])
    draw = lambda shape: np.where(rng.random(shape) < share, kinds[rng.integers(0, 3, shape)], 0.0)
    pool, rows = draw((n_pages, Hkv, page, D)), draw((2, Hkv, K, D))
    dev = lambda x, like: torch.where(torch.from_numpy(x).cuda() != 0, torch.from_numpy(x).cuda().to(like.dtype), like)
    zero = lambda x, like: torch.where(torch.from_numpy(x).cuda() != 0, torch.zeros_like(like), like)
    bad = np.zeros((2, Hkv, int(max(s["lens"])) + K, D))
    for b in range(2):
        n = int(s["lens"][b])
        for j in range(n):
            if 0 <= s["table"][b, j // page] < n_pages:
                bad[b, :, j] = pool[s["table"][b, j // page], :, j % page]
        bad[b, :, n:n + K] = rows[b]
    add = reached(s, bad, **mask)
    t, clean = dict(s, vp=dev(pool, s["vp"])), dict(s, vp=zero(pool, s["vp"]))
    if block:
        t["vb"], clean["vb"] = dev(rows, s["vb"]), zero(rows, s["vb"])
    want, want_abs = oracle_outputs(clean, **mask)
    step = 2.0 ** -8 if dtype == "bf16" else 1e-5
    for splits in (0, 1, 3):
        got = to_f64_host(call_attention(gpu_lib, t, kv_splits=splits, **mask))
        finite = add == 0
        assert (np.abs(got - want)[finite] <= (step * 1.05 * (want_abs + 2 * np.abs(want)) + 1e-6)[finite]).all()
        assert np.array_equal(got[~finite], add[~finite], equal_nan=True)
    assert (add != 0).any()


def test_they_cost_the_same_at_any_length(gpu_lib):
    """What they are looked for and added in are the tiles that rows see in part; the others are not read again."""
    for K, Hq, n in ((300, 8, 60000), (40, 4, 60000), (4, 8, 60000)):
        s = attention_problem(72, "bf16", 1, Hq, 2, 128, K, 64, [n], None, False)
        call_attention(gpu_lib, s, causal=True, kv_splits=1)
        times = []
        for bad in (False, True):
            if bad:
                s["vp"][int(s["table"][0, (n - K // 2) // 64]), :, (n - K // 2) % 64, 5] = float("inf")
            t0 = time.perf_counter()
            call_attention(gpu_lib, s, causal=True, kv_splits=1)
            times.append(time.perf_counter() - t0)
        # the one workgroup or wave of a head takes a few ms; with every row over every key again it would be hundreds
        assert times[1] < times[0] + 0.05, times
