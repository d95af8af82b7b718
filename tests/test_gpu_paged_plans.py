"""GPU parity at the borders between the ways in which the paged operators share out their work: rows per K/V head, keys, batch sizes;
other streams, calls side by side, workspaces that captured calls share.  Bounds as in paged_util."""
import numpy as np
import pytest
import torch

from gpu_util import to_f64_host
from oracle.paged import norm_rope as oracle_norm_rope, paged_extend as oracle_extend
from paged_util import attention_problem, call_attention, check_attention, error_ratio, make_tables, oracle_outputs, SENTINEL

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


# Rows per K/V head (Hq / Hkv * K) on both sides of 16, 32, 64, 128, 256 and 512, where kernels, tiles and shares change
@pytest.mark.parametrize("Hq,K", [(4, 8), (1, 17), (4, 16), (1, 33), (1, 64), (5, 13), (1, 128), (3, 43), (2, 128), (1, 257), (3, 171)])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_per_head(gpu_lib, Hq, K, D):
    lens = [K + 70, 0, K + 601, 333, K]
    s = attention_problem(K + Hq, "bf16", 5, 2 * Hq, 2, D, K, 16, lens, [K, K, K - K // 3, 1, 0], True)
    for mask in (dict(), dict(causal=True), dict(causal=True, window=90, sinks=3), dict(causal=True, kv_splits=3), dict(kv_splits=1)):
        check_attention(gpu_lib, s, "bf16", **mask)


# Keys on both sides of what one workgroup takes for itself
@pytest.mark.parametrize("dtype,n", [("bf16", 1024), ("bf16", 1025), ("bf16", 2049), ("fp32", 320), ("fp32", 321), ("fp32", 641)])
@pytest.mark.parametrize("D,page", [(64, 64), (128, 32)])
@pytest.mark.parametrize("K", [1, 3])
def test_keys_of_a_workgroup(gpu_lib, dtype, n, D, page, K):
    s = attention_problem(n + K, dtype, 3, 8, 2, D, K, page, [n, 1 if K == 1 else K, n // 2], None, False)
    for mask in (dict(causal=True), dict(window=100, sinks=5)):
        check_attention(gpu_lib, s, dtype, **mask)


# Units (sequences times K/V heads, in fp32 times 16-row tiles) on both sides of 256, 1024 and 4096
@pytest.mark.parametrize("dtype,B,Hkv,K,most", [("bf16", 127, 8, 1, 900), ("bf16", 128, 8, 1, 900), ("bf16", 130, 8, 2, 60), ("bf16", 513, 8, 1, 40),
                                                ("bf16", 1030, 1, 33, 40), ("bf16", 2100, 1, 40, 20), ("bf16", 70, 2, 140, 50),
                                                ("fp32", 32, 8, 1, 600), ("fp32", 31, 8, 1, 600), ("fp32", 33, 4, 17, 100), ("fp32", 520, 8, 1, 40)])
def test_large_batches(gpu_lib, dtype, B, Hkv, K, most):
    rng = np.random.default_rng(B)
    lens = np.maximum(rng.integers(0, most, B), K)
    lens[[0, B // 2]] = K, most
    s = attention_problem(B, dtype, B, Hkv, Hkv, 64, K, 16, lens.tolist(), None, False)
    check_attention(gpu_lib, s, dtype, causal=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K,Hq", [(1, 2), (48, 2), (90, 4)])
def test_windows_and_sinks_as_large_as_their_type(gpu_lib, dtype, K, Hq):
    """They hide nothing, also for rows in front of the first key."""
    s = attention_problem(21, dtype, 2, Hq, 2, 64, K, 16, [30, 40], None, False)
    top = 2 ** 31 - 1
    for causal in (False, True):
        want = call_attention(gpu_lib, s, causal=causal)
        for mask in (dict(window=top), dict(window=2 ** 30), dict(window=top, sinks=top), dict(window=1, sinks=top)):
            assert torch.equal(call_attention(gpu_lib, s, causal=causal, **mask), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K,Hq", [(5, 4), (16, 4), (17, 4), (40, 8), (150, 4)])
@pytest.mark.parametrize("splits", [0, 4])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(gpu_lib, dtype, K, Hq, splits):
    """In every kernel, also where a row's keys are shared out.  Rows that do not see the value: bit for bit the same.  The other columns of
    those that do: two results within the bound of paged_util, so twice that from one another."""
    s = attention_problem(22, dtype, 2, Hq, 2, 64, K, 16, [K + 400, K + 90], None, False)
    clean = to_f64_host(call_attention(gpu_lib, s, causal=True, kv_splits=splits))
    want_abs = oracle_outputs(s, causal=True)[1]
    for b, back, bad in ((0, 2, float("inf")), (1, K - 1, float("nan")), (0, K // 2, float("-inf"))):
        t = dict(s, vp=s["vp"].clone())
        j = int(s["lens"][b]) - 1 - back                   # position of row K - 1 - back
        t["vp"][int(s["table"][b, j // 16]), :, j % 16, 3] = bad
        got = to_f64_host(call_attention(gpu_lib, t, causal=True, kv_splits=splits))
        same = got == clean
        assert same[1 - b].all() and same[b, :, :K - 1 - back].all()
        assert not np.isfinite(got[b, :, K - 1 - back:, 3]).any()
        got[..., 3] = clean[..., 3]
        assert error_ratio(got, clean, want_abs, dtype) <= 2.0


@pytest.mark.parametrize("K,Hq,stride", [(40, 4, 64 * 8), (300, 1, 64 * 8), (70, 2, 1 << 26), (33, 2, (1 << 26) + 64)])
def test_block_rows_far_apart(gpu_lib, K, Hq, stride):
    """Block rows at a projection's distance, and at one whose bytes pass 32 bits (rows of a view over a large tensor)."""
    s = attention_problem(23, "bf16", 1, Hq, 1, 64, K, 16, [75], None, True)
    want = call_attention(gpu_lib, s)
    base = torch.empty((K - 1) * stride + 64, dtype=BF16, device="cuda") if stride >= 1 << 26 else torch.empty(K * stride, dtype=BF16, device="cuda")
    views = {}
    for x in ("kb", "vb"):
        big = base if x == "kb" else torch.empty_like(base)
        v = torch.as_strided(big, (1, 1, K, 64), (stride, stride, stride, 1))
        v.copy_(s[x])
        views[x] = v
    assert torch.equal(call_attention(gpu_lib, dict(s, **views)), want)


@pytest.mark.parametrize("dtype,K", [("bf16", 1), ("bf16", 50), ("fp32", 3)])
def test_on_another_stream_and_side_by_side(gpu_lib, dtype, K):
    """Calls on two streams at the same time, each with tensors of its own, and a workspace made by the call."""
    problems = [attention_problem(24 + i, dtype, 3, 8, 2, 128, K, 16, [4000, 3 + K, 900 + 400 * i], None, False) for i in range(2)]
    want = [call_attention(gpu_lib, s, causal=True) for s in problems]
    args = [[s["q"], s["kp"], s["vp"], dev(s["table"]), dev(s["lens"]), 4000] for s in problems]
    outs = [[torch.full_like(s["q"], SENTINEL) for _ in range(8)] for s in problems]
    want = [gpu_lib.paged_attention(*a, causal=True) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in problems]
    for i in range(8):
        for a, o, st in zip(args, outs, streams):
            gpu_lib.paged_attention(*a, causal=True, out=o[i], stream=st)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(x, w) for x in o)


def test_captured_calls_that_share_a_workspace(gpu_lib):
    """Two graphs on one stream whose calls were bound to the same workspace, replayed in turn with eager calls between."""
    sd = gpu_lib
    sd.init()
    cases = [("bf16", 1, 2), ("bf16", 40, 4), ("fp32", 2, 2)]
    problems = [attention_problem(30 + i, dt, 2, 2 * g, 2, 128, K, 16, [3000, 1700], None, False) for i, (dt, K, g) in enumerate(cases)]
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    graphs, outs, want = [], [], []
    for s in problems:
        a = [s["q"], s["kp"], s["vp"], dev(s["table"]), dev(s["lens"]), 3000]
        want.append(sd.paged_attention(*a, causal=True))
        outs.append(torch.full_like(s["q"], SENTINEL))
        torch.cuda.synchronize()
        call = sd.bind_paged_attention(*a, causal=True, out=outs[-1], workspace=ws, stream=side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
            call()
        graphs.append((g, call))
    for turn in range(4):
        for (g, call), o, w in zip(graphs, outs, want):
            o.fill_(SENTINEL)
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                g.replay()
                ws[:1024].fill_(turn)
                call() if turn % 2 else None
            torch.cuda.synchronize()
            assert torch.equal(o, w)


def test_extend_gives_back_long_sequences(gpu_lib):
    """More pages of a sequence than a wave's loads take in one go, and a stack too small for all of them."""
    rng = np.random.default_rng(31)
    lens = np.array([20000, 3, 8192, 8193, 16 * 511, 0], dtype=np.int32)
    B, K, page = len(lens), 5, 16
    table, spare, n_pages = make_tables(rng, lens, page, 1400, spare=20)
    release = np.array([1, 1, 0, 1, 1, 1], dtype=np.uint8)
    for pool in (n_pages, 1500):
        stack = np.full(pool, -1, dtype=np.int32)
        stack[:20] = spare[:20]
        want = oracle_extend(table, lens, stack, 20, page, K, release=release)
        d = [dev(x) for x in (table, lens, stack, np.array([20], dtype=np.int32))]
        slots, granted, lens_out, n_out = gpu_lib.paged_extend(*d, page, K, release=dev(release))
        torch.cuda.synchronize()
        got = [d[0], lens_out, d[2], n_out, slots, granted]
        for x, y in zip(got, want):
            assert np.array_equal(x.cpu().numpy().reshape(-1), np.asarray(y).reshape(-1))


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_of_many_rows(gpu_lib, dtype, interleaved):
    """More bytes than the caches hold are stored another way; the parts of the batch by themselves are not: the same bits."""
    B, K, Hq, Hkv, D, page = 2, 4100 if dtype == BF16 else 2050, 14, 2, 128, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(32)
    q, k, v = (torch.randn((B, K, h, D), generator=g, device="cuda").to(dtype).transpose(1, 2) for h in (Hq, Hkv, Hkv))
    w = torch.randn((D,), generator=g, device="cuda").to(dtype)
    pos = torch.tensor([5, 70000], dtype=torch.int32, device="cuda")
    slots = torch.randperm(B * K, generator=g, device="cuda").to(torch.int32).view(B, K)
    n_pages = -(-B * K // page)
    run = lambda at, kp, vp: gpu_lib.qk_norm_rope(q[:, :, at], k[:, :, at], pos + at.start, 1e4, w, w, interleaved=interleaved, v=v[:, :, at],
                                                  k_pages=kp, v_pages=vp, slots=slots[:, at].contiguous())[0]
    pools = [torch.zeros((n_pages, Hkv, page, D), dtype=dtype, device="cuda") for _ in range(4)]
    whole = run(slice(0, K), *pools[:2])
    for t in range(0, K, 500):
        at = slice(t, min(t + 500, K))
        assert torch.equal(run(at, *pools[2:]), whole[:, :, at])
    assert torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])


def test_positions_that_pass_31_bits(gpu_lib):
    """The first row's position fits the type, later ones need not.  Angles of 2^31 rad in double are off by 2^-53 2^31 = 2.4e-7 in the
    oracle and in the kernel, 5e-7 together; the rest of a row's error is at most 2.1e-6 of the pair's sum (|q| <= 6: 12)."""
    B, K, H, D = 2, 9, 3, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(33)
    q = torch.randn((B, H, K, D), generator=g, device="cuda").clamp(-6, 6)
    start = np.array([2 ** 31 - 4, -5], dtype=np.int32)
    got, _ = gpu_lib.qk_norm_rope(q, q.clone(), dev(start), 1e4, eps=0.0, interleaved=True)
    want = oracle_norm_rope(to_f64_host(q), None, start[:, None].astype(np.int64) + np.arange(K)[None], 1e4, interleaved=True)
    assert np.abs(to_f64_host(got) - want).max() <= (2.1e-6 + 5e-7) * 12


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_largest_scale(gpu_lib, dtype):
    """Weights of one and zero: the value of the key with the largest score."""
    s = attention_problem(34, dtype, 2, 4, 2, 64, 2, 16, [90, 40], None, False)
    check_attention(gpu_lib, s, dtype, scale=0.99e38)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K,Hq", [(1, 2), (9, 4), (20, 4), (50, 4), (150, 4)])
@pytest.mark.parametrize("page", [16, 32])
def test_holes_in_long_tables(gpu_lib, dtype, K, Hq, page):
    """Entries that are no pages on both sides of every 64th entry, alone and in runs, and behind the last one."""
    s = attention_problem(35, dtype, 2, Hq, 2, 64, K, page, [3300, 1100], None, True)
    for b, holes in ((0, [0, 1, 31, 62, 63, 64, 65, 66, 100, 127, 128, 192, 206]), (1, [33, 34, 35, 36, 63, 64])):
        for e in holes:
            if e < s["table"].shape[1]:
                s["table"][b, e] = -1 if e % 2 else s["kp"].shape[0] + e
    for mask in (dict(), dict(causal=True), dict(causal=True, window=1500, sinks=1100), dict(kv_splits=5)):
        check_attention(gpu_lib, s, dtype, **mask)


def test_append_of_many_rows(gpu_lib):
    """More bytes than the caches hold are read another way; the layers one by one are not: the same pages."""
    L, B, K, Hkv, D, page = 8, 4, 256, 32, 128, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(36)
    k, v = (torch.randn((L, B, Hkv, K, D), generator=g, device="cuda").to(BF16) for _ in range(2))
    n_pages = B * (K // page + 1) + 1
    slots = torch.randperm(n_pages * page, generator=g, device="cuda")[:B * K].to(torch.int32).view(B, K)
    slots[1, ::3] = -1
    whole = [torch.zeros((L, n_pages, Hkv, page, D), dtype=BF16, device="cuda") for _ in range(2)]
    parts = [torch.zeros_like(x) for x in whole]
    gpu_lib.paged_kv_append(*whole, k, v, slots)
    for l in range(L):
        gpu_lib.paged_kv_append(parts[0][l:l + 1], parts[1][l:l + 1], k[l:l + 1], v[l:l + 1], slots)
    assert torch.equal(whole[0], parts[0]) and torch.equal(whole[1], parts[1])
    at = slots[0].long()
    assert torch.equal(whole[0][:, at // page, :, at % page], k[:, 0].permute(2, 0, 1, 3)) and whole[1].abs().sum() > 0
