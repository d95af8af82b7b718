"""Inputs of the paged operators for the GPU tests: pools whose unused rows hold NaN, tables whose unused entries are invalid."""
import numpy as np
import torch

from oracle.paged import paged_attention as oracle_attention
from gpu_util import to_f64_host


def dtype_of(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def make_tables(rng, lens, page_size, width=None, spare=3):
    """Block tables with each sequence's pages at random places of the pool; invalid ids (-1 and one far too large) elsewhere."""
    held = [-(-n // page_size) for n in lens]
    width = max(max(held), 1) + 1 if width is None else width
    n_pages = sum(held) + spare
    perm = rng.permutation(n_pages).astype(np.int32)
    table = np.where(np.arange(len(lens) * width).reshape(len(lens), width) % 2 == 0, -1, 2 ** 31 - 1).astype(np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = perm[at:at + h]
        at += h
    return table, perm[at:], n_pages


def fill_pool(g, table, lens, n_pages, Hkv, page_size, D, dtype, std=1.0):
    """[n_pages,Hkv,page_size,D]: normal draws in the rows that sequences hold, NaN everywhere else."""
    pool = torch.full((n_pages, Hkv, page_size, D), float("nan"), dtype=dtype, device="cuda")
    for b, n in enumerate(lens):
        for e in range(-(-n // page_size)):
            rows = min(page_size, n - e * page_size)
            if 0 <= table[b, e] < n_pages:
                pool[int(table[b, e]), :, :rows] = (torch.randn((Hkv, rows, D), generator=g, device="cuda") * std).to(dtype)
    return pool


def attention_problem(seed, dtype, B, Hq, Hkv, D, K, page_size, lens, q_lens=None, block=False, std=1.0):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = dtype_of(dtype)
    table, _, n_pages = make_tables(rng, lens, page_size)
    s = {"table": table, "lens": np.array(lens, dtype=np.int32), "q_lens": None if q_lens is None else np.array(q_lens, dtype=np.int32)}
    s["kp"] = fill_pool(g, table, lens, n_pages, Hkv, page_size, D, dt, std)
    s["vp"] = fill_pool(g, table, lens, n_pages, Hkv, page_size, D, dt)
    draw = lambda h, scale: (torch.randn((B, h, K, D), generator=g, device="cuda") * scale).to(dt)
    s["q"] = draw(Hq, std)
    s["kb"], s["vb"] = (draw(Hkv, std), draw(Hkv, 1.0)) if block else (None, None)
    if q_lens is not None:
        for b, n in enumerate(q_lens):
            for x in ("q", "kb", "vb"):
                if s[x] is not None:
                    s[x][b, :, n:] = float("nan")
    return s


SENTINEL = 7.0


def call_attention(sd, s, max_kv_len=None, out=None, **kw):
    dev = lambda x: None if x is None else torch.from_numpy(x).cuda()
    out = torch.full_like(s["q"], SENTINEL) if out is None else out
    sd.paged_attention(s["q"], s["kp"], s["vp"], dev(s["table"]), dev(s["lens"]),
                       int(max(s["lens"].max(), 0)) if max_kv_len is None else max_kv_len, k_block=s["kb"], v_block=s["vb"],
                       q_lens=dev(s["q_lens"]), out=out, **kw)
    torch.cuda.synchronize()
    return out


def oracle_outputs(s, **kw):
    f = lambda t: None if t is None else to_f64_host(t)
    kw.pop("kv_splits", None)
    fill = np.full(tuple(s["q"].shape), SENTINEL)
    args = (f(s["q"]), f(s["kp"]))
    rest = (s["table"], s["lens"])
    want = oracle_attention(*args, f(s["vp"]), *rest, f(s["kb"]), f(s["vb"]), s["q_lens"], out=fill, **kw)
    absv = lambda t: None if t is None else np.abs(f(t))
    want_abs = oracle_attention(*args, absv(s["vp"]), *rest, f(s["kb"]), absv(s["vb"]), s["q_lens"], out=fill, **kw)
    return want, want_abs


def error_ratio(got, want, want_abs, dtype):
    """Largest error over its bound (<= 1 passes).  With A = sum_j p_j |v_jd| / sum_j p_j:
    bf16: probabilities and output rounded to bf16 (2^-8 each; the sum's rounding likewise): 2^-8 (A + 2 |o|), 5 % and 1e-6 for
    the fp32 rest, as for the dense attention.
    fp32: a score is a sum of D products, |error| <= about sqrt(D) 2^-24 sum |q k| / sqrt(D) <= 4e-6 for unit draws, the
    exponential and the sums add a few 2^-24: relative error of a weight <= 1e-5, so 1e-5 (A + |o|) + 1e-6."""
    if dtype == "bf16":
        bound = 2.0 ** -8 * (want_abs + 2.0 * np.abs(want)) * 1.05 + 1e-6
    else:
        bound = 1e-5 * (want_abs + np.abs(want)) + 1e-6
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    return float((err / bound).max())


def check_attention(sd, s, dtype, max_kv_len=None, **kw):
    got = to_f64_host(call_attention(sd, s, max_kv_len, **kw))
    want, want_abs = oracle_outputs(s, **kw)
    if s["q_lens"] is not None:
        for b, n in enumerate(s["q_lens"]):
            assert (got[b, :, n:] == SENTINEL).all()
    ratio = error_ratio(got, want, want_abs, dtype)
    assert ratio <= 1.0, ratio
    return ratio
