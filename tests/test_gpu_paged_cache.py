"""GPU parity: sdllm_paged_extend (integers, equal), sdllm_paged_kv_append (bit for bit) and sdllm_qk_norm_rope against the
oracle, and all four paged operators together in a serving loop, eagerly and as a replayed graph."""
import numpy as np
import pytest
import torch

from gpu_util import to_f64_host
from oracle.paged import norm_rope, paged_attention as oracle_attention, paged_extend as oracle_extend
from paged_util import dtype_of, error_ratio, make_tables

pytestmark = pytest.mark.gpu


def dev(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _extend_both(sd, table, lens, stack, top, page, K, in_place=True, **kw):
    want = oracle_extend(table, lens, stack, top, page, K, **kw)
    t, l, s, n = dev(table), dev(lens), dev(stack), dev(np.array([top], dtype=np.int32))
    outs = {} if in_place else dict(kv_lens_out=torch.empty_like(l), n_free_out=torch.empty_like(n))
    slots, granted, lo, no = sd.paged_extend(t, l, s, n, page, K, **{k: dev(v) for k, v in kw.items()}, **outs)
    torch.cuda.synchronize()
    got = (t, lo, s, no, slots, granted)
    for name, g, w in zip(("table", "lens", "stack", "n_free", "slots", "granted"), got, want):
        assert (g.cpu().numpy().reshape(-1) == np.asarray(w).reshape(-1)).all(), name
    if not in_place:
        assert (l.cpu().numpy() == lens).all() and n.item() == top
    return [x.cpu().numpy() for x in got]


@pytest.mark.parametrize("B,K,page,most", [(1, 1, 16, 100), (8, 1, 16, 4000), (64, 4, 32, 500), (65, 1, 16, 90), (300, 3, 16, 700),
                                           (1025, 1, 64, 3000), (2100, 7, 16, 100), (3, 5461, 128, 9000), (3, 5462, 128, 9000),
                                           (40, 700, 256, 20000), (5, 4097, 1024, 1)])
def test_extend(gpu_lib, B, K, page, most):
    rng = np.random.default_rng(B + K)
    lens = rng.integers(0, most + 1, B).astype(np.int32)
    new = rng.integers(0, K + 1, B).astype(np.int32)
    width = -(-(most + K) // page)
    table, spare, n_pages = make_tables(rng, lens, page, width, spare=B * (-(-K // page) + 1))
    stack = np.full(n_pages, -1, dtype=np.int32)
    stack[:len(spare)] = spare
    full = len(spare)
    flags = lambda share: (rng.random(B) < share).astype(np.uint8)
    for in_place in (True, False):
        _extend_both(gpu_lib, table, lens, stack, full, page, K, in_place)
        _extend_both(gpu_lib, table, lens, stack, full, page, K, in_place, new_lens=new)
        _extend_both(gpu_lib, table, lens, stack, full, page, K, in_place, new_lens=new, do_append=flags(0.5), release=flags(0.3))
        few = min(full, B // 3)                                                  # the pool runs out
        _extend_both(gpu_lib, table, lens, stack, few, page, K, in_place, new_lens=new, release=flags(0.1))
        _extend_both(gpu_lib, table, lens, stack, 0, page, K, in_place, release=np.ones(B, dtype=np.uint8))


def test_extend_values_out_of_range(gpu_lib):
    """Lengths and counts out of range are clamped, a sequence longer than its table row gets nothing, ids outside the pool give
    slot -1."""
    table = np.array([[3, -5, 7, 1], [0, 2, 99, -1], [-1, -1, -1, -1]], dtype=np.int32)
    stack = np.array([4, 77, 5, 6, -1, -1, -1, -1], dtype=np.int32)
    for lens, top, kw in (([62, 40, -9], 4, {}), ([100, 2 ** 31 - 1, 0], 4, {}), ([0, 0, 0], 900, {}), ([0, 0, 0], -3, {}),
                          ([10, 40, 0], 4, dict(new_lens=np.array([-4, 9000, 3], dtype=np.int32))),
                          ([10, 64, 0], 7, dict(release=np.array([0, 1, 0], dtype=np.uint8)))):
        _extend_both(gpu_lib, table, np.array(lens, dtype=np.int32), stack, top, 16, 5, **kw)


def test_extend_over_many_steps(gpu_lib):
    """A pool in use for a long time: the device state after each step is the next step's input."""
    rng = np.random.default_rng(5)
    B, width, page, n_pages = 70, 12, 16, 400
    table, lens = np.full((B, width), -1, dtype=np.int32), np.zeros(B, dtype=np.int32)
    stack, top = rng.permutation(n_pages).astype(np.int32), n_pages
    for step in range(60):
        table, lens, stack, n, _, _ = _extend_both(gpu_lib, table, lens, stack, top, page, 40, release=(rng.random(B) < 0.2).astype(np.uint8),
                                                   new_lens=rng.integers(0, 41, B).astype(np.int32))
        top = int(n[0])
        held = [int(p) for b in range(B) for p in table[b, :-(-lens[b] // page)]]
        assert sorted(held + stack[:top].tolist()) == list(range(n_pages))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("L,B,Hkv,K,D,page", [(1, 1, 1, 1, 64, 16), (2, 3, 4, 27, 128, 16), (3, 2, 2, 33, 96, 64), (32, 4, 8, 1, 128, 16),
                                              (1, 5, 3, 300, 8, 256)])
def test_append(gpu_lib, dtype, L, B, Hkv, K, D, page):
    rng = np.random.default_rng(K)
    n_pages = B * (-(-K // page) + 1) + 3
    slots = rng.permutation(n_pages * page)[:B * K].reshape(B, K).astype(np.int32)
    slots[rng.random((B, K)) < 0.2] = -1
    slots[0, 0] = n_pages * page                                   # one behind the last
    if B > 1:
        slots[1, 0] = -2 ** 31
        slots[-1] = -1                                             # a sequence that appends nothing
    dt = dtype_of(dtype)
    pages = [torch.randn((L, n_pages, Hkv, page, D), device="cuda").to(dt) for _ in range(2)]
    blocks = [torch.randn((L, B, Hkv, K, D), device="cuda").to(dt) for _ in range(2)]
    want = [p.clone() for p in pages]
    for w, x in zip(want, blocks):
        for b in range(B):
            for t in range(K):
                if 0 <= slots[b, t] < n_pages * page:
                    w[:, slots[b, t] // page, :, slots[b, t] % page] = x[:, b, :, t]
    gpu_lib.paged_kv_append(*pages, *blocks, dev(slots))
    torch.cuda.synchronize()
    assert torch.equal(pages[0], want[0]) and torch.equal(pages[1], want[1])


def test_append_layers_apart(gpu_lib):
    """Layers at a distance larger than their size, with other data between them that stays."""
    wide = [torch.full((3, 7 * 2 * 16 * 64 + 128), 5.0, device="cuda") for _ in range(2)]
    pages = [w[:, :7 * 2 * 16 * 64].view(3, 7, 2, 16, 64) for w in wide]
    blocks = [torch.randn((3, 40 + 2 * 2 * 9 * 64), device="cuda")[:, 40:].view(3, 2, 2, 9, 64) for _ in range(2)]
    slots = torch.arange(18, dtype=torch.int32, device="cuda").view(2, 9) * 6
    gpu_lib.paged_kv_append(*pages, *blocks, slots)
    torch.cuda.synchronize()
    for w, p, x in zip(wide, pages, blocks):
        assert (w[:, 7 * 2 * 16 * 64:] == 5.0).all()
        at = slots.view(-1).long()
        got = torch.stack([p[l][at // 16, :, at % 16] for l in range(3)])
        assert torch.equal(got, x.transpose(2, 3).reshape(3, 18, 2, 64))


def _norm_rope_bound(x, w, pos, dtype, amplitude, want, **kw):
    """y has a relative error of at most 1.5e-6 (sum of squares over a lane's 8 or 16 elements and the lanes, reciprocal root, two
    products), cos and sin 3e-7 (fraction of a turn as a float, the functions, the amplitude), two products and a sum 2e-7: 2e-6 of
    |y_a| + |y_b|; then half a step of bf16."""
    D = x.shape[-1]
    y = norm_rope(x, w, pos, 10000.0, **dict(kw, rotary_dim=0))
    R = kw.get("rotary_dim", D)
    pair = np.abs(y).copy()
    a = np.abs(y[..., :R])
    if kw.get("interleaved"):
        pair[..., :R] = np.repeat(a[..., 0::2] + a[..., 1::2], 2, -1)
    else:
        pair[..., :R] = np.tile(a[..., :R // 2] + a[..., R // 2:], 2)
    bound = 2.1e-6 * max(amplitude, 1.0) * pair + 1e-9
    return bound + (2.0 ** -8 * np.abs(want) * 1.001 if dtype == "bf16" else 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,K,Hq,Hkv,D,R,norm,extra", [
    (1, 1, 4, 1, 64, 64, True, {}),
    (3, 27, 16, 4, 128, 128, True, {}),
    (2, 33, 3, 3, 96, 32, True, {}),
    (2, 5, 40, 2, 256, 256, False, {}),
    (1, 70, 7, 1, 80, 48, True, dict(scale_factor=8.0)),
    (2, 9, 8, 2, 64, 16, True, dict(scale_factor=4.0, original_len=4096, amplitude=1.1386)),
    (4, 2, 5, 5, 16, 0, True, {}),
    (1, 3, 28, 4, 128, 128, True, dict(scale_factor=32.0, original_len=8192, low_turns=1.0, high_turns=4.0)),
])
def test_norm_rope(gpu_lib, dtype, interleaved, B, K, Hq, Hkv, D, R, norm, extra):
    g = torch.Generator(device="cuda")
    g.manual_seed(D + K)
    dt = dtype_of(dtype)
    draw = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dt)
    qkv = draw(B, K, Hq + 2 * Hkv, D) * 3
    q, k, v = (x.transpose(1, 2) for x in qkv.split([Hq, Hkv, Hkv], 2))
    wq, wk = (1 + 0.2 * draw(D), 1 + 0.2 * draw(D)) if norm else (None, None)
    rng = np.random.default_rng(D)
    start = rng.integers(0, 500000, B).astype(np.int32)
    start[0] = 0
    rows = (start[:, None] + np.sort(rng.permutation(3 * K)[:K])[None]).astype(np.int32)
    theta = 500000.0
    f = lambda t: None if t is None else to_f64_host(t)
    amp = extra.get("amplitude", 1.0)
    page, n_pages = 16, B * (K // 16 + 2)
    slots = rng.permutation(n_pages * page)[:B * K].reshape(B, K).astype(np.int32)
    slots[rng.random((B, K)) < 0.2] = -1
    for per_row in (False, True):
        pos = rows if per_row else start[:, None] + np.arange(K)[None]
        kw = dict(eps=1e-5, rotary_dim=R, interleaved=interleaved, **extra)
        want = [norm_rope(f(x), f(w), pos, theta, **kw) for x, w in ((q, wq), (k, wk))]
        scaling = {n: kw[n] for n in ("eps", "rotary_dim", "interleaved")}
        bounds = [_norm_rope_bound(f(x), f(w), pos, dtype, amp, y, **scaling) for x, w, y in ((q, wq, want[0]), (k, wk, want[1]))]
        positions = dev(rows if per_row else start)
        args = dict(q_weight=wq, k_weight=wk, **kw)
        for src in ((q, k), (q.contiguous(), k.contiguous())):
            got = gpu_lib.qk_norm_rope(*src, positions, theta, **args)
            torch.cuda.synchronize()
            for y, w, bound in zip(got, want, bounds):
                assert (np.abs(to_f64_host(y) - w) <= bound).all()
        # in place, and the keys and values into their pages: the same bits
        qi, ki = src[0].clone(), src[1].clone()
        gpu_lib.qk_norm_rope(qi, ki, positions, theta, q_out=qi, k_out=ki, **args)
        kp, vp = torch.full((n_pages, Hkv, page, D), 5.0, device="cuda").to(dt), torch.full((n_pages, Hkv, page, D), 5.0, device="cuda").to(dt)
        want_k, want_v = kp.clone(), vp.clone()
        q2, none = gpu_lib.qk_norm_rope(q, k, positions, theta, v=v, k_pages=kp, v_pages=vp, slots=dev(slots), **args)
        torch.cuda.synchronize()
        assert none is None and torch.equal(q2, got[0]) and torch.equal(qi, got[0]) and torch.equal(ki, got[1])
        for b in range(B):
            for t in range(K):
                if slots[b, t] >= 0:
                    want_k[slots[b, t] // page, :, slots[b, t] % page] = got[1][b, :, t]
                    want_v[slots[b, t] // page, :, slots[b, t] % page] = v[b, :, t]
        assert torch.equal(kp, want_k) and torch.equal(vp, want_v)


def test_norm_of_zero_and_of_large_rows(gpu_lib):
    """A row of zeros stays zero (eps > 0); rows whose squares fit fp32 are normed as any other."""
    q = torch.zeros((1, 2, 3, 64), device="cuda")
    q[0, 1] = 1e15
    pos = torch.zeros((1,), dtype=torch.int32, device="cuda")
    out, _ = gpu_lib.qk_norm_rope(q, q.clone(), pos, 1e4, q_weight=torch.ones(64, device="cuda"), rotary_dim=0)
    assert (out[0, 0] == 0).all() and (out[0, 1] - 1).abs().max() < 1e-6


class Serving:
    """A two-layer stack without weights between the layers: every layer's q, k, v rows are given.  Prompts, then blocks, then
    single tokens go through extend, norm + rope, append and attention; the reference keeps dense rows per sequence."""

    def __init__(self, sd, seed, dtype="bf16", B=3, L=2, Hq=8, Hkv=2, D=64, page=16, width=20):
        self.sd, self.B, self.L, self.Hq, self.Hkv, self.D, self.page = sd, B, L, Hq, Hkv, D, page
        self.dt, self.dtype = dtype_of(dtype), dtype
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        n_pages = B * width
        i32 = dict(dtype=torch.int32, device="cuda")
        self.table = torch.full((B, width), -1, **i32)
        self.lens, self.free = torch.zeros((B,), **i32), torch.randperm(n_pages, generator=self.g, device="cuda").to(torch.int32)
        self.n_free = torch.full((1,), n_pages, **i32)
        self.kp, self.vp = (torch.full((L, n_pages, Hkv, page, D), float("nan"), dtype=self.dt, device="cuda") for _ in range(2))
        self.w = [1 + 0.1 * torch.randn((D,), generator=self.g, device="cuda").to(self.dt) for _ in range(2)]
        self.dense = [[[np.zeros((Hkv, 0, D)), np.zeros((Hkv, 0, D))] for _ in range(B)] for _ in range(L)]
        self.cap = page * width

    def rows(self, K):
        draw = torch.randn((self.L, self.B, K, self.Hq + 2 * self.Hkv, self.D), generator=self.g, device="cuda").to(self.dt)
        return [tuple(x.transpose(1, 2) for x in d.split([self.Hq, self.Hkv, self.Hkv], 2)) for d in draw]

    def reference(self, rows, starts, counts, keep, causal):
        """Per layer the attention outputs [B,Hq,K,D] and bounds; rows join the dense caches if `keep`."""
        res = []
        for l, (q, k, v) in enumerate(rows):
            K = q.shape[2]
            pos = np.array(starts)[:, None] + np.arange(K)[None]

            qr = norm_rope(to_f64_host(q), to_f64_host(self.w[0]), pos, 1e4)
            kr = norm_rope(to_f64_host(k), to_f64_host(self.w[1]), pos, 1e4)
            rnd = lambda x: to_f64_host(torch.from_numpy(x).to(torch.float32).to(self.dt))
            qr, kr, vf = rnd(qr), rnd(kr), to_f64_host(v)
            out, out_abs = np.zeros(qr.shape), np.zeros(qr.shape)
            for b in range(self.B):
                c = counts[b]
                ks, vs = self.dense[l][b]
                ks, vs = np.concatenate([ks, kr[b, :, :c]], 1), np.concatenate([vs, vf[b, :, :c]], 1)
                n = ks.shape[1]
                pool = lambda x: np.pad(x, ((0, 0), (0, -n % 16), (0, 0))).reshape(self.Hkv, -1, 16, self.D).transpose(1, 0, 2, 3)
                ident = np.arange(-(-n // 16))[None]
                for o, values in ((out, vs), (out_abs, np.abs(vs))):
                    if c:
                        o[b, :, :c] = oracle_attention(qr[b:b + 1, :, :c], pool(ks), pool(values), ident, [n], causal=causal)[0]
                if keep[b]:
                    self.dense[l][b] = [ks, vs]
            res.append((out, out_abs))
        return res

    def check(self, outs, ref, counts):
        # q and k are rounded to bf16 between the two calls on both sides, but a value at the border of two bf16 numbers may go
        # either way: one step (2^-7 relative) of a key's element moves a score by 2^-7 |q_d k_d| / sqrt(D), about 1e-3 for unit
        # rows, and a weight by as much of itself: 2e-3 A beside the attention's own bound
        for got, (want, want_abs) in zip(outs, ref):
            for b, c in enumerate(counts):
                g, w, a = to_f64_host(got)[b, :, :c], want[b, :, :c], want_abs[b, :, :c]
                slack = 2e-3 if self.dtype == "bf16" else 1e-5
                bound = (2.0 ** -8 * 1.05 if self.dtype == "bf16" else 1e-5) * (a + 2 * np.abs(w)) + slack * (a + np.abs(w)) + 1e-6
                assert (np.abs(g - w) <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_serving_loop(gpu_lib, dtype):
    """Prompts of different lengths in a padded batch, a block that is decoded twice before it is appended, single tokens, a request
    that ends and one that takes its place."""
    sd = gpu_lib
    s = Serving(sd, 3, dtype)
    lens = [0] * s.B
    # prompts: straight into the pages, causal, each over its own rows only
    counts = [37, 5, 64]
    rows = s.rows(64)
    ref = s.reference(rows, lens, counts, [True] * s.B, causal=True)
    start = s.lens.clone()
    cnt = dev(np.array(counts, dtype=np.int32))
    slots, granted, _, _ = sd.paged_extend(s.table, s.lens, s.free, s.n_free, s.page, 64, new_lens=cnt)
    outs = []
    for l, (q, k, v) in enumerate(rows):
        qo, _ = sd.qk_norm_rope(q, k, start, 1e4, *s.w, v=v, k_pages=s.kp[l], v_pages=s.vp[l], slots=slots)
        outs.append(sd.paged_attention(qo, s.kp[l], s.vp[l], s.table, s.lens, s.cap, q_lens=granted, causal=True))
    torch.cuda.synchronize()
    lens = counts[:]
    assert s.lens.tolist() == lens
    s.check(outs, ref, counts)
    # a block of 8, twice with other rows; only sequences 0 and 2 finish it the second time
    for step, done in enumerate(([0, 0, 0], [1, 0, 1])):
        rows = s.rows(8)
        ref = s.reference(rows, lens, [8] * s.B, done, causal=False)
        kb, vb, outs = [], [], []
        for l, (q, k, v) in enumerate(rows):
            qo, ko = sd.qk_norm_rope(q, k, s.lens, 1e4, *s.w)
            outs.append(sd.paged_attention(qo, s.kp[l], s.vp[l], s.table, s.lens, s.cap, k_block=ko, v_block=v))
            kb.append(ko); vb.append(v)
        slots, granted, _, _ = sd.paged_extend(s.table, s.lens, s.free, s.n_free, s.page, 8, do_append=dev(np.array(done, dtype=np.uint8)))
        sd.paged_kv_append(s.kp, s.vp, torch.stack(kb), torch.stack(vb).contiguous(), slots)
        torch.cuda.synchronize()
        lens = [n + 8 * d for n, d in zip(lens, done)]
        assert s.lens.tolist() == lens and granted.tolist() == [8 * d for d in done]
        s.check(outs, ref, [8] * s.B)
    # sequence 1 ends, a prompt of 20 rows takes its place; the others go on by single tokens in the same batch
    for step in range(4):
        counts = [1, 20 if step == 0 else 1, 1]
        gone = [0, int(step == 0), 0]
        if step == 0:
            lens[1] = 0
            for l in range(s.L):
                s.dense[l][1] = [np.zeros((s.Hkv, 0, s.D))] * 2
        K = max(counts)
        rows = s.rows(K)
        ref = s.reference(rows, lens, counts, [True] * s.B, causal=True)
        slots, granted, _, _ = sd.paged_extend(s.table, s.lens, s.free, s.n_free, s.page, K, new_lens=dev(np.array(counts, dtype=np.int32)),
                                               release=dev(np.array(gone, dtype=np.uint8)))
        start = s.lens - granted
        outs = []
        for l, (q, k, v) in enumerate(rows):
            qo, _ = sd.qk_norm_rope(q, k, start, 1e4, *s.w, v=v, k_pages=s.kp[l], v_pages=s.vp[l], slots=slots)
            outs.append(sd.paged_attention(qo, s.kp[l], s.vp[l], s.table, s.lens, s.cap, q_lens=granted, causal=True))
        torch.cuda.synchronize()
        lens = [n + c for n, c in zip(lens, counts)]
        assert s.lens.tolist() == lens
        s.check(outs, ref, counts)


def test_a_captured_token_step(gpu_lib):
    """extend, norm + rope into the pages and attention of one token, captured once: every replay continues the sequences where the
    last one left them and equals the eager calls bit for bit."""
    sd = gpu_lib
    sd.init()
    a, b = Serving(sd, 4), Serving(sd, 4)
    prompt = a.rows(30)
    _ = b.rows(30)
    for s in (a, b):
        slots, *_ = sd.paged_extend(s.table, s.lens, s.free, s.n_free, s.page, 30, new_lens=dev(np.array([30, 11, 16], dtype=np.int32)))
        for l, (q, k, v) in enumerate(prompt):
            sd.qk_norm_rope(q, k, torch.zeros_like(s.lens), 1e4, *s.w, v=v, k_pages=s.kp[l], v_pages=s.vp[l], slots=slots)
    torch.cuda.synchronize()

    def step(s, rows, outs, stream=None):
        calls = []
        start = s.lens.clone()
        new = torch.zeros_like(s.lens)
        slots = torch.zeros((s.B, 1), dtype=torch.int32, device="cuda")
        ext = sd.bind_paged_extend(s.table, s.lens, s.free, s.n_free, s.page, 1, kv_lens_out=new, slots=slots, stream=stream)
        for l, (q, k, v) in enumerate(rows):
            qo = torch.empty((s.B, s.Hq, 1, s.D), dtype=s.dt, device="cuda")
            calls.append(sd.bind_qk_norm_rope(q, k, s.lens, 1e4, *s.w, v=v, q_out=qo, k_pages=s.kp[l], v_pages=s.vp[l], slots=slots, stream=stream))
            calls.append(sd.bind_paged_attention(qo, s.kp[l], s.vp[l], s.table, new, s.cap, causal=True, out=outs[l], stream=stream))
        def run():
            ext()
            for c in calls:
                c()
            s.lens.copy_(new)
        return run

    rows = [tuple(x.clone() for x in r) for r in a.rows(1)]
    outs = {id(s): [torch.zeros((s.B, s.Hq, 1, s.D), dtype=s.dt, device="cuda") for _ in range(s.L)] for s in (a, b)}
    eager = step(a, rows, outs[id(a)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        run = step(b, rows, outs[id(b)], side)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            run()
    for i in range(6):
        for r, new in zip(rows, a.rows(1)):
            for x, y in zip(r, new):
                x.copy_(y)
        eager()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        torch.randn((1000,), device="cuda").sum().item()
        assert a.lens.tolist() == b.lens.tolist() == [31 + i, 12 + i, 17 + i]
        assert torch.equal(a.table, b.table) and a.n_free.item() == b.n_free.item()
        for x, y in zip(outs[id(a)], outs[id(b)]):
            assert torch.equal(x, y) and torch.isfinite(x.float()).all()
