"""The README's lines on the paged cache, run as they stand and compared with the oracle on dense rows."""
import os
import re

import numpy as np
import pytest
import torch

from gpu_util import to_f64_host
from oracle.paged import norm_rope, paged_attention as oracle_attention

pytestmark = pytest.mark.gpu
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def code_blocks():
    text = open(README).read()
    text = text[text.index("Sequences of different lengths"):text.index("`bind_*` variants")]
    blocks = ["".join(line[4:] for line in b.splitlines(True)) for b in re.findall(r"(?:^    .*\n|^\n(?=    ))+", text, re.M)]
    return [compile(b, README, "exec") for b in blocks if "sd." in b]


def test_the_lines_of_the_readme(gpu_lib):
    tokens, block = code_blocks()
    B, Hq, Hkv, D, page, width, n_pages = 3, 4, 2, 64, 16, 12, 36
    g = torch.Generator(device="cuda")
    g.manual_seed(81)
    i32 = dict(dtype=torch.int32, device="cuda")
    flags = lambda *x: torch.tensor(x, dtype=torch.uint8, device="cuda")
    rows = lambda h, K: torch.randn((B, h, K, D), generator=g, device="cuda")
    pools = [torch.full((1, n_pages, Hkv, page, D), float("nan"), device="cuda") for _ in range(2)]
    ns = dict(sd=gpu_lib, table=torch.full((B, width), -1, **i32), lens=torch.zeros(B, **i32), free_pages=torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32),
              n_free=torch.full((1,), n_pages, **i32), page_size=page, max_len=page * width, l=0, k_pages=pools[0], v_pages=pools[1],
              wq=torch.ones(D, device="cuda") * 0.5, wk=torch.ones(D, device="cuda") * 2.0)
    f = to_f64_host
    dense = [[np.zeros((Hkv, 0, D))] * 2 for _ in range(B)]

    def check(q, k, v, keep, causal):
        """This step's rows behind the dense ones; they stay there where keep is set."""
        for b in range(B):
            at = dense[b][0].shape[1] + np.arange(q.shape[2])[None]
            qr = norm_rope(f(q[b:b + 1]), f(ns["wq"]), at, 1e6)
            ks, vs = (np.concatenate([old, new], 1) for old, new in zip(dense[b], (norm_rope(f(k[b:b + 1]), f(ns["wk"]), at, 1e6)[0], f(v[b]))))
            n = ks.shape[1]
            pool = lambda x: np.pad(x, ((0, 0), (0, -n % 16), (0, 0))).reshape(Hkv, -1, 16, D).transpose(1, 0, 2, 3)
            want = oracle_attention(qr, pool(ks), pool(vs), np.arange(-(-n // 16))[None], [n], causal=causal)[0]
            # Norm and rotation are off by 2.1e-6 of a pair's sum on either side: with |q| = 4 and |k| = 16 (norms of 8, weights 1/2 and 2)
            # a score, 64 / 8 at most, by 4.2e-6 * 2 * 8 = 7e-5, a weight by as much of itself, and 1e-5 for the attention
            # (paged_util): twice 8e-5 of values up to 6
            assert np.abs(f(ns["out"][b]) - want).max() <= 2 * 8e-5 * 6
            if keep[b]:
                dense[b] = [ks, vs]

    for K, finished in ((21, (0, 0, 0)), (1, (0, 0, 0)), (5, (0, 1, 0)), (1, (0, 0, 0))):
        q, k, v = rows(Hq, K), rows(Hkv, K), rows(Hkv, K)
        for b in range(B):
            if finished[b]:
                dense[b] = [np.zeros((Hkv, 0, D))] * 2
        ns.update(K=K, finished=flags(*finished), q=q, k=k, v=v)
        exec(tokens, ns)
        check(q, k, v, [1] * B, True)
    for done in ((0, 0, 0), (1, 0, 1), (1, 1, 1)):
        K = 8
        q, k, v = rows(Hq, K), rows(Hkv, K), rows(Hkv, K)
        ns.update(K=K, block_done=flags(*done), q=q, k=k, v=v, v_blocks=v[None])
        start = [dense[b][0].shape[1] for b in range(B)]
        ns["k_blocks"] = gpu_lib.qk_norm_rope(q, k, ns["lens"], 1e6, ns["wq"], ns["wk"])[1][None]
        exec(block, ns)
        check(q, k, v, done, False)
        assert ns["lens"].tolist() == [n + K * d for n, d in zip(start, done)]
