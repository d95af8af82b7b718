"""sdllm_paged_extend where entries of released sequences are no pages, against the oracle (integers, equal)."""
import numpy as np
import pytest
import torch

from oracle.paged import paged_extend as oracle_extend
from paged_util import make_tables

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def extend_both(sd, table, lens, stack, top, page, K, **kw):
    want = oracle_extend(table, lens, stack, top, page, K, **kw)
    t, l, s, n = dev(table), dev(lens), dev(stack), dev(np.array([top], dtype=np.int32))
    slots, granted, lo, no = sd.paged_extend(t, l, s, n, page, K, **{k: dev(v) for k, v in kw.items()})
    torch.cuda.synchronize()
    for name, g, w in zip(("table", "lens", "stack", "n_free", "slots", "granted"), (t, lo, s, no, slots, granted), want):
        assert np.array_equal(g.cpu().numpy().reshape(-1), np.asarray(w).reshape(-1)), name
    return want


# batches of one wave, one and several chunks of a workgroup; one launch and two; more pages of a sequence than a pass takes
@pytest.mark.parametrize("B,K,page,most", [(1, 1, 16, 100), (5, 3, 16, 9000), (64, 4, 32, 500), (65, 1, 16, 90), (300, 3, 16, 700),
                                           (1025, 1, 64, 3000), (2100, 7, 16, 100), (40, 700, 256, 20000), (3, 6000, 16, 90000)])
@pytest.mark.parametrize("holes,gone", [(0.0, 0.3), (0.4, 0.3), (0.4, 1.0), (1.0, 0.5)])
def test_holes_in_released_rows(gpu_lib, B, K, page, most, holes, gone):
    rng = np.random.default_rng(B + K)
    lens = rng.integers(0, most + 1, B).astype(np.int32)
    table, spare, n_pages = make_tables(rng, lens, page, -(-(most + K) // page), spare=B)
    bad = np.array([-1, n_pages, -2 ** 31, 2 ** 31 - 1], dtype=np.int32)
    table = np.where(rng.random(table.shape) < holes, bad[rng.integers(0, 4, table.shape)], table).astype(np.int32)
    stack = np.full(n_pages, -1, dtype=np.int32)
    stack[:B] = spare[:B]
    release = (rng.random(B) < gone).astype(np.uint8)
    new = rng.integers(0, K + 1, B).astype(np.int32)
    for top in (B, B // 2, 0):
        extend_both(gpu_lib, table, lens, stack, top, page, K, new_lens=new, release=release)
    full = np.concatenate([stack[:B], np.zeros(n_pages - B, dtype=np.int32)])
    extend_both(gpu_lib, table, lens, full, n_pages - 1, page, K, new_lens=new, release=release)      # hardly any room


def test_a_window_gives_pages_back_before_the_end(gpu_lib):
    """The device state over many steps: pages wholly behind a window go back early, all others when their sequence is released."""
    rng = np.random.default_rng(7)
    B, width, page, n_pages = 70, 14, 16, 400
    table, lens = np.full((B, width), -1, dtype=np.int32), np.zeros(B, dtype=np.int32)
    stack, top = rng.permutation(n_pages).astype(np.int32), n_pages
    for step in range(40):
        table, lens, stack, top, slots, got = extend_both(gpu_lib, table, lens, stack, top, page, 40, release=(rng.random(B) < 0.2).astype(np.uint8),
                                                          new_lens=rng.integers(0, 41, B).astype(np.int32))
        assert ((slots >= 0).sum(1) == got).all()
        held = [int(p) for b in range(B) for p in table[b, :-(-lens[b] // page)] if p >= 0]
        assert sorted(held + stack[:top].tolist()) == list(range(n_pages))
        for b in range(B):
            for e in range((lens[b] - 30) // page):
                if table[b, e] >= 0 and rng.random() < 0.5:
                    stack[top], top, table[b, e] = table[b, e], top + 1, -1
