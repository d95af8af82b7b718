"""Pins of the oracle's extend where entries of released sequences are no pages (a page behind the window may be given back early)."""
import numpy as np

from oracle.paged import paged_extend


def test_only_pages_come_back():
    table = np.array([[-1, 9, 4, 5], [-1, -1, -1, -1]], dtype=np.int32)          # 9: outside the pool of 9
    stack = np.array([7, -1, -1, -1, -1, -1, -1, -1, -1], dtype=np.int32)
    t, lens, st, top, slots, got = paged_extend(table, [64, 0], stack, 1, 16, 48, new_lens=[0, 48], release=[1, 0])
    assert st[:3].tolist() == [7, 4, 5] and top == 0 and lens.tolist() == [0, 48] and got.tolist() == [0, 48]
    assert t[1].tolist() == [5, 4, 7, -1] and slots[1].tolist() == [p * 16 + r for p in (5, 4, 7) for r in range(16)]
    # one page more than there is
    t, lens, st, top, slots, got = paged_extend(table, [64, 0], stack, 1, 16, 49, new_lens=[0, 49], release=[1, 0])
    assert got.tolist() == [0, 0] and top == 3 and (slots == -1).all() and (t == table).all()


def test_rows_that_are_granted_have_a_slot():
    """Sequences that give pages back behind a window and are released later: every granted row has a slot, no page is lost or shared."""
    rng = np.random.default_rng(1)
    B, width, page, n_pages = 7, 14, 16, 60
    table, lens = np.full((B, width), -1, dtype=np.int32), np.zeros(B, dtype=np.int32)
    stack, top = rng.permutation(n_pages).astype(np.int32), n_pages
    for step in range(300):
        gone = (rng.random(B) < 0.15).astype(np.uint8)
        table, lens, stack, top, slots, got = paged_extend(table, lens, stack, top, page, 40, new_lens=rng.integers(0, 41, B), release=gone)
        assert ((slots >= 0).sum(1) == got).all()
        held = [int(p) for b in range(B) for p in table[b, :-(-lens[b] // page)] if p >= 0]
        assert sorted(held + stack[:top].tolist()) == list(range(n_pages))
        for b in range(B):
            for e in range((lens[b] - 30) // page):                          # pages wholly behind a window of 30
                if table[b, e] >= 0 and rng.random() < 0.5:
                    stack[top], top, table[b, e] = table[b, e], top + 1, -1
