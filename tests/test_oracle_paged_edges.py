"""Pins of oracle/paged.py at the edges of its definitions: values out of range, flags, partial rotations, rows in front of the cache."""
import math

import numpy as np
import pytest

from oracle.paged import norm_rope, paged_attention, paged_extend, rotary_frequencies

STACK = np.array([6, 2, 8, 7, -1, -1, -1, -1, -1, -1], dtype=np.int32)       # 4 free of 10


def empty(B, width=3):
    return np.full((B, width), -1, dtype=np.int32)


def test_requests_lengths_and_stack_out_of_range():
    t, lens, st, top, slots, got = paged_extend(empty(3), [0, 0, 0], STACK, 4, 16, 20, new_lens=[-5, 900, 3])
    assert got.tolist() == [0, 20, 3] and lens.tolist() == [0, 20, 3] and top == 1
    assert t.tolist() == [[-1, -1, -1], [7, 8, -1], [2, -1, -1]]
    # a length past the table row is the whole row, a negative one is none
    table = np.array([[1, 3, 5], [-1, -1, -1]], dtype=np.int32)
    t, lens, st, top, slots, got = paged_extend(table, [1000, -7], STACK, 4, 16, 2)
    assert lens.tolist() == [48, 2] and got.tolist() == [0, 2] and slots.tolist() == [[-1, -1], [112, 113]]
    # more free pages than the pool has, or fewer than none
    full = np.arange(3, dtype=np.int32)
    t, lens, st, top, slots, got = paged_extend(empty(1), [0], full, 100, 16, 1)
    assert t[0, 0] == 2 and top == 2 and got.tolist() == [1]
    assert paged_extend(empty(1), [0], full, -4, 16, 1)[3:4] == (0,)


def test_what_is_pushed_past_the_pool_is_dropped():
    table = np.array([[0, 1, 2]], dtype=np.int32)
    t, lens, st, top, slots, got = paged_extend(table, [48], np.array([2, 1, -1], dtype=np.int32), 2, 16, 1, new_lens=[0], release=[1])
    assert st.tolist() == [2, 1, 0] and top == 3 and lens.tolist() == [0]


def test_flags_full_rows_and_sequences_that_need_no_page():
    table = np.array([[1, 3, 5], [4, -1, -1], [9, -1, -1]], dtype=np.int32)
    # 0 fills its table row to the last place; 1 does not append; 2 grows within its page
    t, lens, st, top, slots, got = paged_extend(table, [46, 16, 3], STACK, 4, 16, 2, do_append=[1, 0, 1])
    assert got.tolist() == [2, 0, 2] and lens.tolist() == [48, 16, 5] and top == 4 and (t == table).all()
    assert slots.tolist() == [[94, 95], [-1, -1], [147, 148]]
    # nothing is free: 1 needs a page and gets nothing, 2 behind it needs none and grows
    t, lens, st, top, slots, got = paged_extend(table, [40, 16, 3], STACK, 0, 16, 2)
    assert got.tolist() == [2, 0, 2] and lens.tolist() == [42, 16, 5]


def test_rows_of_pages_outside_the_pool_have_no_slot():
    table = np.array([[-3, 3, -1], [99, -1, -1]], dtype=np.int32)
    t, lens, st, top, slots, got = paged_extend(table, [15, 4], STACK, 4, 16, 2)
    assert got.tolist() == [2, 2] and slots.tolist() == [[-1, 7 * 16], [-1, -1]]
    bad = np.array([55, 2, 1], dtype=np.int32)                                   # the stack's own entries are taken as they are
    t, lens, st, top, slots, got = paged_extend(empty(1), [0], bad, 1, 16, 2)
    assert t[0, 0] == 55 and slots.tolist() == [[-1, -1]] and got.tolist() == [2]


def test_the_norm_of_small_rows():
    """eps is added to the mean square: a row of 1e-3 with eps 1e-6 is divided by sqrt(2e-6)."""
    y = norm_rope(np.full((1, 1, 1, 16), 1e-3), np.ones(16), np.zeros((1, 1)), 1e4, eps=1e-6, rotary_dim=0)
    assert np.allclose(y, 1 / math.sqrt(2), rtol=1e-12)


def test_part_of_the_head_has_the_frequencies_of_that_part():
    x = np.zeros((1, 1, 1, 64))
    x[..., 0:8] = 1.0                                                            # the first halves of pairs (i, i + 8)
    y = norm_rope(x, None, np.array([[3.0]]), 100.0, rotary_dim=16)[0, 0, 0]
    angle = 3.0 * 100.0 ** (-np.arange(8) / 8)
    assert np.allclose(y[:8], np.cos(angle)) and np.allclose(y[8:16], np.sin(angle)) and (y[16:] == 0).all()


def test_the_ramp_between_the_turns():
    """Pair 8 of 16 at base 1e4: f = 1e-2.  4000 pi rows are 20 turns of it, half way between 10 and 30."""
    f = rotary_frequencies(32, 1e4, 5.0, 4000 * np.pi, 10.0, 30.0)
    assert np.isclose(f[8], 0.5 * 1e-2 + 0.5 * 1e-2 / 5.0, rtol=1e-12)


@pytest.mark.parametrize("block", [False, True])
def test_positions_when_some_rows_are_missing(block):
    """Two of five query rows: without a block the last two of the cached positions, with one the first two of the block behind them."""
    rng = np.random.default_rng(9)
    kp, vp = rng.standard_normal((2, 2, 1, 16, 8))
    q, kb, vb = rng.standard_normal((3, 1, 1, 5, 8))
    got = paged_attention(q, kp, vp, np.array([[1, 0]]), [20], *((kb, vb) if block else (None, None)), [2], causal=True, out=np.full((1, 1, 5, 8), 4.0))
    keys, vals = (np.concatenate([x[1, 0], x[0, 0, :4]] + ([y[0, 0, :2]] if block else [])) for x, y in ((kp, kb), (vp, vb)))
    for r in range(2):
        n = 21 + r if block else 19 + r
        w = np.exp(keys[:n] @ q[0, 0, r] / math.sqrt(8))
        assert np.allclose(got[0, 0, r], (w / w.sum()) @ vals[:n], atol=1e-12)
    assert (got[0, 0, 2:] == 4.0).all()


def test_rows_in_front_of_the_cache_see_nothing():
    """Six rows on four keys: the first two lie before the first key; sinks do not make a key visible that lies ahead."""
    rng = np.random.default_rng(10)
    kp, vp = rng.standard_normal((2, 1, 1, 16, 8))
    q = rng.standard_normal((1, 1, 6, 8))
    for kw in (dict(), dict(window=2, sinks=3)):
        got = paged_attention(q, kp, vp, np.array([[0]]), [4], causal=True, out=np.full((1, 1, 6, 8), 4.0), **kw)[0, 0]
        assert (got[:2] == 0).all() and np.allclose(got[2], vp[0, 0, 0]) and not np.allclose(got[3], vp[0, 0, 0])


def test_the_scale_and_large_scores():
    rng = np.random.default_rng(11)
    kp, vp = rng.standard_normal((2, 1, 1, 16, 8))
    q = rng.standard_normal((1, 1, 1, 8))
    a, b = (paged_attention(q * f, kp, vp, np.array([[0]]), [9], scale=s) for f, s in ((1.0, 0.7), (7.0, 0.1)))
    assert np.allclose(a, b, atol=1e-12)
    assert not np.allclose(a, paged_attention(q, kp, vp, np.array([[0]]), [9]))
    best = np.argmax(kp[0, 0, :9] @ q[0, 0, 0])
    assert np.allclose(paged_attention(q, kp, vp, np.array([[0]]), [9], scale=1e5)[0, 0, 0], vp[0, 0, best])
