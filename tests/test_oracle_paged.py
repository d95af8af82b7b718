"""Pins of oracle/paged.py: closed forms and equality with other routes."""
import numpy as np
import pytest

from oracle import block_attention, rope_rotate
from oracle.paged import norm_rope, paged_attention, paged_extend, rotary_frequencies


def test_extend_by_hand():
    table = np.array([[5, -1, -1], [2, 3, -1], [-1, -1, -1]], dtype=np.int32)
    stack = np.array([7, 0, 1, 4, -1, -1, -1, -1], dtype=np.int32)
    t, lens, st, top, slots, got = paged_extend(table, [15, 20, 0], stack, 4, 16, 3)
    # sequence 0 crosses into a new page (4, the top), 1 stays in its own, 2 opens its first (1)
    assert t.tolist() == [[5, 4, -1], [2, 3, -1], [1, -1, -1]]
    assert slots.tolist() == [[5 * 16 + 15, 64, 65], [3 * 16 + 4, 53, 54], [16, 17, 18]]
    assert lens.tolist() == [18, 23, 3] and got.tolist() == [3, 3, 3] and top == 2 and (st == stack).all()


def test_extend_refuses_whole_sequences_in_batch_order():
    table = np.full((4, 4), -1, dtype=np.int32)
    stack = np.array([9, 8, 7, -1, -1, -1, -1, -1, -1, -1], dtype=np.int32)
    t, lens, st, top, slots, got = paged_extend(table, [0, 0, 0, 0], stack, 3, 16, 64, new_lens=[20, 40, 0, 16])
    # two pages for the first; the second needs three with one left; the third needs none; the fourth would have fitted, but the
    # refused one stands before it in the queue
    assert got.tolist() == [20, 0, 0, 0] and top == 1 and lens.tolist() == [20, 0, 0, 0]
    assert (slots[1:] == -1).all() and (slots[0, 20:] == -1).all() and t[0].tolist() == [7, 8, -1, -1]
    # longer than a table row: refused, and not counted
    got = paged_extend(table, [50, 0, 0, 0], stack, 3, 16, 64, new_lens=[20, 40, 0, 16])[5]
    assert got.tolist() == [0, 40, 0, 0]


def test_extend_takes_back_pages_before_it_gives():
    table = np.array([[3, 1], [0, 2]], dtype=np.int32)
    stack = np.full(4, -1, dtype=np.int32)
    t, lens, st, top, slots, got = paged_extend(table, [17, 32], stack, 0, 16, 1, new_lens=[1, 0], release=[1, 0])
    assert st.tolist() == [3, 1, -1, -1] and t.tolist() == [[1, 1], [0, 2]] and lens.tolist() == [1, 32] and top == 1
    assert slots.tolist() == [[16], [-1]]


def test_pages_are_neither_lost_nor_shared():
    rng = np.random.default_rng(0)
    B, width, ps, n_pages = 7, 12, 16, 60
    table, lens = np.full((B, width), -1, dtype=np.int32), np.zeros(B, dtype=np.int32)
    stack, top = rng.permutation(n_pages).astype(np.int32), n_pages
    for step in range(200):
        gone = (rng.random(B) < 0.15).astype(np.uint8)
        table, lens, stack, top, slots, got = paged_extend(table, lens, stack, top, ps, 40, new_lens=rng.integers(0, 41, B), release=gone)
        held = [int(p) for b in range(B) for p in table[b, :-(-lens[b] // ps)]]
        assert sorted(held + stack[:top].tolist()) == list(range(n_pages))
        used = slots[slots >= 0]
        assert len(set(used.tolist())) == len(used) == got.sum()


def test_norm_rope_against_the_rotation_oracle_and_closed_forms():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 3, 5, 32))
    pos = np.array([[4, 5, 6, 7, 8], [100, 7, 3, 0, 2000]])
    for il in (False, True):
        y = norm_rope(x, None, pos, 10000.0, interleaved=il)
        for b in range(2):
            assert np.allclose(y[b], rope_rotate(x[b:b + 1], pos[b], 10000.0, il)[0], atol=1e-12)
    w = rng.standard_normal(32)
    y = norm_rope(x, w, pos, 10000.0, eps=0.0, rotary_dim=0)
    assert np.allclose((y / w) ** 2 @ np.ones(32), 32.0)
    y = norm_rope(x, None, pos, 10000.0, rotary_dim=16, amplitude=2.0)
    assert (y[..., 16:] == x[..., 16:]).all()
    assert np.allclose((y[..., :16] ** 2).sum(-1), 4 * (x[..., :16] ** 2).sum(-1))


def test_scaled_frequencies():
    f = rotary_frequencies(64, 10000.0)
    assert f[0] == 1.0 and np.isclose(f[16], 10000.0 ** -0.5)
    assert np.allclose(rotary_frequencies(64, 10000.0, 4.0), f / 4)
    s = rotary_frequencies(64, 10000.0, 4.0, 4096)
    turns = f * 4096 / (2 * np.pi)
    assert np.allclose(s[turns >= 32], f[turns >= 32]) and np.allclose(s[turns <= 1], f[turns <= 1] / 4)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and (s[mid] < f[mid]).all() and (s[mid] > f[mid] / 4).all()


@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (4, 2)])
def test_attention_equals_the_dense_oracle(Hq, Hkv):
    """Equal lengths, no mask: the paged form of block_attention without a suffix."""
    rng = np.random.default_rng(2)
    B, D, K, P, ps = 2, 16, 5, 37, 16
    table = rng.permutation(9)[:6].reshape(B, 3)
    kp, vp = rng.standard_normal((2, 9, Hkv, ps, D))
    q, kb, vb = rng.standard_normal((B, Hq, K, D)), rng.standard_normal((B, Hkv, K, D)), rng.standard_normal((B, Hkv, K, D))
    got = paged_attention(q, kp, vp, table, [P, P], kb, vb)
    kc, vc = (np.stack([x[table[b]].transpose(1, 0, 2, 3).reshape(Hkv, -1, D) for b in range(B)]) for x in (kp, vp))
    none = np.zeros((B, Hkv, 0, D))
    want = block_attention(q, np.zeros((B, Hq, 0, D)), kc, vc, kb, vb, none, none, np.zeros(0, dtype=np.int32), P)
    assert np.allclose(got, want, atol=1e-12)


def test_attention_masks_by_brute_force():
    rng = np.random.default_rng(3)
    D, K, n, ps = 8, 6, 21, 16
    kp, vp = rng.standard_normal((2, 3, 1, ps, D))
    q, kb, vb = rng.standard_normal((1, 1, K, D)), rng.standard_normal((1, 1, K, D)), rng.standard_normal((1, 1, K, D))
    table = np.array([[2, 0]])
    keys = np.concatenate([kp[2, 0], kp[0, 0, :5], kb[0, 0]])
    vals = np.concatenate([vp[2, 0], vp[0, 0, :5], vb[0, 0]])
    for causal, window, sinks in [(True, 0, 0), (True, 4, 0), (True, 4, 2), (False, 4, 0), (False, 3, 1), (True, 1, 0)]:
        got = paged_attention(q, kp, vp, table, [n], kb, vb, causal=causal, window=window, sinks=sinks)
        for r in range(K):
            num, den = np.zeros(D), 0.0
            for j in range(n + K):
                if (causal and j > n + r) or (window and n + r - j >= window and j >= sinks):
                    continue
                e = np.exp(float(q[0, 0, r] @ keys[j]) / np.sqrt(D))
                num, den = num + e * vals[j], den + e
            assert np.allclose(got[0, 0, r], num / den, atol=1e-12)
    # the window of one key: the row's own value; no key at all: zero; a page that is not there: hidden
    assert np.allclose(got[0, 0], vb[0, 0])
    assert (paged_attention(q, kp, vp, table, [0])[0, 0] == 0).all()
    full, part = (paged_attention(q, kp, vp, t, [n], kb, vb) for t in (np.array([[2, -1]]), np.array([[2, 5]])))
    assert np.allclose(full, part)
