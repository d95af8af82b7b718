"""Oracle of the operators over a paged K/V cache, numpy float64 / Python integers, written from their definitions."""
import numpy as np


def paged_extend(block_table, kv_lens, free_pages, n_free, page_size, K, new_lens=None, do_append=None, release=None):
    """One sequence after the other, one page after the other.  Returns (block_table, kv_lens, free_pages, n_free, slots, granted)
    as new arrays; `need so far` counts the sequences that were refused for want of pages, too.  Entries of a released sequence that
    are no pages of the pool do not go on the stack."""
    table, lens, stack = block_table.copy(), [int(x) for x in kv_lens], free_pages.copy()
    B, max_pages = table.shape
    n_pages, top = len(stack), min(max(int(n_free), 0), len(free_pages))
    lens = [min(max(n, 0), max_pages * page_size) for n in lens]
    pages = lambda n: -(-n // page_size)
    if release is not None:
        for b in range(B):
            if release[b]:
                for e in range(pages(lens[b])):
                    if 0 <= block_table[b, e] < n_pages and top < n_pages:
                        stack[top] = block_table[b, e]
                        top += 1
                lens[b] = 0
    slots = np.full((B, K), -1, dtype=np.int32)
    granted = np.zeros(B, dtype=np.int32)
    available, so_far = top, 0
    for b in range(B):
        n = K if new_lens is None else min(max(int(new_lens[b]), 0), K)
        if do_append is not None and not do_append[b]:
            n = 0
        if lens[b] + n > max_pages * page_size:
            continue
        need = pages(lens[b] + n) - pages(lens[b])
        so_far += need
        if need > 0 and so_far > available:
            continue
        for e in range(pages(lens[b]), pages(lens[b] + n)):
            top -= 1
            table[b, e] = stack[top]
        for t in range(n):
            page, row = divmod(lens[b] + t, page_size)
            if 0 <= table[b, page] < n_pages:
                slots[b, t] = table[b, page] * page_size + row
        granted[b] = n
        lens[b] += n
    return table, np.array(lens, dtype=np.int32), stack, top, slots, granted


def rotary_frequencies(rotary_dim, theta_base, scale_factor=1.0, original_len=0, low_turns=1.0, high_turns=32.0):
    """Radians per position of each pair, with the scaling by parts."""
    out = []
    for i in range(rotary_dim // 2):
        f = float(theta_base) ** (-2.0 * i / rotary_dim)
        u = 0.0
        if original_len > 0:
            u = min(max((f * original_len / (2.0 * np.pi) - low_turns) / (high_turns - low_turns), 0.0), 1.0)
        out.append(u * f + (1.0 - u) * f / scale_factor)
    return np.array(out)


def norm_rope(x, weight, positions, theta_base, eps=1e-6, rotary_dim=None, interleaved=False, amplitude=1.0, **scaling):
    """x [B,H,K,D] (one of q, k), positions [B,K]."""
    D = x.shape[-1]
    R = D if rotary_dim is None else rotary_dim
    y = x.copy()
    if weight is not None:
        y = y / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    freq = rotary_frequencies(R, theta_base, **scaling)
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        angle = positions[:, None, :] * freq[i]
        c, s = np.cos(angle) * amplitude, np.sin(angle) * amplitude
        y[..., a], y[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    return y


def paged_attention(q, k_pages, v_pages, block_table, kv_lens, k_block=None, v_block=None, q_lens=None, causal=False, window=0,
                    sinks=0, scale=0.0, out=None):
    """One query row after the other over the list of the keys it sees (float64 inputs).  Rows from q_lens[b] on keep `out`."""
    B, Hq, K, D = q.shape
    n_pages, Hkv, page_size, _ = k_pages.shape
    out = np.zeros_like(q) if out is None else out.copy()
    scale = scale if scale > 0 else 1.0 / np.sqrt(D)
    for b in range(B):
        n = int(kv_lens[b])
        ql = K if q_lens is None else int(q_lens[b])
        total = n + (ql if k_block is not None else 0)
        valid = np.array([0 <= block_table[b, j // page_size] < n_pages for j in range(n)] + [True] * (total - n), dtype=bool)
        at = [(block_table[b, j // page_size], j % page_size) for j in range(n)]
        for h in range(Hkv):
            rows = lambda pages, block: np.stack([pages[p, h, r] if ok else np.zeros(D) for (p, r), ok in zip(at, valid)]
                                                 + [block[b, h, j] for j in range(total - n)]) if total else np.zeros((0, D))
            k, v = rows(k_pages, k_block), rows(v_pages, v_block)
            for m in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                for r in range(ql):
                    p = total - ql + r
                    j = np.arange(total)
                    seen = valid & ((j <= p) | (not causal))
                    if window:
                        seen &= (p - j < window) | (j < sinks)
                    if not seen.any():
                        out[b, m, r] = 0.0
                        continue
                    z = k[seen] @ q[b, m, r] * scale
                    w = np.exp(z - z.max())
                    out[b, m, r] = (w / w.sum()) @ v[seen]
    return out
