"""pytest plugin used only by test_oracle_paged_pin_strength.py: single mistakes in oracle/paged.py, planted as oracle_mutants.py does."""
import os

import oracle_mutants

MUTANTS = {
    # pages, tables and slots
    "extend_pushes_what_is_no_page": ("if 0 <= block_table[b, e] < n_pages and top < n_pages:", "if top < n_pages:"),
    "extend_pushes_past_the_pool": ("if 0 <= block_table[b, e] < n_pages and top < n_pages:", "if 0 <= block_table[b, e] < n_pages:"),
    "extend_release_keeps_the_length": ("                lens[b] = 0\n", "                pass\n"),
    "extend_release_in_reverse": ("stack[top] = block_table[b, e]", "stack[top] = block_table[b, pages(lens[b]) - 1 - e]"),
    "extend_pops_from_below": ("table[b, e] = stack[top]", "table[b, e] = stack[available - 1 - top]"),
    "extend_refused_do_not_count": ("        so_far += need\n        if need > 0 and so_far > available:\n            continue\n",
                                    "        if need > 0 and so_far + need > available:\n            continue\n        so_far += need\n"),
    "extend_nothing_needed_is_refused": ("if need > 0 and so_far > available:", "if so_far > available:"),
    "extend_last_page_refused": ("if need > 0 and so_far > available:", "if need > 0 and so_far >= available:"),
    "extend_page_counts_rounded_down": ("pages = lambda n: -(-n // page_size)", "pages = lambda n: n // page_size"),
    "extend_full_row_refused": ("if lens[b] + n > max_pages * page_size:", "if lens[b] + n >= max_pages * page_size:"),
    "extend_new_lens_unbounded_below": ("min(max(int(new_lens[b]), 0), K)", "min(int(new_lens[b]), K)"),
    "extend_new_lens_unbounded_above": ("min(max(int(new_lens[b]), 0), K)", "max(int(new_lens[b]), 0)"),
    "extend_lens_unbounded": ("lens = [min(max(n, 0), max_pages * page_size) for n in lens]", "lens = [max(n, 0) for n in lens]"),
    "extend_n_free_unbounded": ("min(max(int(n_free), 0), len(free_pages))", "max(int(n_free), 0)"),
    "extend_flags_ignored": ("if do_append is not None and not do_append[b]:", "if False:"),
    "extend_slots_from_the_wrong_row": ("divmod(lens[b] + t, page_size)", "divmod(lens[b] + t + 1, page_size)"),
    "extend_slot_of_what_is_no_page": ("if 0 <= table[b, page] < n_pages:", "if True:"),
    "extend_length_stays": ("        lens[b] += n\n", "        pass\n"),
    "extend_granted_is_the_request": ("        granted[b] = n\n", "        granted[b] = K\n"),
    # norm and rotation
    "norm_sum_for_mean": ("(x * x).mean(-1, keepdims=True)", "(x * x).sum(-1, keepdims=True)"),
    "norm_eps_outside_the_root": ("np.sqrt((x * x).mean(-1, keepdims=True) + eps)", "(np.sqrt((x * x).mean(-1, keepdims=True)) + eps)"),
    "norm_weight_dropped": ("keepdims=True) + eps) * weight", "keepdims=True) + eps)"),
    "rope_frequency": ("(-2.0 * i / rotary_dim)", "(-1.0 * i / rotary_dim)"),
    "rope_sign": ("c, s = np.cos(angle) * amplitude, np.sin(angle) * amplitude", "c, s = np.cos(angle) * amplitude, -np.sin(angle) * amplitude"),
    "rope_amplitude_of_one_part": ("c, s = np.cos(angle) * amplitude, np.sin(angle) * amplitude", "c, s = np.cos(angle) * amplitude, np.sin(angle)"),
    "rope_pair_layout": ("if interleaved else (i, i + R // 2)", "if not interleaved else (i, i + R // 2)"),
    "rope_pairs_over_the_head": ("else (i, i + R // 2)", "else (i, i + D // 2)"),
    "rope_frequencies_over_the_head": ("freq = rotary_frequencies(R, theta_base, **scaling)", "freq = rotary_frequencies(D, theta_base, **scaling)"),
    "scaling_parts_swapped": ("u * f + (1.0 - u) * f / scale_factor", "(1.0 - u) * f + u * f / scale_factor"),
    "scaling_radians_for_turns": ("f * original_len / (2.0 * np.pi)", "f * original_len"),
    "scaling_ramp_unbounded": ("u = min(max((f * original_len / (2.0 * np.pi) - low_turns) / (high_turns - low_turns), 0.0), 1.0)",
                               "u = (f * original_len / (2.0 * np.pi) - low_turns) / (high_turns - low_turns)"),
    "scaling_ramp_to_high_turns": ("(high_turns - low_turns)", "high_turns"),
    # attention
    "attn_scale": ("1.0 / np.sqrt(D)", "1.0 / D"),
    "attn_scale_argument_ignored": ("scale = scale if scale > 0 else 1.0 / np.sqrt(D)", "scale = 1.0 / np.sqrt(D)"),
    "attn_causal_off_by_one": ("((j <= p) | (not causal))", "((j < p) | (not causal))"),
    "attn_causal_always": ("((j <= p) | (not causal))", "(j <= p)"),
    "attn_positions_from_the_cache": ("p = total - ql + r", "p = n + r"),
    "attn_positions_of_a_full_block": ("p = total - ql + r", "p = total - K + r"),
    "attn_window_off_by_one": ("(p - j < window)", "(p - j <= window)"),
    "attn_sinks_off_by_one": ("| (j < sinks)", "| (j <= sinks)"),
    "attn_sinks_always_on": ("seen &= (p - j < window) | (j < sinks)", "seen &= (p - j < window)"),
    "attn_sinks_past_causality": ("seen &= (p - j < window) | (j < sinks)", "seen = valid & ((seen & (p - j < window)) | (j < sinks))"),
    "attn_holes_seen": ("[0 <= block_table[b, j // page_size] < n_pages for j in range(n)]", "[True for j in range(n)]"),
    "attn_gqa_map": ("for m in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):", "for m in range(h, Hq, Hkv):"),
    "attn_values_from_keys": ("out[b, m, r] = (w / w.sum()) @ v[seen]", "out[b, m, r] = (w / w.sum()) @ k[seen]"),
    "attn_block_values_from_keys": ("rows(k_pages, k_block), rows(v_pages, v_block)", "rows(k_pages, k_block), rows(v_pages, k_block)"),
    "attn_rows_of_another_page": ("at = [(block_table[b, j // page_size], j % page_size) for j in range(n)]",
                                  "at = [(block_table[b, (j + 1) // page_size], j % page_size) for j in range(n)]"),
    "attn_q_lens_ignored": ("ql = K if q_lens is None else int(q_lens[b])", "ql = K"),
    "attn_no_maximum": ("w = np.exp(z - z.max())", "w = np.exp(z)"),
    "attn_empty_rows_kept": ("                        out[b, m, r] = 0.0\n", "                        pass\n"),
}
PIN_FILES = ["test_oracle_paged.py", "test_paged_release.py", "test_oracle_paged_edges.py"]


def pytest_configure(config):
    name = os.environ.get("SDLLM_ORACLE_MUTANT")
    if name:
        oracle_mutants.MUTANTS[name] = ("paged", *MUTANTS[name])
        oracle_mutants.plant(name)
