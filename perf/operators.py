"""What the operators over a paged key / value cache are judged on: their calls, their plain forms and their sizes.

A paged cache holds the K/V rows of many sequences in pages of `page_size` rows, [n_pages, Hkv, page_size, D]; row t of
sequence b is row t % page_size of page block_table[b][t / page_size], its slot is page * page_size + row in page.

Four operators, one kind of case each:
  extend     pages for a step's new rows: a stack of free pages, the block tables and the rows' slots, all on the device.
             Released sequences give their pages back first; then, in batch order, each sequence takes
             ceil((len + n) / page_size) - ceil(len / page_size) pages from the top of the stack, or nothing at all.
  norm_rope  y = rotate(x / sqrt(mean(x^2) + eps) * w) for each head's query and key row, pair i of rotary_dim / 2 turned
             by position * f_i and multiplied by an amplitude; f_i = theta^(-2i/rotary_dim), scaled by parts for long
             contexts: with r = f_i * original_len / 2 pi turns in the original context and
             u = clamp((r - low) / (high - low), 0, 1), f_i becomes u f_i + (1 - u) f_i / factor (original_len = 0: f_i /
             factor).  Keys go to a dense tensor or, with the values beside them, straight into the pages.
  append     a finished block's K/V rows of every layer into their slots.
  attention  softmax(scale q k^T) v of K query rows per sequence over the cache's kv_len rows and, if given, the block's
             own rows behind them.  The queries are the last q_len of the sequence's positions; a key at position j is
             visible to a query at position p if j <= p (causal) and p - j < window or j < sinks (window > 0).  A row that
             sees nothing is zero.  One token's row, a block's rows and a prompt's rows are the same call.

Weights and activations are seeded normal draws.  Lengths are spread evenly over the logarithm of their range and dealt to the
sequences by the seed.  Head counts follow workloads.py (32/32, 32/8, 28/4 of 128, 64-wide ones) unless a comment differs.
"""
import math

import torch

own = False
THETA = 500000.0


# ---------------------------------------------------------------------------------------------- cases
def _extend(name, B, K, page, len_lo, len_hi, new_lo, released, calls):
    return {"name": name, "kind": "extend", "B": B, "K": K, "page": page, "len_lo": len_lo, "len_hi": len_hi, "new_lo": new_lo,
            "released": released, "short": 0, "calls": calls}


def _norm_rope(name, dtype, B, K, Hq, Hkv, D, pos_hi, **more):
    case = {"name": name, "kind": "norm_rope", "dtype": dtype, "B": B, "K": K, "Hq": Hq, "Hkv": Hkv, "D": D, "pos_hi": pos_hi,
            "rotary": D, "interleaved": False, "factor": 1.0, "original": 0, "amplitude": 1.0, "pages": 0, "per_row": False,
            "norm": True, "calls": "bound"}
    case.update(more)
    return case


def _append(name, dtype, L, B, K, Hkv, D, page, skipped, calls):
    return {"name": name, "kind": "append", "dtype": dtype, "L": L, "B": B, "K": K, "Hkv": Hkv, "D": D, "page": page,
            "skipped": skipped, "calls": calls}


def _attention(name, dtype, B, Hq, Hkv, D, K, page, len_lo, len_hi, **more):
    case = {"name": name, "kind": "attention", "dtype": dtype, "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "K": K, "page": page,
            "len_lo": len_lo, "len_hi": len_hi, "q_lo": K, "block": False, "causal": False, "window": 0, "sinks": 0,
            "calls": "bound"}
    case.update(more)
    return case


def listed():
    return [
        # the next row of each of a few running sequences: most need no page, the call is its launch
        _extend("extend_token_b8", 8, 1, 16, 1, 4000, 1, 0.0, "bound"),
        # a batch that changes: a third of the sequences gave up their place and new prompts of all lengths come in
        _extend("extend_prompts_b64", 64, 2048, 16, 1, 8000, 1, 0.34, "plain"),
        # one new token per sequence, grouped-query heads; keys and values go straight into their pages
        _norm_rope("norm_rope_token_b16", "bf16", 16, 1, 32, 8, 128, 30000, pages=16),
        # the rows of a batch of blocks, dense (they change with every step), positions given row by row; fp32, 64-wide heads of
        # which half is rotated, interleaved pairs
        _norm_rope("norm_rope_block_f32", "fp32", 3, 27, 16, 4, 64, 5000, rotary=32, interleaved=True, per_row=True,
                   calls="plain"),
        # long prompts, frequencies scaled by parts to four times the original context
        _norm_rope("norm_rope_prompt_b2", "bf16", 2, 4096, 28, 4, 128, 120000, factor=4.0, original=32768, amplitude=1.1386,
                   pages=64),
        # a finished block of four sequences goes into all 32 layers' pages
        _append("append_block_l32", "bf16", 32, 4, 64, 32, 128, 64, 0.0, "bound"),
        # two fp32 layers of a ragged block, one sequence in three has not finished it
        _append("append_ragged_f32", "fp32", 2, 3, 27, 4, 64, 16, 0.34, "plain"),
        # interactive use: one new token of one sequence, its row already in the cache
        _attention("token_b1", "bf16", 1, 32, 8, 128, 1, 16, 700, 700, causal=True),
        # serving: one new token for each of 32 sequences of very different lengths
        _attention("token_ragged_b32", "bf16", 32, 32, 8, 128, 1, 16, 200, 16384, causal=True),
        # block diffusion: the rows of a block see the paged prefix and each other
        _attention("block_b8", "bf16", 8, 28, 4, 128, 32, 32, 500, 8000, block=True, calls="plain"),
        # prompts that come in pieces of up to 2048 tokens, behind prefixes of different lengths, a padded batch
        _attention("prompt_b2", "bf16", 2, 32, 8, 128, 2048, 64, 1000, 4096, q_lo=1501, block=True, causal=True),
        # fp32, 64-wide heads, a few query rows at a time under a sliding window with the first tokens kept visible
        _attention("window_f32_b4", "fp32", 4, 16, 4, 64, 5, 16, 300, 9000, causal=True, window=1024, sinks=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_extend(rng):
    K = rng.choice([1, 1, 32, _log_int(rng, 1, 4096)])
    lo = rng.choice([0, 1, _log_int(rng, 1, 2000)])
    case = _extend("", _log_int(rng, 1, 512), K, rng.choice([16, 16, 32, 64, 128, 256]), lo, lo + _log_int(rng, 1, 16000),
                   rng.choice([K, rng.randint(0, K)]), rng.choice([0.0, 0.0, 0.2, 0.9]), rng.choice(["bound", "plain"]))
    case["short"] = rng.choice([0, 0, 0, rng.randint(1, 40)])      # pages that the pool lacks
    return case


def _heads(rng, most):
    Hkv = rng.choice([1, 2, 4, 8, 16, 32])
    return Hkv * rng.choice([g for g in (1, 2, 3, 4, 7, 8, 16) if Hkv * g <= most]), Hkv


def _draw_norm_rope(rng):
    D = rng.choice([64, 64, 128, 128, 96, 256])
    Hq, Hkv = _heads(rng, 64)
    case = _norm_rope("", rng.choice(["bf16", "bf16", "fp32"]), _log_int(rng, 1, 64), _log_int(rng, 1, 4096), Hq, Hkv, D,
                      _log_int(rng, 10, 500000), interleaved=rng.random() < 0.3, per_row=rng.random() < 0.3,
                      norm=rng.random() < 0.8, calls=rng.choice(["bound", "plain"]))
    case["rotary"] = rng.choice([D, D, 16 * rng.randint(1, D // 16)])
    if rng.random() < 0.4:
        case["factor"] = rng.choice([2.0, 4.0, 8.0, rng.uniform(1.0, 32.0)])
        case["original"] = rng.choice([0, 4096, 8192, 32768])
        case["amplitude"] = 1.0 + 0.1 * math.log(case["factor"])
    case["pages"] = rng.choice([0, 0, 16, 32, 64, 256])
    return case


def _draw_append(rng):
    return _append("", rng.choice(["bf16", "bf16", "fp32"]), rng.choice([1, 1, 2, 8, 32, 40]), _log_int(rng, 1, 64),
                   _log_int(rng, 1, 512), rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([64, 96, 128, 256]),
                   rng.choice([16, 32, 64, 128, 256]), rng.choice([0.0, 0.3, 0.9]), rng.choice(["bound", "plain"]))


def _draw_attention(rng):
    Hq, Hkv = _heads(rng, 64)
    K = rng.choice([1, 1, 1, rng.randint(2, 8), rng.choice([16, 32, 64]), rng.randint(5, 200), _log_int(rng, 128, 2048)])
    block = rng.random() < 0.5
    hi = _log_int(rng, 8, 32768)
    if not block:
        hi = max(hi, K)
    lo = rng.choice([0, _log_int(rng, 1, hi)]) if block else max(_log_int(rng, 1, hi), K)
    case = _attention("", "fp32" if rng.random() < 0.25 else "bf16", _log_int(rng, 1, 64), Hq, Hkv, rng.choice([64, 128, 128]), K,
                      rng.choice([16, 16, 32, 64, 128, 256]), lo, hi, q_lo=rng.choice([K, K, max(1, K // 2)]), block=block,
                      causal=rng.random() < 0.6, calls=rng.choice(["bound", "plain"]))
    if rng.random() < 0.35:
        case["window"] = _log_int(rng, 1, 8192)
        case["sinks"] = rng.choice([0, 1, 4, rng.randint(0, 200)])
    return case


def draw(rng):
    """One more case: batches 1..64 (extend: 512), 1..2048 (rows 4096) new rows, lengths to 32768, 1..64 heads of 64 / 128 (norms
    and append also 96 and 256), pages of 16..256 rows, all masks, both types."""
    makers = [_draw_extend, _draw_norm_rope, _draw_append, _draw_attention, _draw_attention, _draw_attention]
    while True:
        case = rng.choice(makers)(rng)
        del case["name"]
        w = work(case)
        if case["kind"] == "attention":                 # the plain form holds one sequence's scores in fp32
            if case["Hq"] * case["K"] * (case["len_hi"] + case["K"]) > 4.1e8:
                continue
            if w["flops"] > (4e10 if case["dtype"] == "fp32" else 3.4e11):
                continue
        if w["bytes"] <= 5.3e8:
            return case


# ---------------------------------------------------------------------------------------------- sizes
def _spread(lo, hi, n):
    """n whole numbers from lo to hi, even in the logarithm (hi among them)."""
    if n == 1 or lo >= hi:
        return [hi] * n
    a, b = math.log(max(lo, 0.5)), math.log(hi)
    out = [int(round(math.exp(a + (b - a) * i / (n - 1)))) for i in range(n)]
    out[0], out[-1] = lo, hi
    return out


def _lens(case):
    return _spread(case["len_lo"], case["len_hi"], case["B"])


def _q_lens(case):
    return _spread(case["q_lo"], case["K"], case["B"])[::-1]


def _pairs(case, n, q):
    """Visible (query, key) pairs and distinct visible cache keys of a sequence with n cached rows and q query rows."""
    total = n + (q if case["block"] else 0)
    w, s, pairs, first = case["window"], case["sinks"], 0, total
    for r in range(q) if w or case["causal"] else ():
        p = total - q + r
        hi = min(p + 1, total) if case["causal"] else total
        lo = max(0, p - w + 1) if w else 0
        lo, hi = min(lo, max(hi, 0)), max(hi, 0)
        pairs += hi - lo + min(s, lo) if w else hi
        first = min(first, lo)
    if not (w or case["causal"]):
        return q * total, n
    seen = min(n, max(0, n - first) + min(s, first))
    return pairs, seen


def work(case):
    e = 4 if case.get("dtype") == "fp32" else 2
    kind = case["kind"]
    if kind == "extend":
        new = sum(_spread(case["new_lo"], case["K"], case["B"]))
        B, K, page = case["B"], case["K"], case["page"]
        return {"bytes": float(4 * (B * K + 6 * B + 3 * new // page)), "flops": float(B * K)}
    if kind == "norm_rope":
        rows = case["B"] * case["K"] * (case["Hq"] + case["Hkv"])
        v = 2 * case["B"] * case["K"] * case["Hkv"] * case["D"] * e if case["pages"] else 0
        return {"bytes": float(2 * rows * case["D"] * e + v), "flops": 8.0 * rows * case["D"]}
    if kind == "append":
        b = 4 * case["L"] * case["B"] * case["K"] * case["Hkv"] * case["D"] * e * (1 - case["skipped"])
        return {"bytes": float(b), "flops": 0.0}
    pairs = keys = 0
    for n, q in zip(_lens(case), _q_lens(case)):
        p, seen = _pairs(case, n, q)
        pairs += p
        keys += seen + (q if case["block"] else 0)
    rows = sum(_q_lens(case)) * case["Hq"]
    return {"bytes": float((2 * keys * case["Hkv"] + 2 * rows) * case["D"] * e), "flops": 4.0 * pairs * case["Hq"] * case["D"]}


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed, what, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed((int(seed) * 1000003 + what) & 0x7FFFFFFFFFFFFFFF)
    return g


def _normal(seed, what, shape, dtype, std=1.0, mean=0.0):
    x = torch.randn(shape, generator=_gen(seed, what), device="cuda", dtype=dtype)
    if std != 1.0:
        x.mul_(std)
    return x.add_(mean) if mean else x


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _dealt(values, seed, what):
    order = torch.randperm(len(values), generator=_gen(seed, what, "cpu")).tolist()
    return [values[i] for i in order]


def _tables(lens, page, width, seed, n_pages=0):
    """Block tables of sequences that hold `lens` rows, their pages in random order over the pool; -1 where none is held."""
    held = [-(-n // page) for n in lens]
    n_pages = n_pages or sum(held) + 3
    perm = torch.randperm(n_pages, generator=_gen(seed, 90, "cpu"))
    table = torch.full((len(lens), width), -1, dtype=torch.int64)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = perm[at:at + h]
        at += h
    return table.to(torch.int32), perm[at:].to(torch.int32), n_pages


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _prepare_extend(case, seed):
    B, K, page = case["B"], case["K"], case["page"]
    lens = _dealt(_lens(case), seed, 1)
    new = _dealt(_spread(case["new_lo"], K, B), seed, 2)
    width = -(-(case["len_hi"] + K) // page)
    g = _gen(seed, 3, "cpu")
    gone = [int(x) for x in torch.rand((B,), generator=g) < case["released"]]
    takes = sum(-(-((0 if r else n) + m) // page) - (-(-(0 if r else n) // page)) for n, m, r in zip(lens, new, gone))
    # as many pages as would do at any dealing; the stack holds five more than are taken, or too few
    n_pages = sum(-(-n // page) for n in lens) + sum(-(-m // page) for m in new) + 5
    table, spare, n_pages = _tables(lens, page, width, seed, n_pages)
    spare = spare[:max(takes + 5 - case["short"], 0)]
    stack = torch.full((n_pages,), -1, dtype=torch.int32)
    stack[:len(spare)] = spare
    s = {"case": case, "table": table.cuda(), "lens": _int32(lens), "new": _int32(new), "free": stack.cuda(),
         "n_free": _int32([len(spare)]), "release": None}
    s["lens_out"], s["n_free_out"] = torch.zeros_like(s["lens"]), torch.zeros_like(s["n_free"])
    s["slots"] = torch.zeros((B, K), dtype=torch.int32, device="cuda")
    s["granted"] = torch.zeros((B,), dtype=torch.int32, device="cuda")
    if case["released"]:
        s["release"] = torch.tensor(gone, dtype=torch.uint8, device="cuda")
        s["table_before"], s["free_before"] = s["table"].clone(), s["free"].clone()
    return s


def _slots_of(lens, K, table, page, skip=()):
    """Slots of rows len .. len + K - 1 of each sequence (host lists and a host table); -1 for skipped sequences."""
    t = torch.tensor(lens).view(-1, 1) + torch.arange(K)
    s = table.long().gather(1, t // page) * page + t % page
    for b in skip:
        s[b] = -1
    return s.to(torch.int32).cuda()


def _prepare_norm_rope(case, seed):
    dt, B, K, Hq, Hkv, D = _dtype(case), case["B"], case["K"], case["Hq"], case["Hkv"], case["D"]
    # q, k and v as a fused projection leaves them: one row per token, the heads side by side
    qkv = _normal(seed, 10, (B, K, Hq + 2 * Hkv, D), dt, 2.0)
    s = {"case": case}
    s["q"], s["k"], s["v"] = (x.transpose(1, 2) for x in qkv.split([Hq, Hkv, Hkv], 2))
    s["wq"] = _normal(seed, 11, (D,), dt, 0.1, 1.0) if case["norm"] else None
    s["wk"] = _normal(seed, 12, (D,), dt, 0.1, 1.0) if case["norm"] else None
    starts = _dealt(_spread(0, case["pos_hi"], B), seed, 1)
    if case["per_row"]:            # rows that were picked from a longer stretch keep their positions
        pos = torch.tensor(starts).view(B, 1) + torch.rand((B, 2 * K), generator=_gen(seed, 2, "cpu")).argsort(1)[:, :K].sort(1).values
        s["pos"] = pos.to(torch.int32).cuda()
    else:
        s["pos"] = _int32(starts)
    s["q_out"] = torch.zeros((B, Hq, K, D), dtype=dt, device="cuda")
    if case["pages"]:
        page = case["pages"]
        at = [p % page for p in starts]                      # the sequence's last page is partly full
        table, _, n_pages = _tables([a + K for a in at], page, -(-(page + K) // page), seed)
        s["slots"] = _slots_of(at, K, table, page)
        s["k_pages"] = _normal(seed, 13, (n_pages, Hkv, page, D), dt)
        s["v_pages"] = _normal(seed, 14, (n_pages, Hkv, page, D), dt)
        s["k_out"] = None
    else:
        s["k_out"] = torch.zeros((B, Hkv, K, D), dtype=dt, device="cuda")
    return s


def _prepare_append(case, seed):
    dt, L, B, K, Hkv, D, page = _dtype(case), case["L"], case["B"], case["K"], case["Hkv"], case["D"], case["page"]
    lens = [int(x) for x in torch.randint(0, page, (B,), generator=_gen(seed, 1, "cpu"))]
    width = -(-(page + K) // page)
    table, _, n_pages = _tables([n + K for n in lens], page, width, seed, B * width + 3)
    skip = torch.randperm(B, generator=_gen(seed, 2, "cpu")).tolist()[:int(case["skipped"] * B)]
    s = {"case": case, "slots": _slots_of(lens, K, table, page, skip)}
    for i, x in enumerate("kv"):
        s[x + "_pages"] = _normal(seed, 10 + i, (L, n_pages, Hkv, page, D), dt)
        s[x + "_blocks"] = _normal(seed, 20 + i, (L, B, Hkv, K, D), dt)
    return s


def _prepare_attention(case, seed):
    dt, B, Hq, Hkv, D, K, page = (_dtype(case),) + tuple(case[x] for x in ("B", "Hq", "Hkv", "D", "K", "page"))
    lens = _dealt(_lens(case), seed, 1)
    q_lens = _dealt(_q_lens(case), seed, 2)
    if not case["block"]:                                    # the queries' own rows are in the cache
        q_lens = [min(q, n) for q, n in zip(q_lens, lens)]
    table, _, n_pages = _tables(lens, page, -(-case["len_hi"] // page) + 1, seed)
    s = {"case": case, "host_lens": lens, "host_q_lens": q_lens, "table": table.cuda(), "lens": _int32(lens)}
    s["q_lens"] = _int32(q_lens) if min(q_lens) < K else None
    s["q"] = _normal(seed, 10, (B, Hq, K, D), dt)
    s["k_pages"] = _normal(seed, 11, (n_pages, Hkv, page, D), dt)
    s["v_pages"] = _normal(seed, 12, (n_pages, Hkv, page, D), dt)
    s["k_block"] = _normal(seed, 13, (B, Hkv, K, D), dt) if case["block"] else None
    s["v_block"] = _normal(seed, 14, (B, Hkv, K, D), dt) if case["block"] else None
    s["out"] = torch.zeros((B, Hq, K, D), dtype=dt, device="cuda")
    return s


_PREPARE = {"extend": _prepare_extend, "norm_rope": _prepare_norm_rope, "append": _prepare_append, "attention": _prepare_attention}


def prepare(case, seed):
    state = _PREPARE[case["kind"]](case, seed)
    # a serving loop over fixed buffers marshals its calls once
    state["bound"] = _calls(state, "bind_")() if own and case["calls"] == "bound" else None
    return state


# ---------------------------------------------------------------------------------------------- the framework's calls
def _calls(s, form):
    """The framework's call of a state, as a function without arguments: the one-shot form ("") or the marshalled one ("bind_")."""
    import paper_2601_17917_amd as sd
    case = s["case"]
    if case["kind"] == "extend":
        def call():
            return getattr(sd, form + "paged_extend")(s["table"], s["lens"], s["free"], s["n_free"], case["page"], case["K"],
                                                      new_lens=s["new"], release=s["release"], kv_lens_out=s["lens_out"],
                                                      n_free_out=s["n_free_out"], slots=s["slots"], granted=s["granted"])
    elif case["kind"] == "norm_rope":
        def call():
            paged = dict(v=s["v"], k_pages=s["k_pages"], v_pages=s["v_pages"], slots=s["slots"]) if case["pages"] else dict(k_out=s["k_out"])
            return getattr(sd, form + "qk_norm_rope")(s["q"], s["k"], s["pos"], THETA, q_weight=s["wq"], k_weight=s["wk"], eps=1e-6,
                                                      rotary_dim=case["rotary"], interleaved=case["interleaved"],
                                                      scale_factor=case["factor"], original_len=case["original"],
                                                      amplitude=case["amplitude"], q_out=s["q_out"], **paged)
    elif case["kind"] == "append":
        def call():
            return getattr(sd, form + "paged_kv_append")(s["k_pages"], s["v_pages"], s["k_blocks"], s["v_blocks"], s["slots"])
    else:
        def call():
            return getattr(sd, form + "paged_attention")(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], case["len_hi"],
                                                         k_block=s["k_block"], v_block=s["v_block"], q_lens=s["q_lens"],
                                                         causal=case["causal"], window=case["window"], sinks=case["sinks"],
                                                         out=s["out"])
    return call


def run(state):
    kind = state["case"]["kind"]
    if kind == "extend" and state["release"] is not None:
        # pages that were given back change the table and the stack: both start as they were, so that a pass can be repeated
        state["table"].copy_(state["table_before"])
        state["free"].copy_(state["free_before"])
    if not own:
        _PLAIN[kind](state)
    elif state["bound"] is not None:
        state["bound"]()
    else:
        _calls(state, "")()
    return {x: state[x] for x in _outputs(state["case"])}


def _outputs(case):
    if case["kind"] == "extend":
        return ("table", "lens_out", "n_free_out", "slots", "granted", "free")
    if case["kind"] == "norm_rope":
        return ("q_out", "k_pages", "v_pages") if case["pages"] else ("q_out", "k_out")
    return ("k_pages", "v_pages") if case["kind"] == "append" else ("out",)


# ---------------------------------------------------------------------------------------------- plain forms
def _plain_extend(s):
    case = s["case"]
    page, K = case["page"], case["K"]
    table, free = s["table"], s["free"]
    width, n_pages = table.shape[1], free.shape[0]
    cols = torch.arange(width, device="cuda")
    lens, n_free = s["lens"].long(), s["n_free"].long()
    if s["release"] is not None:
        gone = s["release"] != 0
        back = (gone.view(-1, 1) & (cols < ((lens + page - 1) // page).view(-1, 1))).view(-1)
        count = back.long().cumsum(0)
        dest = torch.where(back, n_free + count - 1, n_pages)
        room = torch.cat([free, free.new_zeros(1)])
        room.scatter_(0, dest, torch.where(back, table.view(-1), 0))
        free.copy_(room[:n_pages])
        n_free = n_free + count[-1:]
        lens = torch.where(gone, 0, lens)
    new = s["new"].long().clamp(0, K)
    held = (lens + page - 1) // page
    need = (lens + new + page - 1) // page - held
    fits = lens + new <= width * page
    need = torch.where(fits, need, 0)
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= n_free))
    base = upto - need
    taken = torch.where(ok & (need > 0), upto, 0).max()
    granted = torch.where(ok, new, 0)
    # table entries held .. held + need - 1 of the sequences that got their pages
    i = cols.view(1, -1) - held.view(-1, 1)
    fresh = ok.view(-1, 1) & (i >= 0) & (i < need.view(-1, 1))
    at = (n_free - 1 - base.view(-1, 1) - i).clamp(0, n_pages - 1)
    table.copy_(torch.where(fresh, free[at], table))
    t = torch.arange(K, device="cuda").view(1, -1)
    pos = lens.view(-1, 1) + t
    slots = table.long().gather(1, (pos // page).clamp(max=width - 1)) * page + pos % page
    s["slots"].copy_(torch.where(t < granted.view(-1, 1), slots, -1))
    s["granted"].copy_(granted)
    s["lens_out"].copy_(lens + granted)
    s["n_free_out"].copy_(n_free - taken)


def _frequencies(case):
    """Radians per position of each pair, in 64 bits."""
    R, factor = case["rotary"], case["factor"]
    f = THETA ** (-2.0 * torch.arange(R // 2, dtype=torch.float64, device="cuda") / R)
    if factor == 1.0:
        return f
    if case["original"] == 0:
        return f / factor
    u = ((f * case["original"] / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    return u * f + (1 - u) * f / factor


def _plain_head_rows(x, w, pos, case):
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w.float()
    R = case["rotary"]
    angle = pos[:, None, :, None].double() * _frequencies(case)
    c, sn = (angle.cos() * case["amplitude"]).float(), (angle.sin() * case["amplitude"]).float()
    if case["interleaved"]:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        turned = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    else:
        a, b = y[..., :R // 2], y[..., R // 2:R]
        turned = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    return torch.cat([turned, y[..., R:]], -1).to(x.dtype)


def _to_pages(pages, slots, rows):
    """pages[slot's page, :, slot's row] <- rows [B, H, K, D]."""
    page = pages.shape[-2]
    flat = slots.view(-1).long()
    pages[flat // page, :, flat % page] = rows.transpose(1, 2).flatten(0, 1)


def _plain_norm_rope(s):
    case = s["case"]
    pos = s["pos"] if case["per_row"] else s["pos"].view(-1, 1) + torch.arange(case["K"], device="cuda")
    s["q_out"].copy_(_plain_head_rows(s["q"], s["wq"], pos, case))
    k = _plain_head_rows(s["k"], s["wk"], pos, case)
    if case["pages"]:
        _to_pages(s["k_pages"], s["slots"], k)
        _to_pages(s["v_pages"], s["slots"], s["v"])
    else:
        s["k_out"].copy_(k)


def _plain_append(s):
    """Every layer's rows into their slots; rows whose slot is -1 are left out."""
    slots = s["slots"].view(-1).long()
    L, n_pages, Hkv, page, D = s["k_pages"].shape
    for x in "kv":
        # a row of the pool behind the last takes what has no slot
        pool = torch.cat([s[x + "_pages"].transpose(2, 3).reshape(L, n_pages * page, Hkv, D), s[x + "_pages"].new_zeros(L, 1, Hkv, D)], 1)
        rows = s[x + "_blocks"].transpose(2, 3).reshape(L, -1, Hkv, D)
        pool[:, torch.where(slots < 0, n_pages * page, slots)] = rows
        s[x + "_pages"].copy_(pool[:, :n_pages * page].view(L, n_pages, page, Hkv, D).transpose(2, 3))


def _plain_attention(s):
    case = s["case"]
    Hq, Hkv, K, D, page = (case[x] for x in ("Hq", "Hkv", "K", "D", "page"))
    g = Hq // Hkv
    for b, (n, q) in enumerate(zip(s["host_lens"], s["host_q_lens"])):
        ids = s["table"][b, :-(-n // page)].long()
        k = s["k_pages"][ids].float().transpose(0, 1).reshape(Hkv, -1, D)[:, :n]
        v = s["v_pages"][ids].float().transpose(0, 1).reshape(Hkv, -1, D)[:, :n]
        if case["block"]:
            k = torch.cat([k, s["k_block"][b, :, :q].float()], 1)
            v = torch.cat([v, s["v_block"][b, :, :q].float()], 1)
        total = k.shape[1]
        rows = s["q"][b, :, :q].float().reshape(Hkv, g * q, D)
        z = torch.matmul(rows, k.transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(D)).view(Hkv, g, q, total)
        if case["causal"] or case["window"]:
            j = torch.arange(total, device="cuda").view(1, -1)
            p = torch.arange(total - q, total, device="cuda").view(-1, 1)
            seen = j <= p if case["causal"] else torch.ones_like(j <= p)
            if case["window"]:
                seen = seen & ((p - j < case["window"]) | (j < case["sinks"]))
            z.masked_fill_(~seen, -math.inf)
        z = z.sub_(z.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
        total_weight = z.sum(-1, keepdim=True)
        z = torch.where(total_weight > 0, z / total_weight, 0.0).view(Hkv, g * q, total)
        s["out"][b, :, :q] = torch.matmul(z, v).view(Hq, q, D).to(s["out"].dtype)


_PLAIN = {"extend": _plain_extend, "norm_rope": _plain_norm_rope, "append": _plain_append, "attention": _plain_attention}


# ---------------------------------------------------------------------------------------------- 64 bits
def _exact_rotated(x, w, s):
    """norm_rope by complex numbers: pair (a, b) is a + ib times amplitude * exp(i angle)."""
    case = s["case"]
    B, H, K, D = x.shape
    R = case["rotary"]
    y = x.double()
    if w is not None:
        y = y / (y.pow(2).sum(-1, keepdim=True) / D + 1e-6).sqrt() * w.double()
    i = torch.arange(0, R, 2, dtype=torch.float64, device="cuda")
    f = torch.exp(-i / R * math.log(THETA))
    if case["factor"] != 1.0:
        share = torch.zeros_like(f)
        if case["original"]:
            turns = case["original"] * f / (2 * math.pi)
            share = torch.where(turns < 1.0, 0.0, torch.where(turns > 32.0, 1.0, (turns - 1.0) / (32.0 - 1.0)))
        f = f * (share + (1.0 - share) / case["factor"])
    pos = s["pos"].double() if case["per_row"] else s["pos"].double().view(B, 1) + torch.arange(K, device="cuda")
    turn = torch.polar(torch.full_like(pos[..., None] * f, case["amplitude"]), pos[..., None] * f)[:, None]
    head = y[..., :R].reshape(B, H, K, R // 2, 2) if case["interleaved"] else y[..., :R].reshape(B, H, K, 2, R // 2).transpose(-1, -2)
    out = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
    out = out if case["interleaved"] else out.transpose(-1, -2)
    return torch.cat([out.reshape(B, H, K, R), y[..., R:]], -1)


def _exact_attention(s):
    case = s["case"]
    Hq, Hkv, D, page, w = (case[x] for x in ("Hq", "Hkv", "D", "page", "window"))
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    table = s["table"].tolist()
    for b, (n, q) in enumerate(zip(s["host_lens"], s["host_q_lens"])):
        total = n + (q if case["block"] else 0)
        slots = torch.tensor([table[b][t // page] * page + t % page for t in range(n)], dtype=torch.long, device="cuda")
        distance = torch.arange(total - q, total, device="cuda")[:, None] - torch.arange(total, device="cuda")[None]
        hidden = torch.zeros_like(distance, dtype=torch.bool)
        if case["causal"]:
            hidden |= distance < 0
        if w:
            hidden |= (distance >= w) & (torch.arange(total, device="cuda")[None] >= case["sinks"])
        for h in range(Hkv):
            k = s["k_pages"][:, h].reshape(-1, D)[slots].double()
            v = s["v_pages"][:, h].reshape(-1, D)[slots].double()
            if case["block"]:
                k, v = torch.cat([k, s["k_block"][b, h, :q].double()]), torch.cat([v, s["v_block"][b, h, :q].double()])
            for m in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                z = s["q"][b, m, :q].double() @ k.t() / math.sqrt(D)
                p = torch.softmax(z.masked_fill(hidden, -math.inf), -1)
                out[b, m, :q] = torch.where(hidden.all(-1, keepdim=True), 0.0, torch.nan_to_num(p) @ v)
    return out


def _exact_pages(pages, slots, rows):
    """pages [L, n_pages, Hkv, page, D] with rows [L, B, Hkv, K, D] in their slots."""
    pool = pages.double()
    for b, of_b in enumerate(slots.tolist()):
        kept = [t for t, slot in enumerate(of_b) if slot >= 0]
        at = torch.tensor([of_b[t] for t in kept], dtype=torch.long, device="cuda")
        for layer, r in zip(pool, rows):
            layer[at // pool.shape[3], :, at % pool.shape[3]] = r[b][:, kept].double().transpose(0, 1)
    return pool


def exact(case, seed):
    if case["kind"] == "extend":
        return None                                          # whole numbers
    s = prepare(dict(case, calls="plain"), seed)
    if case["kind"] == "append":
        return {x + "_pages": _exact_pages(s[x + "_pages"], s["slots"], s[x + "_blocks"]) for x in "kv"}
    if case["kind"] == "attention":
        return {"out": _exact_attention(s)}
    out = {"q_out": _exact_rotated(s["q"], s["wq"], s)}
    k = _exact_rotated(s["k"], s["wk"], s)
    if not case["pages"]:
        return dict(out, k_out=k)
    for x, rows in (("k_pages", k), ("v_pages", s["v"])):
        out[x] = _exact_pages(s[x][None], s["slots"], rows[None])[0]
    return out
