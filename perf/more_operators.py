"""Measured operators: rotary positions, appending to a paged key/value cache, attention over it.

  rope       heads turned by their positions: half or interleaved pairs, part of the head, scaled for long contexts (spd_rope_apply)
  append     new keys (turned on the way) and values into the pages of their sequences, the queries turned beside them (spd_paged_append)
  attention  a chunk of new rows of each sequence over its pages: one token, a verify block or a tree of drafts, a prompt (spd_paged_attention)

A page holds page_size positions of every head, in granules of 16 bytes, G elements (8 in bfloat16, 16 in e4m3):
keys [n_pages, kv_heads, dim / G, page_size, G], values [n_pages, kv_heads, page_size / G, dim, G].  e4m3 values stand for
themselves times their head's scale.  With `own` false the same in elementary torch operations, over sequences padded to the longest.
"""
import math

import torch

own = False

DEV = "cuda"


def listed():
    half = {"rotary": 128, "interleaved": False, "scaling": "none", "theta": 10000.0}
    causal = {"window": 0, "tree": False}
    return [
        # ---- rotary positions: the queries of one token of the 12-layer draft.  The smallest call: launch and latency.
        {"name": "rope_token", "kind": "rope", "rows": 1, "heads": 12, "dim": 64, "far": 2048, "bf16": False, "pad": 0, "inverse": False, **half, "rotary": 64},
        # the queries of a pass of 7B-shaped prompts, four conversations' worth, a context stretched by bands of wavelengths
        {"name": "rope_prompt", "kind": "rope", "rows": 8192, "heads": 32, "dim": 128, "far": 65536, "bf16": True, "pad": 0, "inverse": False, **half,
         "scaling": "ramp", "theta": 500000.0},
        # neighbouring pairs in the first part of a head, turned back, far positions, an odd number of rows in a wider buffer
        {"name": "rope_part_back", "kind": "rope", "rows": 3001, "heads": 20, "dim": 96, "far": 1000000, "bf16": False, "pad": 24, "inverse": True,
         "rotary": 40, "interleaved": True, "scaling": "log_ramp", "theta": 10000.0},
        # ---- append: the verify block of one conversation at draft length 4, 7B shape
        {"name": "append_verify", "kind": "append", "seqs": 1, "new_lo": 5, "new_hi": 5, "len_lo": 640, "len_hi": 640, "heads": 32, "kv_heads": 32, "dim": 128,
         "page": 16, "e4m3": False, "bf16": False, **half},
        # prompts of four conversations in one batch, eight key heads
        {"name": "append_prompts", "kind": "append", "seqs": 4, "new_lo": 1500, "new_hi": 2048, "len_lo": 0, "len_hi": 700, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "e4m3": False, "bf16": True, **half, "scaling": "linear"},
        # tokens and pieces of prompts mixed, an 8-bit cache, part of the head turned in neighbouring pairs
        {"name": "append_mixed_e4m3", "kind": "append", "seqs": 37, "new_lo": 1, "new_hi": 131, "len_lo": 3, "len_hi": 5000, "heads": 16, "kv_heads": 4, "dim": 64,
         "page": 32, "e4m3": True, "bf16": True, "rotary": 32, "interleaved": True, "scaling": "none", "theta": 10000.0},
        # ---- attention: one token of one conversation behind an image and a short text, 7B shape
        {"name": "attention_token", "kind": "attention", "seqs": 1, "new_lo": 1, "new_hi": 1, "len_lo": 640, "len_hi": 640, "heads": 32, "kv_heads": 32, "dim": 128,
         "page": 16, "e4m3": False, "bf16": False, **causal},
        # trees of drafted tokens of eight conversations
        {"name": "attention_trees", "kind": "attention", "seqs": 8, "new_lo": 9, "new_hi": 16, "len_lo": 1500, "len_hi": 2047, "heads": 32, "kv_heads": 32, "dim": 128,
         "page": 32, "e4m3": False, "bf16": False, "window": 0, "tree": True},
        # a decoding batch of uneven conversations, eight key heads
        {"name": "attention_batch", "kind": "attention", "seqs": 64, "new_lo": 1, "new_hi": 1, "len_lo": 100, "len_hi": 8000, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "e4m3": False, "bf16": True, **causal},
        # long documents in an 8-bit cache
        {"name": "attention_long_e4m3", "kind": "attention", "seqs": 4, "new_lo": 1, "new_hi": 5, "len_lo": 60000, "len_hi": 131000, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "e4m3": True, "bf16": True, **causal},
        # a whole prompt
        {"name": "attention_prompt", "kind": "attention", "seqs": 1, "new_lo": 4096, "new_hi": 4096, "len_lo": 0, "len_hi": 0, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "e4m3": False, "bf16": True, **causal},
        # pieces of prompts over caches, seven queries a key head, a sliding window, float32 rows
        {"name": "attention_pieces", "kind": "attention", "seqs": 5, "new_lo": 1, "new_hi": 700, "len_lo": 0, "len_hi": 6000, "heads": 14, "kv_heads": 2, "dim": 64,
         "page": 16, "e4m3": False, "bf16": False, "window": 1000, "tree": False},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "append", "attention", "attention", "attention"])
    dim = rng.choice([64, 128])
    turn = {"rotary": rng.choice([dim, dim // 2, 2 * rng.randint(1, dim // 2)]), "interleaved": rng.random() < 0.5,
            "scaling": rng.choice(["none", "linear", "ramp", "log_ramp"]), "theta": rng.choice([10000.0, 500000.0])}
    if kind == "rope":
        dim = rng.choice([64, 80, 96, 128, 2 * rng.randint(8, 128)])
        heads = _log_int(rng, 1, 64)
        rows = _log_int(rng, 1, min(8192, 8192 * 32 * 128 // (heads * dim)))
        return {"kind": kind, "rows": rows, "heads": heads, "dim": dim, "far": _log_int(rng, 100, 1000000), "bf16": rng.random() < 0.5, "pad": rng.choice([0, 0, 8, 6]),
                "inverse": rng.random() < 0.25, **turn, "rotary": rng.choice([dim // 4 * 2, dim, 2 * rng.randint(1, dim // 2)])}
    kv_heads = rng.choice([1, 2, 4, 8, 12, 32])
    heads = min(kv_heads * rng.choice([1, 1, 2, 3, 4, 7, 8]), 64 // kv_heads * kv_heads)
    seqs = _log_int(rng, 1, 64)
    e4m3 = rng.random() < 0.35
    case = {"kind": kind, "seqs": seqs, "new_lo": 1, "new_hi": 1, "len_lo": 0, "len_hi": 0, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "page": rng.choice([16, 32, 64, 128, 256]), "e4m3": e4m3, "bf16": rng.random() < 0.5}
    if kind == "append":
        rows = _log_int(rng, seqs, 8192 * 48 // max(48, heads + 2 * kv_heads))
        case["new_hi"] = max(1, rows // seqs)
        case["new_lo"] = rng.choice([1, case["new_hi"]])
        case["len_hi"] = _log_int(rng, 1, max(1, min(8000, 250000000 // (seqs * kv_heads * dim) - case["new_hi"])))
        case["len_lo"] = rng.choice([0, case["len_hi"]])
        return {**case, **turn}
    tree = rng.random() < 0.2
    case["new_hi"] = rng.choice([1, _log_int(rng, 2, 64)]) if tree or rng.random() < 0.7 else min(_log_int(rng, 64, 4096), max(64, 8192 // seqs))
    # the scores of padded sequences, and what the caches hold, stay below those of the largest listed cases
    case["new_hi"] = min(case["new_hi"], math.isqrt(250000000 // (seqs * heads)))
    case["new_lo"] = rng.choice([1, case["new_hi"]])
    most = min(250000000 // (seqs * heads * case["new_hi"]), 250000000 // (seqs * kv_heads * dim), 131000)
    case["len_hi"] = min(_log_int(rng, 1, 131000), max(0, most - case["new_hi"]))
    case["len_lo"] = rng.choice([0, case["len_hi"] // 10, case["len_hi"]])
    return {**case, "window": rng.choice([0, 0, 0, _log_int(rng, 1, 8000)]) if not tree else 0, "tree": tree}


# ---- inputs -----------------------------------------------------------------------------------------------------

def _spread(lo, hi, n):
    """n whole numbers from lo to hi, not in order."""
    return [lo + (hi - lo) * (s * 7919 % n) // max(1, n - 1) for s in range(n)]


def _sizes(case):
    """New rows and cached positions of each sequence."""
    new = _spread(case["new_lo"], case["new_hi"], case["seqs"])
    return new, _spread(case["len_lo"], case["len_hi"], case["seqs"])[::-1]


def _frequencies(case):
    """Radians a position of each pair, float64."""
    n = case["rotary"] // 2
    f = case["theta"] ** (-torch.arange(n, dtype=torch.float64) * 2.0 / case["rotary"])
    turns = 8192 * f / (2 * math.pi)
    if case["scaling"] == "linear":
        return f / 4.0
    if case["scaling"] == "ramp":
        keep = ((turns - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f * (keep + (1 - keep) / 8.0)
    if case["scaling"] == "log_ramp":
        keep = (torch.log(turns / 1.0) / math.log(32.0 / 1.0)).clamp(0, 1)
        return f * (keep + (1 - keep) / 8.0)
    return f


def _magnitude(case):
    return 0.1 * math.log(8.0) + 1.0 if case["scaling"] == "log_ramp" else 1.0


def _plan(case):
    """The framework's form of the same."""
    from paper_2404_08856_amd import spd
    kinds = {"none": {}, "linear": {"scaling": spd.SPD_ROPE_LINEAR, "factor": 4.0},
             "ramp": {"scaling": spd.SPD_ROPE_RAMP, "factor": 8.0, "low": 1.0, "high": 4.0, "original_positions": 8192},
             "log_ramp": {"scaling": spd.SPD_ROPE_LOG_RAMP, "factor": 8.0, "low": 1.0, "high": 32.0, "original_positions": 8192}}
    return spd.Rope(case["rotary"], theta=case["theta"], interleaved=case["interleaved"], magnitude=_magnitude(case), **kinds[case["scaling"]])


def _rows(g, rows, heads, dim, bf16, size=1.0):
    x = size * torch.randn((rows, heads, dim), generator=g, device=DEV)
    return x.bfloat16() if bf16 else x


def prepare(case, seed):
    """What a program holds before the call: rows of projections, the cache's pages with the tables of its sequences."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": case}
    if case["kind"] != "attention":
        s["frequencies"] = _frequencies(case).to(DEV)
        if own:
            s["rope"] = _plan(case)
    dtype = torch.bfloat16 if case["bf16"] else torch.float32
    if case["kind"] == "rope":
        wide = _rows(g, case["rows"], 1, case["heads"] * case["dim"] + case["pad"], case["bf16"])
        s["x"] = wide[:, 0, : case["heads"] * case["dim"]].unflatten(1, (case["heads"], case["dim"]))
        s["positions"] = torch.randint(0, case["far"], (case["rows"],), generator=g, device=DEV, dtype=torch.int32)
        s["out"] = torch.empty((case["rows"], case["heads"], case["dim"]), dtype=dtype, device=DEV)
        return s
    new, lens = _sizes(case)
    H, HK, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    rows = sum(new)
    each = [(a + b + P - 1) // P for a, b in zip(new, lens)]
    n_pages = sum(each) + 3
    G = 16 if case["e4m3"] else 8
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros((case["seqs"], max(each)), dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(each):
        table[i, :n] = order[at : at + n]
        at += n
    s["table"] = table
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["row_start"] = torch.tensor([sum(new[:i]) for i in range(case["seqs"] + 1)], dtype=torch.int32, device=DEV)
    s["most"] = (max(new), max(a + b for a, b in zip(new, lens)))
    # values of a channel have a mean of their own
    k = torch.randn((n_pages, HK, D // G, P, G), generator=g, device=DEV)
    v = torch.randn((n_pages, HK, P // G, D, G), generator=g, device=DEV) + torch.randn((1, HK, 1, D, 1), generator=g, device=DEV)
    if case["e4m3"]:
        s["scales"] = [0.01 + 0.02 * torch.rand((HK,), generator=g, device=DEV) for _ in "kv"]
        k, v = [(t / c.view(1, HK, 1, 1, 1)).clamp(-448, 448).to(torch.float8_e4m3fn) for t, c in zip((k, v), s["scales"])]
    else:
        k, v = k.bfloat16(), v.bfloat16()
    s["k_pages"], s["v_pages"] = k, v
    if own:
        from paper_2404_08856_amd import spd
        s["cache"] = spd.PagedCache(k, v, *s.get("scales", ()))
        s["batch"] = spd.PagedBatch(table, s["lens"], rows, s["row_start"])
    if case["kind"] == "append":
        s["qkv"] = _rows(g, rows, H + 2 * HK, D, case["bf16"])
        s["q_out"] = torch.empty((rows, H, D), dtype=dtype, device=DEV)
        return s
    s["q"] = _rows(g, rows, H, D, case["bf16"], 2.0)
    s["seen"] = None
    if case["tree"]:                                       # every drafted token sees itself, the token it follows and what that one sees
        parents = torch.randint(0, 1 << 30, (rows,), generator=g, device=DEV).tolist()
        words, at = [], 0
        for n in new:
            seen = []
            for j in range(n):
                seen.append((seen[parents[at + j] % j] if j else 0) | 1 << j)
            words += seen
            at += n
        s["seen"] = torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, device=DEV)
    s["out"] = torch.empty((rows, H, D), dtype=dtype, device=DEV)
    s["lse"] = torch.empty((rows, H), dtype=torch.float32, device=DEV)
    if own:
        s["workspace"] = torch.empty(max(1, spd.spd_paged_attention_workspace_bytes(s["cache"], s["batch"], H)), dtype=torch.uint8, device=DEV)
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------

def _turned(x, positions, frequencies, case, back=False):
    """x [rows, heads, dim] turned, in float32."""
    angle = positions.double()[:, None] * frequencies
    cos = (torch.cos(angle) * _magnitude(case)).float()[:, None]
    sin = (torch.sin(angle) * _magnitude(case) * (-1.0 if back else 1.0)).float()[:, None]
    R = case["rotary"]
    x = x.float()
    turn, rest = x[..., :R], x[..., R:]
    if case["interleaved"]:
        a, b = turn[..., 0::2], turn[..., 1::2]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), rest], -1)
    a, b = turn[..., : R // 2], turn[..., R // 2 :]
    return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], -1)


def _places(s, rows):
    """Sequence, index among its new rows, and position of each row."""
    row = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(s["row_start"], row.to(torch.int32), right=True) - 1
    i = row - s["row_start"][seq]
    return seq, i, s["lens"][seq] + i


def _append(s):
    c = s["case"]
    H, HK, P = c["heads"], c["kv_heads"], c["page"]
    q, k, v = s["qkv"].split([H, HK, HK], 1)
    seq, _, pos = _places(s, q.shape[0])
    q, k, v = _turned(q, pos, s["frequencies"], c), _turned(k, pos, s["frequencies"], c), v.float()
    kp, vp = s["k_pages"], s["v_pages"]
    if c["e4m3"]:
        k, v = [(t / scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for t, scale in zip((k, v), s["scales"])]
        kp, vp = kp.view(torch.uint8), vp.view(torch.uint8)
    else:
        k, v = k.bfloat16(), v.bfloat16()
    G = kp.shape[-1]
    page, slot = s["table"][seq, pos // P].long(), pos % P
    kp[page, :, :, slot] = k.unflatten(-1, (-1, G))
    vp[page, :, slot // G, :, slot % G] = v
    s["q_out"].copy_(q)
    return [s["q_out"], s["k_pages"], s["v_pages"]]


def _attention(s):
    c = s["case"]
    H, HK, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    most_new, most_keys = s["most"]
    B, rows, group = c["seqs"], s["q"].shape[0], H // HK
    seq, i, pos = _places(s, rows)
    # the pages of each sequence as [sequences, heads, keys, dim]
    kp, vp = s["k_pages"].view(torch.uint8 if c["e4m3"] else torch.bfloat16), s["v_pages"].view(torch.uint8 if c["e4m3"] else torch.bfloat16)
    table = s["table"].long()
    k = kp[table].to(torch.uint8 if c["e4m3"] else torch.float32).permute(0, 2, 1, 4, 3, 5).reshape(B, HK, -1, D)
    v = vp[table].to(torch.uint8 if c["e4m3"] else torch.float32).permute(0, 2, 1, 3, 5, 4).reshape(B, HK, -1, D)
    if c["e4m3"]:
        k, v = [t.view(torch.float8_e4m3fn).float() * scale[:, None, None] for t, scale in zip((k, v), s["scales"])]
    k, v = k[:, :, :most_keys], v[:, :, :most_keys]
    keys = k.shape[2]
    q = torch.zeros((B, most_new, H, D), device=DEV)
    q[seq, i] = s["q"].float()
    q = q.view(B, most_new, HK, group, D).permute(0, 2, 3, 1, 4).reshape(B, HK, group * most_new, D)
    scores = (torch.matmul(q, k.transpose(2, 3)) / math.sqrt(D)).view(B, HK, group, most_new, keys)
    # which keys each new row of a sequence sees
    key = torch.arange(keys, device=DEV)
    old = s["lens"][:, None, None].long()
    own_pos = old + torch.arange(most_new, device=DEV)[None, :, None]
    if c["tree"]:
        words = torch.zeros((B, most_new), dtype=torch.int64, device=DEV)
        words[seq, i] = s["seen"]
        bit = (key - old).clamp(0, 63)
        sees = (key < old) | ((key >= old) & (key - old < 64) & ((words[:, :, None] >> bit) & 1).bool())
    else:
        sees = key <= own_pos
        if c["window"]:
            sees = sees & (key > own_pos - c["window"])
    scores = scores.masked_fill(~sees[:, None, None], -math.inf)
    best = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(best > -math.inf, best, torch.zeros_like(best)))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, HK, group * most_new, keys), v).view(B, HK, group, most_new, D) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (torch.log(total) + best)[..., 0]
    s["out"].copy_(out.permute(0, 3, 1, 2, 4).reshape(B, most_new, H, D)[seq, i])
    s["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(B, most_new, H)[seq, i])
    return [s["out"], s["lse"]]


def run(state):
    c = state["case"]
    if own:
        from paper_2404_08856_amd import spd
        if c["kind"] == "rope":
            spd.spd_rope_apply(state["rope"], state["x"], state["positions"], state["out"], inverse=c["inverse"])
            return state["out"]
        if c["kind"] == "append":
            q, k, v = state["qkv"].split([c["heads"], c["kv_heads"], c["kv_heads"]], 1)
            spd.spd_paged_append(state["cache"], state["batch"], k, v, rope=state["rope"], q=q, q_out=state["q_out"])
            return [state["q_out"], state["k_pages"], state["v_pages"]]
        spd.spd_paged_attention(state["cache"], state["batch"], state["q"], state["out"], window=c["window"], seen=state["seen"], lse_out=state["lse"], workspace=state["workspace"])
        return [state["out"], state["lse"]]
    if c["kind"] == "rope":
        state["out"].copy_(_turned(state["x"], state["positions"], state["frequencies"], c, c["inverse"]))
        return state["out"]
    return _append(state) if c["kind"] == "append" else _attention(state)


# ---- in 64 bits -------------------------------------------------------------------------------------------------

def _complex_turned(x, positions, case, back):
    """The first rotary elements as complex numbers, times e^(i position frequency)."""
    R = case["rotary"]
    x = x.double()
    pairs = x[..., :R].unflatten(-1, (R // 2, 2)) if case["interleaved"] else x[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous())
    angle = positions.double()[:, None] * _frequencies(case).to(DEV)
    z = z * torch.polar(torch.full_like(angle, _magnitude(case)), -angle if back else angle)[:, None]
    turned = torch.view_as_real(z)
    turned = turned.flatten(-2) if case["interleaved"] else turned.transpose(-1, -2).flatten(-2)
    return torch.cat([turned, x[..., R:]], -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return _complex_turned(s["x"], s["positions"], case, case["inverse"])
    new, lens = _sizes(case)
    H, HK, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    wide = lambda t: t.view(torch.uint8) if case["e4m3"] else t
    if case["kind"] == "append":
        q_out = torch.empty((sum(new), H, D), dtype=torch.float64, device=DEV)
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        at = 0
        for b in range(case["seqs"]):
            rows = s["qkv"][at : at + new[b]]
            pos = lens[b] + torch.arange(new[b], device=DEV)
            q_out[at : at + new[b]] = _complex_turned(rows[:, :H], pos, case, False)
            k, v = _complex_turned(rows[:, H : H + HK], pos, case, False), rows[:, H + HK :].double()
            if case["e4m3"]:
                k, v = [(t / c.double()[:, None]).clamp(-448, 448) for t, c in zip((k, v), s["scales"])]
            page, slot = s["table"][b][(pos // P)].long(), pos % P
            G = k_pages.shape[-1]
            for d in range(0, D, G):
                k_pages[page, :, d // G, slot] = k[..., d : d + G]
            v_pages[page, :, slot // G, :, slot % G] = v
            at += new[b]
        return [q_out, k_pages, v_pages]
    out = torch.empty((sum(new), H, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((sum(new), H), dtype=torch.float64, device=DEV)
    at = 0
    for b in range(case["seqs"]):
        n, keys = new[b], new[b] + lens[b]
        pages = s["table"][b][: (keys + P - 1) // P].long()
        pos = lens[b] + torch.arange(n, device=DEV)
        key = torch.arange(keys, device=DEV)
        sees = key[None] <= pos[:, None]
        if case["window"]:
            sees &= pos[:, None] - key[None] < case["window"]
        if case["tree"]:
            words = s["seen"][at : at + n].tolist()
            for i in range(n):
                for j in range(n):
                    sees[i, lens[b] + j] = bool(words[i] >> j & 1)
        for h in range(HK):
            k, v = wide(s["k_pages"])[pages, h], wide(s["v_pages"])[pages, h]
            if case["e4m3"]:
                k, v = k.view(torch.float8_e4m3fn).float(), v.view(torch.float8_e4m3fn).float()
            k = k.double().permute(0, 2, 1, 3).reshape(-1, D)[:keys]
            v = v.double().permute(0, 1, 3, 2).reshape(-1, D)[:keys]
            if case["e4m3"]:
                k, v = k * s["scales"][0][h].double(), v * s["scales"][1][h].double()
            for j in range(h * (H // HK), (h + 1) * (H // HK)):
                z = (s["q"][at : at + n, j].double() @ k.T.contiguous() / math.sqrt(D)).masked_fill(~sees, -math.inf)
                lse[at : at + n, j] = torch.logsumexp(z, -1)
                out[at : at + n, j] = torch.softmax(z, -1) @ v
        at += n
    return [out, lse]


def work(case):
    one = 2 if case["bf16"] else 4
    if case["kind"] == "rope":
        n = case["rows"] * case["heads"]
        return {"bytes": float(2 * one * n * case["dim"] + 4 * case["rows"]), "flops": 3.0 * n * case["rotary"]}
    new, lens = _sizes(case)
    H, HK, D = case["heads"], case["kv_heads"], case["dim"]
    held = 1 if case["e4m3"] else 2
    if case["kind"] == "append":
        return {"bytes": float(sum(new) * D * (one * (2 * H + 2 * HK) + held * 2 * HK)), "flops": 3.0 * sum(new) * (H + HK) * case["rotary"]}
    w = case["window"] or 1 << 30
    keys = sum(min(n + l, n + w - 1) for n, l in zip(new, lens))
    pairs = sum(n * l + n * (n + 1) // 2 if w >= n + l else sum(min(w, l + i + 1) for i in range(n)) for n, l in zip(new, lens))
    return {"bytes": float(2 * held * keys * HK * D + sum(new) * H * (2 * one * D + 4)), "flops": 4.0 * pairs * H * D}
