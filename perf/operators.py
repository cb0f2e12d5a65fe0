"""The work around a paged key/value cache, as cases that can be timed.

Every case is one pass through an operator on device-resident data:

  window  wq4_window_attention: one new token per sequence attends to the last
          `window` tokens and to the first `sinks` ones
  prompt  wq4_prompt_attention: the new tokens of a prompt (or of a chunk of
          one) attend causally, with or without a window, over the cache
  append  wq4_prompt_append: a prompt's fused QKV rows, queries and keys
          rotated, keys and values written into the cache
  pages   wq4_kv_fork, wq4_kv_compact, wq4_kv_copy_pages, and wq4_kv_trim with
          wq4_kv_reserve: the bookkeeping and the copies of a page pool

Head counts are those of the 3B- and 8B-shaped models of
paper_2412_15803_gb300.model (24 and 32 query heads, 8 key/value heads of 128)
and odd groupings in between.  Pages lie in the pool in random order.  Queries
are scaled so that the scores' standard deviation is 2.5, as peaked as the
attention of trained models; keys and values are normal.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
HEADS = {"8b": (32, 8), "3b": (24, 8), "mha": (16, 16), "mqa": (8, 1), "g5": (10, 2)}
THETA = 500000.0


def listed():
    return [
        # one conversation whose window has just begun to slide: one token's latency
        {"name": "window-8b-b1", "kind": "window", "heads": "8b", "batch": 1, "lo": 700, "hi": 700, "page": 16,
         "window": 512, "sinks": 4},
        # an odd window over a few contexts, some shorter than it
        {"name": "window-3b-b7-odd", "kind": "window", "heads": "3b", "batch": 7, "lo": 90, "hi": 9001, "page": 32,
         "window": 1023, "sinks": 5},
        # a serving batch of long conversations
        {"name": "window-8b-b64", "kind": "window", "heads": "8b", "batch": 64, "lo": 1, "hi": 65536, "page": 16,
         "window": 4096, "sinks": 16},
        # a short prompt of odd length, nothing cached
        {"name": "prompt-3b-77", "kind": "prompt", "heads": "3b", "batch": 1, "new_lo": 77, "new_hi": 77, "ctx": 0,
         "page": 16, "window": 0, "sinks": 0, "pad": 0},
        # a long prompt in one piece
        {"name": "prompt-8b-8192", "kind": "prompt", "heads": "8b", "batch": 1, "new_lo": 8192, "new_hi": 8192, "ctx": 0,
         "page": 16, "window": 0, "sinks": 0, "pad": 0},
        # ragged chunks of several prompts, each with its cached context, under a window; the rows padded
        {"name": "prompt-8b-b5-window", "kind": "prompt", "heads": "8b", "batch": 5, "new_lo": 130, "new_hi": 1500,
         "ctx": 3000, "page": 32, "window": 1024, "sinks": 4, "pad": 37},
        # a follow-up question: a few new tokens over a long cached document
        {"name": "prompt-8b-16-of-32768", "kind": "prompt", "heads": "8b", "batch": 1, "new_lo": 16, "new_hi": 16,
         "ctx": 32752, "page": 16, "window": 0, "sinks": 0, "pad": 0},
        # the QKV rows of ragged prompts behind cached contexts
        {"name": "append-3b-b6", "kind": "append", "heads": "3b", "batch": 6, "new_lo": 1, "new_hi": 301, "ctx": 2000,
         "page": 32, "pad": 5},
        # the QKV rows of a long prompt
        {"name": "append-8b-8192", "kind": "append", "heads": "8b", "batch": 1, "new_lo": 8192, "new_hi": 8192, "ctx": 0,
         "page": 16, "pad": 0},
        # one conversation sampled eight times: its pages shared, the last one copied in every layer
        {"name": "pages-fork-8b", "kind": "pages", "op": "fork", "heads": "8b", "layers": 32, "page": 16, "seqs": 9,
         "pages": 1024, "lo": 500, "hi": 1207, "n": 8},
        # a pool after an hour of serving, its live pages moved to the front
        {"name": "pages-compact-8b", "kind": "pages", "op": "compact", "heads": "8b", "layers": 16, "page": 16, "seqs": 48,
         "pages": 4096, "lo": 1, "hi": 1900, "n": 0},
        # a decode iteration's housekeeping under a window: old pages freed, new ones taken
        {"name": "pages-turn-8b", "kind": "pages", "op": "turn", "heads": "8b", "layers": 1, "page": 16, "seqs": 64,
         "pages": 24576, "lo": 100, "hi": 8192, "n": 64, "window": 4096, "sinks": 16},
    ]


def _log(rng, lo, hi):
    """A whole number spread over [lo, hi] by its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["window", "window", "prompt", "prompt", "prompt", "append", "pages", "pages"])
    heads = rng.choice(["8b", "8b", "3b", "3b", "mha", "mqa", "g5"])
    page = rng.choice([16, 16, 32, 64, 128])
    if kind == "window":
        batch, window = _log(rng, 1, 128), _log(rng, 1, 8192)
        hi = _log(rng, 2, 65536)
        while batch * min(hi, window) > 64 * 4096:
            batch = (batch + 1) // 2
        return {"kind": kind, "heads": heads, "batch": batch, "lo": rng.randint(0, hi), "hi": hi, "page": page, "window": window,
                "sinks": rng.choice([0, 1, 4, 5, 64])}
    if kind in ("prompt", "append"):
        batch, new = _log(rng, 1, 16), _log(rng, 1, 8192)
        ctx = rng.choice([0, _log(rng, 1, 32768)])
        if kind == "prompt":
            while batch * new * (new + ctx) > 8192 * 8192:
                if batch > 1:
                    batch //= 2
                elif ctx > new:
                    ctx //= 2
                else:
                    new //= 2
        else:
            new = min(new, max(1, 8192 // batch))
        case = {"kind": kind, "heads": heads, "batch": batch, "new_lo": rng.randint(0, new), "new_hi": new, "ctx": ctx, "page": page,
                "pad": rng.choice([0, 0, rng.randint(1, 63)])}
        if kind == "prompt":
            window = rng.choice([0, 0, _log(rng, 1, 8192)])
            case.update(window=window, sinks=rng.choice([0, 4, 5, 130]) if window else 0)
        return case
    op = rng.choice(["fork", "compact", "copy", "turn"])
    seqs, page = _log(rng, 2, 64), rng.choice([16, 32])
    layers = 1 if op == "turn" else _log(rng, 1, 32)
    pages = _log(rng, 8 * seqs, 24576 if op == "turn" else max(8 * seqs, 4096 * 16 * 16 // page // layers))
    hi = page * (pages * 6 // 10 // seqs) - rng.randint(0, page - 1)
    case = {"kind": "pages", "op": op, "heads": heads if heads != "mha" else "8b", "layers": layers, "page": page, "seqs": seqs,
            "pages": pages, "lo": rng.randint(0, hi), "hi": hi,
            "n": rng.randint(1, pages // 4) if op == "copy" else rng.randint(1, seqs - 1) if op == "fork" else seqs}
    if op == "turn":
        case.update(window=_log(rng, 1, 8192), sinks=rng.choice([0, 4, 64]))
    return case


# ------------------------------------------------------------------ inputs --

def _spread(lo, hi, n):
    """n whole numbers evenly spread over [lo, hi], largest last; hi alone for one."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape, scale=1.0):
    return (scale * torch.randn(shape, generator=g, device="cuda", dtype=torch.float16)).view(torch.int16)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _kept(T, page, window, sinks):
    """Which pages of a sequence of T tokens hold a token that its last token sees."""
    n = (T + page - 1) // page
    if not window:
        return [True] * n
    return [p * page < sinks or (p + 1) * page > T - window for p in range(n)]


def _table(g, lens, page, spare, window=0, sinks=0, width=0):
    """A page table (-1: no page) over a pool of pages in random order, and the pool's size."""
    kept = [_kept(T, page, window, sinks) for T in lens]
    width = max([width, 1] + [len(k) for k in kept])
    mask = torch.tensor([k + [False] * (width - len(k)) for k in kept])
    used = int(mask.sum())
    pages = max(1, used + spare)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    table[mask.cuda()] = torch.randperm(pages, generator=g, device="cuda")[:used].to(torch.int32)
    return table, pages


def prepare(case, seed):
    g = _generator(seed)
    if case["kind"] == "pages":
        return _prepare_pages(case, g)
    Hq, Hkv = HEADS[case["heads"]]
    P = case["page"]
    s = {"case": case, "Hq": Hq, "Hkv": Hkv, "scale": 1.0 / math.sqrt(D)}
    if case["kind"] == "window":
        lens = _spread(case["lo"], case["hi"], case["batch"])
        table, pages = _table(g, lens, P, 3, case["window"], case["sinks"])
        rows = case["batch"]
    else:
        new = _spread(case["new_lo"], case["new_hi"], case["batch"])
        lens = [n + c for n, c in zip(new, _spread(case["ctx"] // 2, case["ctx"], case["batch"]))]
        table, pages = _table(g, lens, P, 3)
        starts = [sum(new[:b]) for b in range(len(new) + 1)]
        rows = starts[-1] + case["pad"]
        s.update(starts=_ints(starts), new_max=max(new))
    s.update(table=table, lens=_ints(lens), len_max=max(lens), rows=rows)
    s["k"], s["v"] = _normal(g, pages, Hkv, P, D), _normal(g, pages, Hkv, P, D)
    if case["kind"] == "append":
        s["qkv"] = _normal(g, rows, (Hq + 2 * Hkv) * D)
        s["q_out"] = torch.zeros((rows, Hq * D), dtype=torch.int16, device="cuda")
    else:
        s["q"] = _normal(g, rows, Hq * D, scale=2.5)
        s["out"] = torch.zeros((rows, Hq * D), dtype=torch.int16, device="cuda")
    if own:   # what a program makes once: the cache's description and the call's workspace
        from paper_2412_15803_gb300 import wq4
        s["cache"] = wq4.kv_cache_desc(s["k"], s["v"], table, P)
        n = 0
        if case["kind"] == "window":
            n = wq4.wq4_paged_attention_workspace_bytes(rows, Hq, Hkv, D)
        elif case["kind"] == "prompt":
            n = wq4.wq4_prompt_attention_workspace_bytes(case["batch"], rows, Hq, Hkv, D)
        s["ws"] = torch.zeros(n, dtype=torch.uint8, device="cuda")
    return s


def _prepare_pages(case, g):
    """A pool of `pages` pages in every layer and the sequences that hold some of them: one integer array
    with the table, the lengths and the pages' reference counts, and the program's copy of it."""
    Hkv, P, S, N = HEADS[case["heads"]][1], case["page"], case["seqs"], case["pages"]
    s = {"case": case, "P": P, "S": S, "N": N}
    lens = _spread(case["lo"], case["hi"], S)
    if case["op"] == "fork":       # the longest sequence is the parent, the others are replaced
        s["parents"], s["children"] = _ints([S - 1] * case["n"]), _ints(list(range(case["n"])))
    if case["op"] == "turn":
        step = [1 + 7 * i % 19 for i in range(S)]
        s["seqs"], s["new_lens"] = _ints(list(range(S))), _ints([T + d for T, d in zip(lens, step)])
        width = (max(lens) + 20 + P - 1) // P
    else:
        width = (max(lens) + P - 1) // P
    if case["op"] == "copy":
        pick = torch.randperm(N, generator=g, device="cuda")[:2 * case["n"]].to(torch.int32)
        s["src"], s["dst"] = pick[:case["n"]].contiguous(), pick[case["n"]:].contiguous()
    need = sum((T + P - 1) // P for T in lens)
    table, _ = _table(g, lens, P, N - need, width=width)
    W = s["W"] = table.shape[1]
    book = torch.zeros(S * W + S + N, dtype=torch.int32, device="cuda")
    book[:S * W] = table.view(-1)
    book[S * W:S * W + S] = _ints(lens)
    book[S * W + S:] = torch.bincount(table[table >= 0].long(), minlength=N)
    s["saved"], s["book"] = book, book.clone()
    s["table"], s["lens"], s["refs"] = s["book"][:S * W].view(S, W), s["book"][S * W:S * W + S], s["book"][S * W + S:]
    s["kv"] = _normal(g, case["layers"], 2, N, Hkv, P, D)
    if own:
        from paper_2412_15803_gb300 import wq4
        s["layers"] = [wq4.kv_cache_desc(kv[0], kv[1], s["table"], P) for kv in s["kv"]]
        s["ws"] = torch.zeros(wq4.wq4_kv_pool_workspace_bytes(N, S), dtype=torch.uint8, device="cuda")
        s["pool"] = wq4.kv_pool_desc(s["layers"], s["table"], s["lens"], s["refs"], s["ws"])
    return s


# --------------------------------------------------------------- the calls --

def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own(s, kind)
    if kind == "window":
        return _plain_window(s)
    if kind == "prompt":
        return _plain_prompt(s)
    if kind == "append":
        return _plain_append(s)
    return _plain_pages(s)


def _own(s, kind):
    from paper_2412_15803_gb300 import wq4
    case = s["case"]
    if kind == "window":
        wq4.wq4_window_attention(s["cache"], s["q"], s["Hq"] * D, s["lens"], s["out"], s["Hq"] * D, s["rows"], s["Hq"], s["scale"],
                                 case["window"], case["sinks"], s["ws"], s["ws"].numel())
        return s["out"].view(torch.float16)
    if kind == "prompt":
        wq4.wq4_prompt_attention(s["cache"], s["q"], s["Hq"] * D, s["starts"], s["lens"], s["out"], s["Hq"] * D, case["batch"],
                                 s["rows"], s["Hq"], s["scale"], case["window"], case["sinks"], s["ws"], s["ws"].numel())
        return s["out"].view(torch.float16)
    if kind == "append":
        wq4.wq4_prompt_append(s["cache"], s["qkv"], (s["Hq"] + 2 * s["Hkv"]) * D, s["q_out"], s["Hq"] * D, s["starts"], s["lens"],
                              case["batch"], s["rows"], s["Hq"], THETA)
        return {n: s[n].view(torch.float16) for n in ("q_out", "k", "v")}
    s["book"].copy_(s["saved"])
    if case["op"] == "fork":
        wq4.wq4_kv_fork(s["pool"], s["parents"], s["children"], case["n"])
    elif case["op"] == "compact":
        wq4.wq4_kv_compact(s["pool"])
    elif case["op"] == "copy":
        wq4.wq4_kv_copy_pages(s["pool"], s["src"], s["dst"], case["n"])
    else:
        wq4.wq4_kv_trim(s["pool"], s["seqs"], case["n"], case["window"], case["sinks"])
        wq4.wq4_kv_reserve(s["pool"], s["seqs"], s["new_lens"], case["n"])
    return _pool_state(s)


def _pool_state(s):
    return {n: s[n] for n in ("table", "lens", "refs") + (("kv",) if s["case"]["op"] != "turn" else ())}


# --------------------------------------------------------- the plain forms --

def _softmax_values(scores, seen, values, pattern):
    """softmax over the last axis of the scores that are seen, times the values; zero where nothing is seen."""
    scores = scores.masked_fill(~seen, -math.inf)
    m = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(m == -math.inf, torch.zeros_like(m), m))
    z = e.sum(-1, keepdim=True)
    return torch.einsum(pattern, e / torch.where(z == 0, torch.ones_like(z), z), values)


def _rows_of(s, cache, tok):
    """Cached rows [batch][tokens][kv heads][D] of the tokens tok [batch][tokens], in 32 bits."""
    P = s["case"]["page"]
    b = torch.arange(tok.shape[0], device="cuda")[:, None]
    page = s["table"][b, (tok // P).clamp(0, s["table"].shape[1] - 1)].clamp(min=0).long()
    return cache.view(torch.float16)[page, :, tok % P].float()


def _plain_window(s):
    case, B, Hq, Hkv = s["case"], s["rows"], s["Hq"], s["Hkv"]
    T = s["lens"].long()[:, None]
    sinks = T.clamp(max=case["sinks"])
    first = (T - case["window"]).clamp(min=0).maximum(sinks)      # the window, less what the sinks have already
    i = torch.arange(min(s["len_max"], case["window"] + case["sinks"]), device="cuda")[None]
    tok = torch.where(i < sinks, i, i - sinks + first)
    seen = tok < T
    tok = tok.minimum((T - 1).clamp(min=0))
    keys = _rows_of(s, s["k"], tok)
    values = _rows_of(s, s["v"], tok).masked_fill(~seen[:, :, None, None], 0)
    q = s["q"].view(torch.float16).view(B, Hkv, Hq // Hkv, D).float()
    scores = torch.einsum("bhgd,bthd->bhgt", q, keys) * s["scale"]
    o = _softmax_values(scores, seen[:, None, None], values, "bhgt,bthd->bhgd")
    s["out"].copy_(o.reshape(B, Hq * D).half().view(torch.int16))
    return s["out"].view(torch.float16)


def _new_rows(s):
    """Of every sequence's new tokens, padded to the most: the rows, the positions and which are real [batch][new]."""
    starts, T = s["starts"].long(), s["lens"].long()
    i = torch.arange(s["new_max"], device="cuda")[None]
    n = (starts[1:] - starts[:-1])[:, None]
    return (starts[:-1, None] + i).clamp(max=s["rows"] - 1), T[:, None] - n + i, i < n


def _plain_prompt(s):
    case, Hq, Hkv = s["case"], s["Hq"], s["Hkv"]
    rows, pos, real = _new_rows(s)
    t = torch.arange(s["len_max"], device="cuda")
    tok = t[None].expand(rows.shape[0], -1)
    inside = tok < s["lens"].long()[:, None]
    keys = _rows_of(s, s["k"], tok)
    values = _rows_of(s, s["v"], tok).masked_fill(~inside[:, :, None, None], 0)
    seen = t[None, None] <= pos[:, :, None]
    if case["window"]:
        seen &= (t > pos[:, :, None] - case["window"]) | (t < case["sinks"])
    q = s["q"].view(torch.float16)[rows].view(*rows.shape, Hkv, Hq // Hkv, D).float()
    scores = torch.einsum("bnhgd,bthd->bhgnt", q, keys).mul_(s["scale"])
    o = _softmax_values(scores, seen[:, None, None], values, "bhgnt,bthd->bnhgd")
    s["out"][rows[real]] = o[real].view(-1, Hq * D).half().view(torch.int16)
    return s["out"].view(torch.float16)


def _plain_append(s):
    case, Hq, Hkv = s["case"], s["Hq"], s["Hkv"]
    rows, pos, real = _new_rows(s)
    rows, b, pos = rows[real], real.nonzero()[:, 0], pos[real]
    x = s["qkv"].view(torch.float16)[rows].view(-1, Hq + 2 * Hkv, D)
    angle = pos.double()[:, None] * torch.pow(THETA, -torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
    c, n = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    u, w = x[:, :Hq + Hkv, 0::2].float(), x[:, :Hq + Hkv, 1::2].float()
    turned = torch.stack([u * c - w * n, u * n + w * c], -1).view(-1, Hq + Hkv, D).half().view(torch.int16)
    s["q_out"][rows] = turned[:, :Hq].reshape(-1, Hq * D)
    page = s["table"][b, pos // case["page"]].long()
    s["k"][page, :, pos % case["page"]] = turned[:, Hq:]
    s["v"][page, :, pos % case["page"]] = x[:, Hq + Hkv:].view(torch.int16)
    return {n: s[n].view(torch.float16) for n in ("q_out", "k", "v")}


def _plain_pages(s):
    """The bookkeeping by sorting and counting; free pages are taken from the lowest up."""
    case, P, N = s["case"], s["P"], s["N"]
    s["book"].copy_(s["saved"])
    table, lens, refs, kv = s["table"], s["lens"], s["refs"], s["kv"]
    count = lambda entries: torch.bincount((entries + 1).reshape(-1).long(), minlength=N + 1)[1:].to(torch.int32)   # noqa: E731
    if case["op"] == "fork":
        par, child = s["parents"].long(), s["children"].long()
        table[child] = -1
        free = (count(table) == 0).nonzero()[:, 0]
        table[child], lens[child] = table[par], lens[par]
        part = (lens[child] % P != 0).nonzero()[:, 0]         # children whose last page is not full
        last = lens[child[part]].long() // P
        src, dst = table[child[part], last].long(), free[:part.shape[0]]
        table[child[part], last] = dst.to(torch.int32)
        held = torch.arange(P, device="cuda") < (lens[child[part]].long() % P)[:, None]     # rows that hold a token
        kv[:, :, dst] = torch.where(held[None, None, :, None, :, None], kv[:, :, src], kv[:, :, dst])
        refs.copy_(count(table))
    elif case["op"] == "compact":
        live = refs > 0
        at = torch.arange(N, device="cuda")
        front = at < live.sum()
        src, dst = (live & ~front).nonzero()[:, 0], (~live & front).nonzero()[:, 0]
        to = at.to(torch.int32)
        to[src] = dst.to(torch.int32)
        table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], table))
        refs[dst] = refs[src]
        refs[src] = 0
        kv[:, :, dst] = kv[:, :, src]
    elif case["op"] == "copy":
        kv[:, :, s["dst"].long()] = kv[:, :, s["src"].long()]
    else:
        at = torch.arange(s["W"], device="cuda")[None]
        T = lens.long()[:, None]
        keep = (at * P < case["sinks"]) | ((at + 1) * P > T + 1 - case["window"])       # the next token is at T
        table.masked_fill_(~keep, -1)
        refs.copy_(count(table))
        new = (at >= (T + P - 1) // P) & (at < (s["new_lens"].long()[:, None] + P - 1) // P)
        free = (refs == 0).nonzero()[:, 0].to(torch.int32)
        order = (new.view(-1).long().cumsum(0) - 1).clamp(min=0)
        table.copy_(torch.where(new, free[order].view_as(table), table))
        lens.copy_(s["new_lens"])
        refs.copy_(count(table))
    return _pool_state(s)


# --------------------------------------------------------------- 64 bits --

def exact(case, seed):
    """The definitions in 64 bits: a sequence at a time, each token's keys and values looked up one by one."""
    if case["kind"] == "pages":
        return None            # whole numbers and copies
    s = prepare(case, seed)
    P, Hq, Hkv, lens = case["page"], s["Hq"], s["Hkv"], s["lens"].tolist()
    G = Hq // Hkv
    pairs = sum(n * T for n, T in zip([1] * len(lens) if case["kind"] == "window" else _spread(case["new_lo"], case["new_hi"], len(lens)), lens))
    if pairs * Hq * D * 4 > 4e12:
        return None
    at = [0] + [b + 1 for b in range(len(lens))] if case["kind"] == "window" else s["starts"].tolist()

    def places(b, tokens):
        return s["table"][b].long()[tokens // P], tokens % P

    if case["kind"] == "append":
        x = s["qkv"].view(torch.float16).double()
        q, k, v = (s[n].view(torch.float16).double() for n in ("q_out", "k", "v"))
        w = torch.exp(-math.log(THETA) * torch.arange(D // 2, device="cuda", dtype=torch.float64) / (D // 2))
        for b, T in enumerate(lens):
            n = at[b + 1] - at[b]
            if not n:
                continue
            rows, tokens = x[at[b]:at[b + 1]].view(n, -1, D), torch.arange(T - n, T, device="cuda")
            turn = torch.polar(torch.ones(n, D // 2, device="cuda", dtype=torch.float64), tokens[:, None] * w)
            z = torch.view_as_real(torch.view_as_complex(rows[:, :Hq + Hkv].reshape(n, Hq + Hkv, D // 2, 2).contiguous()) * turn[:, None])
            z = z.reshape(n, Hq + Hkv, D)
            q[at[b]:at[b + 1]] = z[:, :Hq].reshape(n, -1)
            page, row = places(b, tokens)
            k[page, :, row], v[page, :, row] = z[:, Hq:], rows[:, Hq + Hkv:]
        return {"q_out": q, "k": k, "v": v}

    out = torch.zeros((s["rows"], Hq, D), dtype=torch.float64, device="cuda")
    q = s["q"].view(torch.float16).double().view(-1, Hq, D)
    for b, T in enumerate(lens):
        n = at[b + 1] - at[b]
        if not n or not T:
            continue
        tokens = torch.arange(T, device="cuda")
        pos = tokens[T - n:] if n <= T else torch.arange(T - n, T, device="cuda")
        seen = tokens <= pos[:, None]
        if case["window"]:
            seen = seen & ((pos[:, None] - tokens < case["window"]) | (tokens < case["sinks"]))
        used = seen.any(0).nonzero()[:, 0]
        page, row = places(b, used)
        bias = torch.zeros(n, used.shape[0], dtype=torch.float64, device="cuda").masked_fill_(~seen[:, used], -math.inf)
        for j in range(Hq):
            key, value = (s[c].view(torch.float16)[page, j // G, row].double() for c in ("k", "v"))
            score = q[at[b]:at[b + 1], j] @ key.T / math.sqrt(D) + bias
            weight = torch.exp(score - torch.logsumexp(score, 1, keepdim=True))
            out[at[b]:at[b + 1], j] = torch.nan_to_num(weight) @ value
    return out.view(s["rows"], Hq * D)


# -------------------------------------------------------------------- work --

def _seen(pos, window, sinks):
    """Tokens that the token at pos sees."""
    if pos < 0:
        return 0
    return pos + 1 if not window else pos + 1 - max(0, pos + 1 - window - sinks if sinks < pos + 1 - window else 0)


def work(case):
    if case["kind"] == "pages":
        Hkv, P, S = HEADS[case["heads"]][1], case["page"], case["seqs"]
        lens = _spread(case["lo"], case["hi"], S)
        page = 2 * case["layers"] * Hkv * P * D * 2
        held = sum((T + P - 1) // P for T in lens)
        if case["op"] == "fork":       # the parent's table row read and the children's written, the rows of its last page copied
            row = 4 * ((lens[-1] + P - 1) // P)
            return {"bytes": 2 * case["n"] * page * (lens[-1] % P) // P + row * (case["n"] + 1), "flops": 0}
        if case["op"] == "compact":    # on average; the reference counts read, the table read and written
            moved = held * (case["pages"] - held) // case["pages"]
            return {"bytes": 2 * moved * page + 4 * case["pages"] + 8 * held, "flops": 0}
        if case["op"] == "copy":
            return {"bytes": 2 * case["n"] * page, "flops": 0}
        return {"bytes": 8 * held, "flops": 0}
    Hq, Hkv = HEADS[case["heads"]]
    if case["kind"] == "append":
        rows = sum(_spread(case["new_lo"], case["new_hi"], case["batch"]))
        return {"bytes": max(1, rows) * (Hq + 2 * Hkv) * D * 4, "flops": rows * (Hq + Hkv) * D * 3}
    if case["kind"] == "window":
        seen = [_seen(T - 1, case["window"], case["sinks"]) for T in _spread(case["lo"], case["hi"], case["batch"])]
        return {"bytes": sum(seen) * Hkv * D * 4 + case["batch"] * Hq * D * 4, "flops": 4 * D * Hq * sum(seen)}
    new = _spread(case["new_lo"], case["new_hi"], case["batch"])
    lens = [n + c for n, c in zip(new, _spread(case["ctx"] // 2, case["ctx"], case["batch"]))]
    seen, read = 0, 0
    for n, T in zip(new, lens):
        seen += sum(_seen(pos, case["window"], case["sinks"]) for pos in range(T - n, T))
        read += min(T, case["window"] + n - 1 + case["sinks"]) if case["window"] and n else T if n else 0
    return {"bytes": max(1, sum(new)) * Hq * D * 4 + read * Hkv * D * 4, "flops": 4 * D * Hq * seen}
