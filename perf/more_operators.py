"""Performance cases of what long contexts add to the attention block: a cache held in 4 bits, windows with first
tokens that stay visible, and the book of a cache's pages.

Operators (``case["op"]``):
  rope4  rotary positions of Q and K (with ``tp`` the norm's Phases B+C in the same pass), K and V written into a
         4-bit cache; the written rows read back as bf16
  attn   attention of new tokens over a paged cache: dtype "fp4" is the 4-bit cache; with a window each token also
         sees the sequence's first ``sinks`` tokens
  pages  what a serving loop does with pages: "fork" (branches dropped, new ones taken from their parents, the
         pages that are only partly full copied in every layer), "admit" (requests leave, others come: pages and
         slots for their tokens), "compact" (pages in use moved to the front of the pools)

The 4-bit format: E2M1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), two to a byte, the lower half first; 32 elements
of a head share an exponent byte E, 2^(E - 127).

Widths are one rank's slices of the library's workloads, 1 to 32768 tokens.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
DEV = "cuda"
FP8 = torch.float8_e4m3fn
BASE = 1e6  # rotary base

# The most that a drawn case may cost: the compaction's bytes, the 8192-token prompt's flops.
MOST_BYTES = 270e6
MOST_FLOPS = 275e9
MOST_SCORES = 16 * 8192 * 8192  # (head, query, key) triples of a padded batch


def _rope4(name, T, heads, kv_heads, D, tp=0, rot=0, interleaved=False, page=16, strided=False):
    """rot 0: the whole head; tp 0: rows come normalised."""
    return {"name": name, "op": "rope4", "T": T, "heads": heads, "kv_heads": kv_heads, "D": D, "tp": tp,
            "rot": rot or D, "interleaved": interleaved, "page": page, "strided": strided}


def _attn(name, B, q, kv, heads, kv_heads, D, dtype="fp4", page=16, window=0, sinks=0, ragged=False, lse=False):
    """q new tokens in each of B sequences, kv tokens in its cache with them; ragged: at most so many."""
    return {"name": name, "op": "attn", "B": B, "q": q, "kv": kv, "heads": heads, "kv_heads": kv_heads, "D": D,
            "dtype": dtype, "page": page, "window": window, "sinks": sinks, "ragged": ragged, "lse": lse}


def _pages(name, kind, B, kv, kv_heads, D, layers=1, dtype="bf16", page=16, fan=1, pages=0, used=0.6):
    """fork: B parents of up to kv tokens, `fan` branches of each; admit: B of 4 B requests leave, as many with up to
    kv tokens come, in a pool of `pages`; compact: a pool of `pages`, of which `used` are in use by sequences of
    up to kv tokens."""
    return {"name": name, "op": "pages", "kind": kind, "B": B, "kv": kv, "kv_heads": kv_heads, "D": D, "layers": layers,
            "dtype": dtype, "page": page, "fan": fan, "pages": pages, "used": used}


def listed():
    return [
        # a decode step of 64 requests into the 4-bit cache: one call's latency
        _rope4("rope4_decode", 64, 8, 2, 128, tp=4),
        # prefill of one rank, norm included, V from a fused QKV buffer
        _rope4("rope4_prefill", 8192, 16, 4, 128, tp=2, page=64, strided=True),
        # a decode batch, contexts of all lengths
        _attn("attn4_decode", 64, 1, 4096, 8, 2, 128, ragged=True),
        # long contexts, what the 4-bit cache is for
        _attn("attn4_decode_long", 16, 1, 32768, 16, 2, 128, page=64, ragged=True),
        # one chunk of a chunked prefill behind a long prefix
        _attn("attn4_chunk", 1, 777, 12001, 16, 4, 128, page=64, lse=True),
        # a whole prompt, the most products
        _attn("attn4_prefill", 1, 8192, 8192, 16, 4, 128, page=64),
        # windowed layer in a decode batch of long contexts: the window and four first tokens
        _attn("sinks_decode", 32, 1, 32768, 16, 4, 128, dtype="bf16", window=4096, sinks=4, ragged=True),
        # prompts' chunks and single tokens in one batch, windowed layer of narrow heads, a system prompt kept
        _attn("sinks_mixed", 12, 512, 4096, 16, 2, 64, dtype="bf16", window=1024, sinks=64, ragged=True),
        # a whole prompt in a windowed layer over an FP8 cache
        _attn("sinks_prefill_fp8", 1, 8192, 8192, 16, 4, 128, dtype="fp8", page=64, window=2048, sinks=128),
        # four branches of each of 16 sequences, four layers
        _pages("pages_fork", "fork", 16, 4096, 4, 128, layers=4, page=64, fan=4),
        # a few requests leave, others come: the smallest call
        _pages("pages_admit", "admit", 8, 2048, 4, 128, pages=8192),
        # a fragmented pool of four FP8 layers moved together, the most bytes
        _pages("pages_compact", "compact", 64, 1024, 8, 128, layers=4, dtype="fp8", pages=4096),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _over(case):
    w = work(case)
    return (w["bytes"] > MOST_BYTES or w["flops"] > MOST_FLOPS or
            case["op"] == "attn" and case["B"] * case["q"] * case["heads"] * case["kv"] > MOST_SCORES)


def draw(rng):
    op = rng.choice(["rope4", "attn4", "attn4", "sinks", "pages"])
    page = rng.choice([16, 32, 64, 128])
    if op == "rope4":
        D, kv_heads = rng.choice([32, 64, 128, 128, 256]), rng.choice([1, 2, 4])
        case = _rope4("", _log_int(rng, 1, 16384), kv_heads * rng.choice([1, 2, 3, 4, 5]), kv_heads, D,
                      rng.choice([0, 1, 2, 4, 8]), rng.choice([D, D, D // 2]), rng.random() < 0.3, page,
                      rng.random() < 0.5)
    elif op == "pages":
        kind = rng.choice(["fork", "admit", "compact"])
        layers, kv_heads = rng.randint(1, 6), rng.choice([1, 2, 4, 8])
        D, dtype, page = rng.choice([64, 128]), rng.choice(["bf16", "fp8"]), rng.choice([16, 32, 64])
        if kind == "fork":
            case = _pages("", kind, _log_int(rng, 1, 64), _log_int(rng, 16, 4096), kv_heads, D, layers, dtype, page,
                          rng.randint(1, 8))
        elif kind == "admit":
            B, kv = _log_int(rng, 1, 200), _log_int(rng, 1, 4096)
            case = _pages("", kind, B, kv, kv_heads, D, 1, dtype, page,
                          pages=5 * B * (-(-kv // page)) + _log_int(rng, 16, 32768))
        else:
            case = _pages("", kind, _log_int(rng, 4, 128), _log_int(rng, 16, 2048), kv_heads, D, layers, dtype, page,
                          pages=_log_int(rng, 64, 8192), used=rng.choice([0.3, 0.5, 0.8, 0.95]))
    else:
        dtype = "fp4" if op == "attn4" else rng.choice(["bf16", "fp8", "fp4"])
        D = rng.choice([64, 128, 128, 256, 96])
        kv_heads = rng.randint(1, max(1, min(8, 1024 // D)))
        B, kv = _log_int(rng, 1, 128), _log_int(rng, 16, 32768)
        q = 1 if rng.random() < 0.5 else _log_int(rng, 2, min(kv, 4096))
        window = _log_int(rng, 16, 4096) if op == "sinks" else 0
        case = _attn("", B, q, kv, kv_heads * rng.choice([1, 2, 3, 4, 5, 8]), kv_heads, D, dtype, page, window,
                     _log_int(rng, 1, 300) if window else 0, rng.random() < 0.7, rng.random() < 0.5)
    del case["name"]
    while _over(case):
        shorter = rng.uniform(0.3, 0.9)
        if op == "rope4":
            case["T"] = max(1, int(case["T"] * shorter))
        elif op == "pages":
            if case["kind"] == "compact":
                case["pages"] = max(16, int(case["pages"] * shorter))
            else:
                case["B"] = max(1, int(case["B"] * shorter))
        elif case["B"] > 1:
            case["B"] = max(1, int(case["B"] * shorter))
        elif case["q"] > 64:
            case["q"] = max(1, int(case["q"] * shorter))
        else:
            case["kv"] = max(case["q"], int(case["kv"] * shorter))
    return case


def _spread(i, step):
    """Of (0, 1], evenly spread; the first is 1."""
    return (1.0 - step * i) % 1.0 or 1.0


def _lengths(case):
    """New tokens and cached tokens (the new ones among them) of each sequence."""
    if not case["ragged"]:
        return [case["q"]] * case["B"], [case["kv"]] * case["B"]
    # short chunks are the most common; the first sequence is the longest
    q = [max(1, round(case["q"] * _spread(i, 0.6180339887) ** 2)) for i in range(case["B"])]
    return q, [max(n, round(case["kv"] * _spread(i, 0.7548776662))) for i, n in enumerate(q)]


def _tokens(case):
    """Tokens of the sequences of a "pages" case."""
    return [max(1, round(case["kv"] * _spread(i, 0.7548776662))) for i in range(case["B"])]


def _in_use(case):
    """Pages of a fragmented pool that are in use, at places spread over it, and the tokens of its sequences."""
    places = [i for i in range(case["pages"]) if (0.6180339887 * i) % 1.0 < case["used"]]
    tokens, left = [], len(places)
    while left:
        n = min(_tokens(case)[len(tokens) % case["B"]], left * case["page"])
        tokens.append(n)
        left -= -(-n // case["page"])
    return places, tokens


def _page_bytes(case):
    return 2 * case["kv_heads"] * case["page"] * case["D"] * (2 if case["dtype"] == "bf16" else 1)


def _row_bytes(D, dtype):
    """Bytes of a head's row in the cache."""
    return 2 * D if dtype == "bf16" else D if dtype == "fp8" else D // 2 + D // 32


def work(case):
    if case["op"] == "rope4":
        T, D = case["T"], case["D"]
        nq, nk = case["heads"] * D, case["kv_heads"] * D
        norm = 4 * (nq + nk) + 2 * 4 * case["tp"] * T if case["tp"] else 0
        cached = 2 * case["kv_heads"] * _row_bytes(D, "fp4")
        # rows in, Q out, the cache written, read back, its rows out; angles, positions, slots
        return {"bytes": T * (4 * nq + 4 * nk + 2 * cached + 4 * nk + 4 * case["rot"] + 20) + norm,
                "flops": 3 * T * (nq + 2 * nk)}
    if case["op"] == "attn":
        D, w, s = case["D"], case["window"], case["sinks"]
        pairs = seen = 0
        for n, m in zip(*_lengths(case)):
            if w:
                ends = range(m - n + 1, m + 1)
                pairs += sum(min(w, e) + min(s, max(0, e - w)) for e in ends)
                seen += min(m, n + w - 1) + min(s, max(0, m - n + 1 - w))
            else:
                pairs += n * (m - n) + n * (n + 1) // 2
                seen += m
        T = sum(_lengths(case)[0])
        return {"bytes": 4 * T * case["heads"] * D + 2 * seen * case["kv_heads"] * _row_bytes(D, case["dtype"])
                + (4 * T * case["heads"] if case["lse"] else 0) + 4 * (seen // case["page"]) + 8 * case["B"],
                "flops": 4 * D * case["heads"] * pairs}
    page = case["page"]
    if case["kind"] == "fork":
        tokens = _tokens(case)
        copies = case["fan"] * sum(n % page != 0 for n in tokens)
        entries = case["fan"] * sum(-(-n // page) for n in tokens)
        # the pages in and out; the branches' old and new entries, their pages' counts down and up
        return {"bytes": 2 * copies * case["layers"] * _page_bytes(case) + 24 * entries, "flops": 4 * entries}
    if case["kind"] == "admit":
        entries, T = sum(-(-n // page) for n in _tokens(case)), sum(_tokens(case))
        return {"bytes": 24 * entries + 12 * T + 16 * case["B"], "flops": 2 * T + 4 * entries}
    places, tokens = _in_use(case)
    moves = sum(i >= len(places) for i in places)
    return {"bytes": 2 * moves * case["layers"] * _page_bytes(case) + 8 * case["pages"] + 8 * len(places),
            "flops": 2 * case["pages"]}


# ------------------------------------------------------------------ inputs

def _normal(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _pool(g, pages, kv_heads, page, D, dtype, spread=1.0):
    x = _normal(g, pages, kv_heads, page, D)
    return x.to(torch.bfloat16) if dtype == "bf16" else x.mul_(spread).clamp_(-448.0, 448.0).to(FP8)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return {"rope4": _prepare_rope4, "attn": _prepare_attn, "pages": _prepare_pages}[case["op"]](case, g)


def _prepare_rope4(case, g):
    T, D, hq, hk, tp = case["T"], case["D"], case["heads"], case["kv_heads"], case["tp"]
    scale = torch.exp(0.5 * _normal(g, T, 1)) if tp else 1.0  # unnormalised rows: one lognormal scale a token
    x = [(_normal(g, T, h * D) * scale).to(torch.bfloat16) for h in (hq, hk)] + [_normal(g, T, hk * D).to(torch.bfloat16)]
    if case["strided"]:  # columns of one QKV buffer
        x = list(torch.cat(x, 1).split([hq * D, hk * D, hk * D], 1))
    page = case["page"]
    pages = -(-T // page) + 2
    first = 1000  # the chunk follows a prefix
    freq = BASE ** (-torch.arange(0, case["rot"], 2, device=DEV, dtype=torch.float64) / case["rot"])
    angle = torch.arange(first + T, device=DEV, dtype=torch.float64)[:, None] * freq
    where = torch.randperm(pages, device=DEV, generator=g)[: pages - 2]
    t = torch.arange(T, device=DEV)

    def codes(width):
        return torch.randint(0, 256, (pages, hk, page, width), device=DEV, generator=g, dtype=torch.uint8)

    def rows():
        return torch.empty(T, hk * D, device=DEV, dtype=torch.bfloat16)
    s = {"op": "rope4", "q": x[0], "k": x[1], "v": x[2], "D": D, "rot": case["rot"], "interleaved": case["interleaved"],
         "table": torch.stack([angle.cos(), angle.sin()], -1).float(), "pos": (t + first).int(),
         "slots": where[t // page] * page + t % page,
         "k_pool": codes(D // 2), "v_pool": codes(D // 2), "k_exp": codes(D // 32), "v_exp": codes(D // 32),
         "y": torch.empty(T, hq * D, device=DEV, dtype=torch.bfloat16), "k_rows": rows(), "v_rows": rows(), "tp": tp}
    if tp:
        s["gamma"] = [torch.rand(h * D, device=DEV, generator=g) + 0.5 for h in (hq, hk)]
        s["d_full"] = [h * D * tp for h in (hq, hk)]
        s["sums"] = []
        for row, h in zip(x, (hq, hk)):  # every rank's statistic; the other ranks' rows are like this one's
            own_sum = row.float().square().sum(1)
            like = 1 + 0.3 * math.sqrt(2.0 / (h * D)) * _normal(g, tp, T).clamp_(-3, 3)
            like[tp - 1] = 1
            s["sums"].append((own_sum * like).contiguous())
    return s


def _prepare_attn(case, g):
    D, hq, hk, page = case["D"], case["heads"], case["kv_heads"], case["page"]
    nq, nkv = _lengths(case)
    T, B, width = sum(nq), case["B"], -(-max(nkv) // page)
    counts = [-(-n // page) for n in nkv]
    pages = sum(counts) + 3
    order = torch.randperm(pages, device=DEV, generator=g).int()
    at = torch.arange(width, device=DEV)
    count = torch.tensor(counts, device=DEV)
    first = count.cumsum(0) - count
    table = torch.where(at < count[:, None], order[(first[:, None] + at).clamp_(max=pages - 1)], 0).int()
    s = {"op": "attn", "q": _normal(g, T, hq * D).to(torch.bfloat16), "D": D, "window": case["window"],
         "sinks": case["sinks"], "k_exp": None, "v_exp": None, "k_scale": None, "v_scale": None, "block_table": table,
         "q_start": torch.tensor([0] + [sum(nq[: i + 1]) for i in range(B)], device=DEV, dtype=torch.int32),
         "kv_len": torch.tensor(nkv, device=DEV, dtype=torch.int32), "max_q": max(nq), "max_kv": max(nkv),
         "scale": D ** -0.5, "out": torch.empty(T, hq * D, device=DEV, dtype=torch.bfloat16),
         "lse": torch.empty(T, hq, device=DEV) if case["lse"] else None}
    for name in "kv":
        if case["dtype"] == "fp4":  # codes and exponents as normal values have them: the largest of 32 is 4 or 6
            s[name + "_pool"], s[name + "_exp"] = _to_codes(_normal(g, pages, hk, page, D))
        else:
            s[name + "_pool"] = _pool(g, pages, hk, page, D, case["dtype"], 64.0)
            if case["dtype"] == "fp8":
                s[name + "_scale"] = (0.75 + 0.5 * torch.rand(hk, device=DEV, generator=g)) / 64.0
    return s


def _prepare_pages(case, g):
    page, kind = case["page"], case["kind"]
    s = {"op": "pages", "kind": kind, "page": page}
    if kind == "compact":
        places, tokens = _in_use(case)
        n_pages, free_rows = case["pages"], 0
        mine = torch.tensor(places, device=DEV)[torch.randperm(len(places), device=DEV, generator=g)].int()
    else:
        # parents, and branches that share their whole pages; or requests, of which the first B leave and come again
        tokens = _tokens(case) * (1 if kind == "fork" else 4)
        need = sum(-(-n // page) for n in tokens)
        free_rows = case["B"] * case["fan"] if kind == "fork" else 0
        n_pages = case["pages"] or need + free_rows + 7
        mine = torch.randperm(n_pages, device=DEV, generator=g).int()
    rows, width = len(tokens) + free_rows, -(-max(tokens) // page) + 1
    length = torch.tensor(tokens + [0] * free_rows, device=DEV, dtype=torch.int32)
    count = (length + page - 1) // page
    first = count.cumsum(0) - count
    at = torch.arange(width, device=DEV)
    held = at < count[:, None]
    table = torch.where(held, mine[(first[:, None] + at).clamp_(max=mine.numel() - 1)], 0).int()
    refs = torch.zeros(n_pages, device=DEV, dtype=torch.int32)
    refs.index_add_(0, table.flatten(), held.flatten().int())
    s.update(table=table, kv_len=length, refs=refs)
    if kind == "fork":
        s["parents"] = torch.arange(case["B"], device=DEV, dtype=torch.int32).repeat_interleave(case["fan"])
        s["rows"] = torch.arange(len(tokens), rows, device=DEV, dtype=torch.int32)
        s["src"], s["dst"], s["done"] = (torch.empty(free_rows, device=DEV, dtype=torch.int32) for _ in range(3))
    elif kind == "admit":
        s["rows"] = torch.randperm(case["B"], device=DEV, generator=g).int()
        s["counts"], s["T"] = length[s["rows"].long()].clone(), sum(tokens[: case["B"]])
        s["slots"] = torch.empty(s["T"], device=DEV, dtype=torch.int64)
        s["pos"] = torch.empty(s["T"], device=DEV, dtype=torch.int32)
        s["done"] = torch.empty(case["B"], device=DEV, dtype=torch.int32)
    else:
        s["new_table"], s["new_refs"] = table.clone(), torch.empty_like(refs)
        s["src"], s["dst"] = (torch.empty(n_pages // 2, device=DEV, dtype=torch.int32) for _ in range(2))
    if kind != "admit":
        s["pools"] = [[_pool(g, n_pages, case["kv_heads"], page, case["D"], case["dtype"], 64.0) for _ in range(2)]
                      for _ in range(case["layers"])]
    return s


# ------------------------------------------------------------------ the calls

def run(s):
    if own:
        return {"rope4": _own_rope4, "attn": _own_attn, "pages": _own_pages}[s["op"]](s)
    return {"rope4": _plain_rope4, "attn": _plain_attn, "pages": _plain_pages}[s["op"]](s)


def _call(s, make):
    """The calls with their arguments marshalled once, as a serving loop keeps them."""
    if "calls" not in s:
        s["calls"] = make()
    for call in s["calls"]:
        call()


def _cache(s):
    import paper_2608_09160_amd as qkn
    if s.get("k_exp") is not None:
        return qkn.KVCache4(s["k_pool"], s["v_pool"], s["k_exp"], s["v_exp"])
    return qkn.KVCache(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])


def _own_rope4(s):
    import paper_2608_09160_amd as qkn

    def make():
        def seg(i, x, y=None):
            more = {"w": s["gamma"][i], "partials": s["sums"][i], "d_full": s["d_full"][i]} if s["tp"] else {}
            return qkn.RopeSeg(x=x, y=y, **more)
        cache = _cache(s)
        return [qkn.PreparedRopeCache(s["table"], s["pos"], s["D"], q=seg(0, s["q"], s["y"]), k=seg(1, s["k"]), v=s["v"],
                                      cache=cache, slots=s["slots"], interleaved=s["interleaved"], eps=EPS),
                qkn.PreparedCache4Load(cache, s["slots"], s["k_rows"], s["v_rows"])]
    _call(s, make)
    return {"q": s["y"], "k": s["k_rows"], "v": s["v_rows"]}


def _own_attn(s):
    import paper_2608_09160_amd as qkn
    _call(s, lambda: [qkn.PreparedAttn(
        s["q"], _cache(s), s["block_table"], s["q_start"], s["kv_len"], max_q=s["max_q"], max_kv=s["max_kv"],
        scale=s["scale"], window=s["window"], sinks=s["sinks"], out=s["out"], lse=s["lse"])])
    return {"out": s["out"], "lse": s["lse"]}


def _own_pages(s):
    import paper_2608_09160_amd as qkn

    def make():
        book = qkn.PageBook(s["refs"], s["table"], s["kv_len"], s["page"])
        caches = [qkn.KVCache(k, v) for k, v in s.get("pools", [])]
        if s["kind"] == "fork":
            return [qkn.PreparedPagesFree(book, s["rows"]),
                    qkn.PreparedPagesFork(book, s["parents"], s["rows"], s["src"], s["dst"], s["done"]),
                    qkn.PreparedPagesCopy(caches, s["src"], s["dst"])]
        if s["kind"] == "admit":
            return [qkn.PreparedPagesFree(book, s["rows"]),
                    qkn.PreparedPagesGrow(book, s["counts"], s["rows"], s["slots"], s["pos"], s["done"])]
        new = qkn.PageBook(s["new_refs"], s["new_table"], s["kv_len"], s["page"])
        return [qkn.PreparedPagesCompact(book, s["src"], s["dst"], out=new),
                qkn.PreparedPagesCopy(caches, s["src"], s["dst"])]
    _call(s, make)
    return _answer(s)


def _answer(s):
    if s["kind"] == "fork":
        return {"table": s["table"], "refs": s["refs"], "kv_len": s["kv_len"], "done": s["done"], "pools": s["pools"]}
    if s["kind"] == "admit":
        return {"table": s["table"], "refs": s["refs"], "kv_len": s["kv_len"], "done": s["done"], "slots": s["slots"],
                "pos": s["pos"]}
    return {"table": s["new_table"], "refs": s["new_refs"], "src": s["src"], "dst": s["dst"], "pools": s["pools"]}


# ------------------------------------------------------------------ plain forms, in 32 bits

_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _to_codes(x):
    """Codes [.., D / 2] and exponents [.., D / 32] of fp32 rows [.., D]: the exponent is the least with which the
    largest of 32 values is below 7, halfway to the value behind the last one; codes are the nearest, ties to even."""
    x = x.unflatten(-1, (-1, 32))
    most = x.abs().amax(-1)
    e = (((most.view(torch.int32) + 0x200000) >> 23) - 129).clamp(-125, 125)
    a = (x * ((127 - e) << 23).view(torch.float32)[..., None]).abs().clamp_(max=6.0)
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte()
            + (a >= 3.5).byte() + (a > 5.0).byte() + 8 * torch.signbit(x).byte()).flatten(-2)
    e = torch.where(most.isnan(), 255, e + 127)
    return code[..., 0::2] | code[..., 1::2] << 4, e.byte()


def _from_codes(codes, exps):
    """fp32 rows of codes and exponents."""
    values = torch.tensor(_VALUES + [-v for v in _VALUES], device=DEV)
    x = torch.stack([values[(codes & 15).int()], values[(codes >> 4).int()]], -1).flatten(-2)
    scale = (exps.int() << 23).view(torch.float32)
    return x * torch.where(exps == 255, math.nan, scale).repeat_interleave(32, -1)


def _rotate(x, cos, sin, rot, interleaved):
    """x [T, heads, D], cos and sin [T, 1, rot / 2]."""
    turn, rest = x[..., :rot], x[..., rot:]
    a, b = (turn[..., 0::2], turn[..., 1::2]) if interleaved else (turn[..., : rot // 2], turn[..., rot // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turn = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turn, rest], -1)


def _plain_rope4(s):
    D, slots = s["D"], s["slots"]
    cos, sin = (t[:, None] for t in s["table"][s["pos"].long()].unbind(-1))
    rows = []
    for i, x in enumerate((s["q"], s["k"])):
        x = x.float()
        if s["tp"]:
            total = s["sums"][i][0]
            for more in s["sums"][i][1:]:  # ascending ranks
                total = total + more
            x = x * s["gamma"][i] * torch.rsqrt(total * (1.0 / s["d_full"][i]) + EPS)[:, None]
        rows.append(_rotate(x.view(x.shape[0], -1, D), cos, sin, s["rot"], s["interleaved"]))
    s["y"].copy_(rows[0].flatten(1))
    page = s["k_pool"].shape[2]
    for name, x in (("k", rows[1]), ("v", s["v"].float().reshape(rows[1].shape))):
        pool, exps = s[name + "_pool"], s[name + "_exp"]
        pool[slots // page, :, slots % page], exps[slots // page, :, slots % page] = _to_codes(x)
        s[name + "_rows"].copy_(_from_codes(pool[slots // page, :, slots % page],
                                            exps[slots // page, :, slots % page]).flatten(1))
    return {"q": s["y"], "k": s["k_rows"], "v": s["v_rows"]}


def _gathered(s, name, n):
    """The first n rows of every sequence: [B, kv_heads, n, D] in 32 bits."""
    pool, exps, scale = s[name + "_pool"], s[name + "_exp"], s[name + "_scale"]
    page = pool.shape[2]
    j = torch.arange(n, device=DEV)
    at = s["block_table"][:, j // page].long()
    x = (pool.view(torch.uint8) if pool.dtype == FP8 else pool)[at, :, j % page]
    x = _from_codes(x, exps[at, :, j % page]) if exps is not None else x.view(pool.dtype).float()
    x = x.transpose(1, 2)
    return (x if scale is None else x * scale[:, None, None]).contiguous()


def _plain_attn(s):
    D, kv_heads = s["D"], s["k_pool"].shape[1]
    T, group = s["q"].shape[0], s["q"].shape[1] // (D * kv_heads)
    start, kv_len = s["q_start"].long(), s["kv_len"].long()
    B, nq, nkv = kv_len.numel(), s["max_q"], s["max_kv"]
    k, v = _gathered(s, "k", nkv), _gathered(s, "v", nkv)
    i, j = torch.arange(nq, device=DEV), torch.arange(nkv, device=DEV)
    rows = (start[:-1, None] + i).clamp_(max=T - 1)
    q = s["q"].float()[rows].view(B, nq, kv_heads, group, D).permute(0, 2, 1, 3, 4).reshape(B, kv_heads, nq * group, D)
    at = (kv_len - (start[1:] - start[:-1]))[:, None] + i  # [B, nq]: the cache position of each new token
    seen = (j <= at[..., None]) & (j < kv_len[:, None, None])
    if s["window"]:
        seen &= (j > at[..., None] - s["window"]) | (j < s["sinks"])
    seen = seen.repeat_interleave(group, 1)[:, None]
    x = (torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]).masked_fill_(~seen, -math.inf)
    most = x.amax(-1, keepdim=True).clamp_(min=-3e38)
    x = x.sub_(most).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v) / total.clamp(min=1e-38)
    seq = torch.searchsorted(start[1:], torch.arange(T, device=DEV), right=True)
    own_row = torch.arange(T, device=DEV) - start[seq]

    def by_token(z):
        return z.view(B, kv_heads, nq, group, -1).permute(0, 2, 1, 3, 4)[seq, own_row]
    s["out"].copy_(by_token(o).flatten(1))
    if s["lse"] is not None:
        s["lse"].copy_(by_token(most + total.log()).flatten(1))
    return {"out": s["out"], "lse": s["lse"]}


def _held(s, length):
    return torch.arange(s["table"].shape[1], device=DEV) < ((length + s["page"] - 1) // s["page"])[:, None]


def _free_first(refs):
    """All pages, the free ones first, each kind ascending."""
    return torch.sort(refs.ne(0).int(), stable=True).indices.int()


def _plain_free(s):
    rows = s["rows"].long()
    held = _held(s, s["kv_len"][rows])
    s["refs"].index_add_(0, s["table"][rows].flatten(), -held.flatten().int())
    s["kv_len"][rows] = 0


def _plain_copy(s, src, dst):
    for pools in s["pools"]:
        for pool in pools:
            bits = pool.view(torch.uint8) if pool.dtype == FP8 else pool
            bits[dst] = bits[src]


def _plain_pages(s):
    page, refs, table = s["page"], s["refs"], s["table"]
    if s["kind"] == "compact":
        n = s["src"].numel()
        used = refs.ne(0)
        src = torch.sort(used.flip(0).int(), stable=True, descending=True).indices[:n]
        src = (refs.numel() - 1 - src).int()  # the pages in use, the last first
        dst = _free_first(refs)[:n]
        k = torch.arange(n, device=DEV)
        moved = (k < used.sum()) & (k < (~used).sum()) & (src > dst)
        where = torch.arange(refs.numel() + 1, device=DEV, dtype=torch.int32)
        where[torch.where(moved, src, refs.numel()).long()] = dst
        s["new_table"].copy_(torch.where(_held(s, s["kv_len"]), where[table.long()], table))
        s["new_refs"].zero_()
        s["new_refs"].index_add_(0, where[:-1], refs)
        s["src"].copy_(torch.where(moved, src, -1))
        s["dst"].copy_(torch.where(moved, dst, -1))
        last = refs.numel() - 1  # never a move's end: copied onto itself
        _plain_copy(s, torch.where(moved, src, last).long(), torch.where(moved, dst, last).long())
        return _answer(s)
    _plain_free(s)
    rows = s["rows"].long()
    at = torch.arange(table.shape[1], device=DEV)
    if s["kind"] == "fork":
        parents = s["parents"].long()
        length = s["kv_len"][parents]
        part = length % page != 0
        new = _free_first(refs)[(part.cumsum(0) - 1).clamp(min=0)]
        last = (length // page)[:, None]
        mine = torch.where((at == last) & part[:, None], new[:, None], table[parents])
        held = _held(s, length)
        s["src"].copy_(torch.where(part, table[parents].gather(1, last.long())[:, 0], -1))
        s["dst"].copy_(torch.where(part, new, -1))
        keep = refs.numel() - 1
        _plain_copy(s, torch.where(part, s["src"], keep).long(), torch.where(part, s["dst"], keep).long())
        table[rows] = torch.where(held, mine, table[rows])
        refs.index_add_(0, mine.flatten(), held.flatten().int())
        s["kv_len"][rows] = length
        s["done"].copy_(length)
        return _answer(s)
    counts = s["counts"]
    held = _held(s, counts)
    rank = (held.flatten().cumsum(0) - 1).clamp_(min=0).view(held.shape)
    mine = _free_first(refs)[rank.clamp(max=refs.numel() - 1)]
    table[rows] = torch.where(held, mine, table[rows])
    refs.index_add_(0, mine.flatten(), held.flatten().int())
    s["kv_len"][rows] = counts
    s["done"].copy_(counts)
    i = torch.repeat_interleave(torch.arange(rows.numel(), device=DEV), counts, output_size=s["T"])
    pos = torch.arange(s["T"], device=DEV) - (counts.cumsum(0) - counts)[i]
    s["pos"].copy_(pos)
    s["slots"].copy_(table[rows[i], pos // page].long() * page + pos % page)
    return _answer(s)


# ------------------------------------------------------------------ the definitions, in 64 bits

def exact(case, seed):
    if case["op"] == "pages":  # nothing is computed in floating point
        return None
    s = prepare(case, seed)
    return _exact_rope4(case, s) if case["op"] == "rope4" else _exact_attn(case, s)


def _nearest4(x):
    """The values that the 4-bit format has for 64-bit rows [T, heads * D]."""
    blocks = x.reshape(-1, 32)
    part, power = torch.frexp(blocks.abs().amax(1, keepdim=True))  # the largest is part * 2^power, 0.5 <= part < 1
    power = (power - 3 + (part >= 0.875)).clamp(-125, 125)
    unit = torch.ldexp(blocks.abs(), -power)
    step = torch.where(unit < 2, 0.5, torch.where(unit < 4, 1.0, 2.0)).double()
    near = ((unit / step).round() * step).clamp(max=6)  # nearest, ties to even multiples: the even codes
    return torch.copysign(torch.ldexp(near, power), blocks).reshape(x.shape)


def _exact_rope4(case, s):
    T, D, rot = case["T"], case["D"], case["rot"]
    half = torch.arange(rot // 2, device=DEV)
    first, second = (2 * half, 2 * half + 1) if case["interleaved"] else (half, half + rot // 2)
    turn = torch.polar(torch.ones((), device=DEV, dtype=torch.float64),
                       s["pos"].double()[:, None] * BASE ** (-2.0 * half.double() / rot))[:, None]
    heads = []
    for i, x in enumerate((s["q"], s["k"])):
        x = x.double()
        if case["tp"]:
            mean = s["sums"][i].double().sum(0) / (x.shape[1] * case["tp"])
            x = x / (mean + EPS).sqrt()[:, None] * s["gamma"][i].double()
        x = x.reshape(T, -1, D)
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        heads.append(x.flatten(1))
    return {"q": heads[0], "k": _nearest4(heads[1]), "v": _nearest4(s["v"].double())}


def _exact_rows(s, name, pages, head, D):
    rows = s[name + "_pool"][pages, head]
    if s[name + "_exp"] is None:
        x = rows.double()
        return (x if s[name + "_scale"] is None else x * s[name + "_scale"][head].double()).reshape(-1, D)
    nibble = torch.stack([rows % 16, rows // 16], -1).reshape(-1, D // 32, 32).long()
    size, up = nibble % 2, nibble // 2 % 4  # mantissa and exponent; exponent 0 has no leading one
    value = torch.where(up == 0, 0.5 * size, torch.ldexp(1 + 0.5 * size, up - 1)).double() * (1 - 2 * (nibble // 8))
    return torch.ldexp(value, s[name + "_exp"][pages, head].reshape(-1, D // 32, 1).long() - 127).reshape(-1, D)


def _exact_attn(case, s):
    D, hk, page = case["D"], case["kv_heads"], case["page"]
    out = torch.zeros(s["q"].shape, device=DEV, dtype=torch.float64)
    lse = torch.zeros(s["q"].shape[0], case["heads"], device=DEV, dtype=torch.float64) if case["lse"] else None
    group, t = case["heads"] // hk, 0
    for b, (n, m) in enumerate(zip(*_lengths(case))):
        pages = s["block_table"][b, : -(-m // page)].long()
        ahead = torch.arange(m, device=DEV) - torch.arange(m - n, m, device=DEV)[:, None]  # key minus query
        allowed = ahead <= 0
        if case["window"]:
            near = ahead > -case["window"]
            near[:, : case["sinks"]] = True
            allowed &= near
        for h in range(case["heads"]):
            k, v = (_exact_rows(s, name, pages, h // group, D)[:m] for name in "kv")
            cols = slice(h * D, (h + 1) * D)
            score = s["q"][t:t + n, cols].double() @ k.t() / math.sqrt(D)
            norm = torch.logsumexp(score.masked_fill(~allowed, -math.inf), 1)
            out[t:t + n, cols] = torch.where(allowed, (score - norm[:, None]).exp(), 0.0) @ v
            if lse is not None:
                lse[t:t + n, h] = norm
        t += n
    return {"out": out, "lse": lse}
