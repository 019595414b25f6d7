"""Performance cases of the attention block's operators around the QK-Norm: adapters beside the projection,
rotary positions with the cache write, attention over the paged cache.

Operators (``case["op"]``):
  rope      rotary positions of Q and K, K and V written into the paged cache; with ``tp`` the norm's Phases
            B+C in the same pass
  attn      attention of new tokens (one each in decode batches) over the paged cache
  adapters  low-rank adapters of many requests added to the projection's output, with its Phase A statistic

Widths are one rank's slices of the library's workloads (Q 4096 to 8192, K 1024 in all, heads of 32 to 256),
1 to 32768 tokens, caches in bf16 and FP8-E4M3.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
DEV = "cuda"
FP8 = torch.float8_e4m3fn
BASE = 1e6  # rotary base

# The most that a drawn case may cost: the 32768-token rotary pass's bytes, the 8192-token prefill's flops.
MOST_BYTES = 330e6
MOST_FLOPS = 275e9
MOST_SCORES = 16 * 8192 * 8192  # (head, query, key) triples of a padded batch


def _rope(name, T, heads, kv_heads, D, tp=0, rot=0, interleaved=False, dtype="bf16", page=16, strided=False):
    """rot 0: the whole head; tp 0: rows come normalised."""
    return {"name": name, "op": "rope", "T": T, "heads": heads, "kv_heads": kv_heads, "D": D, "tp": tp,
            "rot": rot or D, "interleaved": interleaved, "dtype": dtype, "page": page, "strided": strided}


def _attn(name, B, q, kv, heads, kv_heads, D, dtype="bf16", page=16, window=0, ragged=False, lse=False):
    """q new tokens in each of B sequences, kv tokens in its cache with them; ragged: at most so many."""
    return {"name": name, "op": "attn", "B": B, "q": q, "kv": kv, "heads": heads, "kv_heads": kv_heads, "D": D,
            "dtype": dtype, "page": page, "window": window, "ragged": ragged, "lse": lse}


def _adapters(name, T, hidden, q, k, count, rank, runs):
    """runs: tokens of a request follow each other (prefill); else each token is a request (decode)."""
    return {"name": name, "op": "adapters", "T": T, "hidden": hidden, "q": q, "k": k, "count": count, "rank": rank,
            "runs": runs}


def listed():
    return [
        # a decode step of 64 requests: one call's latency
        _rope("rope_decode", 64, 8, 2, 128, tp=4),
        # prefill of one rank, norm included
        _rope("rope_prefill", 8192, 16, 4, 128, tp=2),
        # long prefill into an FP8 cache, V from a fused QKV buffer, the most bytes
        _rope("rope_long_fp8", 32768, 16, 2, 128, tp=4, dtype="fp8", page=64, strided=True),
        # half of each head rotated, neighbours paired, rows already normalised, ragged chunk
        _rope("rope_partial", 777, 10, 2, 64, rot=32, interleaved=True, page=32, strided=True),
        # the smallest calls: a few requests with short contexts
        _attn("attn_decode_short", 4, 1, 500, 5, 1, 128, ragged=True),
        # a decode batch, contexts of all lengths
        _attn("attn_decode", 64, 1, 4096, 8, 2, 128, ragged=True),
        # long contexts in an FP8 cache
        _attn("attn_decode_long_fp8", 16, 1, 32768, 16, 2, 128, dtype="fp8", page=64, ragged=True),
        # one chunk of a chunked prefill behind a long prefix
        _attn("attn_chunk", 1, 777, 12001, 16, 4, 128, page=64, lse=True),
        # a whole prompt, the most products
        _attn("attn_prefill", 1, 8192, 8192, 16, 4, 128, page=64),
        # prompts' chunks and single tokens in one batch, windowed layer of narrow heads
        _attn("attn_mixed_window", 12, 512, 4096, 16, 2, 64, window=1024, ragged=True),
        # a decode batch in which requests have adapters of their own
        _adapters("adapters_decode", 64, 4096, 1024, 256, 32, 16, False),
        # prefill of a few requests
        _adapters("adapters_prefill", 8192, 4096, 2048, 512, 8, 64, True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "attn", "attn", "adapters"])
    D = rng.choice([32, 64, 128, 128, 256])
    kv_heads = rng.randint(1, max(1, min(8, 1024 // D)))
    heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 8])
    dtype, page = rng.choice(["bf16", "fp8"]), rng.choice([16, 32, 64, 128])
    if op == "rope":
        heads = min(heads, kv_heads * max(1, 4096 // (D * kv_heads)))
        case = _rope("", _log_int(rng, 1, 32768), heads, kv_heads, D, rng.choice([0, 1, 2, 4, 8]),
                     rng.choice([D, D // 2]), rng.random() < 0.5, dtype, page, rng.random() < 0.5)
    elif op == "attn":
        B = _log_int(rng, 1, 128)
        kv = _log_int(rng, 16, 32768)
        q = 1 if rng.random() < 0.5 else _log_int(rng, 2, min(kv, 4096))
        case = _attn("", B, q, kv, heads, kv_heads, D, dtype, page, rng.choice([0, 0, 0, 256, 1000]),
                     rng.random() < 0.7, rng.random() < 0.5)
    else:
        runs = rng.random() < 0.5
        T = _log_int(rng, 16, 8192) if runs else _log_int(rng, 1, 512)
        head = rng.choice([64, 128])
        case = _adapters("", T, 64 * rng.randint(16, 96), head * rng.randint(2, 2048 // head),
                         head * rng.randint(1, 512 // head), _log_int(rng, 1, 16 if runs else 64),
                         rng.choice([8, 16, 32, 64]), runs)
    del case["name"]
    while (work(case)["bytes"] > MOST_BYTES or work(case)["flops"] > MOST_FLOPS or
           op == "attn" and case["B"] * case["q"] * case["heads"] * case["kv"] > MOST_SCORES):
        if op != "attn":
            case["T"] = max(1, int(case["T"] * rng.uniform(0.3, 0.9)))
        elif case["B"] > 1:
            case["B"] = max(1, int(case["B"] * rng.uniform(0.3, 0.9)))
        elif case["q"] > 64:
            case["q"] = max(1, int(case["q"] * rng.uniform(0.3, 0.9)))
        else:
            case["kv"] = max(case["q"], int(case["kv"] * rng.uniform(0.3, 0.9)))
    return case


def _lengths(case):
    """New tokens and cached tokens (the new ones among them) of each sequence."""
    if not case["ragged"]:
        return [case["q"]] * case["B"], [case["kv"]] * case["B"]
    q, kv = [], []
    for i in range(case["B"]):
        u, w = (1.0 - 0.6180339887 * i) % 1.0, (1.0 - 0.7548776662 * i) % 1.0
        u, w = u or 1.0, w or 1.0  # the first sequence is the longest
        q.append(max(1, round(case["q"] * u * u)))  # short chunks are the most common
        kv.append(max(q[-1], round(case["kv"] * w)))
    return q, kv


def work(case):
    if case["op"] == "rope":
        T, D = case["T"], case["D"]
        e = 2 if case["dtype"] == "bf16" else 1
        nq, nk = case["heads"] * D, case["kv_heads"] * D
        norm = 4 * (nq + nk) + 2 * 4 * case["tp"] * T if case["tp"] else 0
        return {"bytes": T * (2 * (nq + 2 * nk) + 2 * nq + 2 * e * nk + 4 * case["rot"] + 12) + norm,
                "flops": 3 * T * (nq + nk)}
    if case["op"] == "attn":
        D, e, w = case["D"], 2 if case["dtype"] == "bf16" else 1, case["window"]
        pairs = seen = 0
        for n, m in zip(*_lengths(case)):
            if w:
                pairs += sum(min(w, m - n + i + 1) for i in range(n))
                seen += min(m, n + w - 1)
            else:
                pairs += n * (m - n) + n * (n + 1) // 2
                seen += m
        T = sum(_lengths(case)[0])
        return {"bytes": 4 * T * case["heads"] * D + 2 * seen * case["kv_heads"] * D * e
                + (4 * T * case["heads"] if case["lse"] else 0) + 4 * (seen // case["page"]) + 8 * case["B"],
                "flops": 4 * D * case["heads"] * pairs}
    T, h, d, r = case["T"], case["hidden"], case["q"] + case["k"], case["rank"]
    used = min(T, case["count"])
    return {"bytes": 2 * T * (h + 2 * d) + 2 * used * r * (2 * h + d) + 4 * T * 3,
            "flops": 2 * T * r * (2 * h + d) + 2 * T * d}


# ------------------------------------------------------------------ inputs

def _normal(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _pool(g, pages, kv_heads, page, D, dtype, spread=1.0):
    x = _normal(g, pages, kv_heads, page, D)
    return x.to(torch.bfloat16) if dtype == "bf16" else x.mul_(spread).clamp_(-448.0, 448.0).to(FP8)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return {"rope": _prepare_rope, "attn": _prepare_attn, "adapters": _prepare_adapters}[case["op"]](case, g)


def _prepare_rope(case, g):
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
    s = {"op": "rope", "q": x[0], "k": x[1], "v": x[2], "D": D, "rot": case["rot"], "interleaved": case["interleaved"],
         "table": torch.stack([angle.cos(), angle.sin()], -1).float(), "pos": (t + first).int(),
         "slots": where[t // page] * page + t % page,
         "k_pool": _pool(g, pages, hk, page, D, case["dtype"]), "v_pool": _pool(g, pages, hk, page, D, case["dtype"]),
         "y": torch.empty(T, hq * D, device=DEV, dtype=torch.bfloat16), "tp": tp}
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
    first = torch.tensor([sum(counts[:i]) for i in range(B)], device=DEV)
    count = torch.tensor(counts, device=DEV)
    table = torch.where(at < count[:, None], order[(first[:, None] + at).clamp_(max=pages - 1)], 0).int()
    s = {"op": "attn", "q": _normal(g, T, hq * D).to(torch.bfloat16), "D": D, "window": case["window"],
         "k_pool": _pool(g, pages, hk, page, D, case["dtype"], 64.0), "v_pool": _pool(g, pages, hk, page, D, case["dtype"], 64.0),
         "k_scale": None, "v_scale": None, "block_table": table,
         "q_start": torch.tensor([0] + [sum(nq[: i + 1]) for i in range(B)], device=DEV, dtype=torch.int32),
         "kv_len": torch.tensor(nkv, device=DEV, dtype=torch.int32), "max_q": max(nq), "max_kv": max(nkv),
         "scale": D ** -0.5, "out": torch.empty(T, hq * D, device=DEV, dtype=torch.bfloat16),
         "lse": torch.empty(T, hq, device=DEV) if case["lse"] else None}
    if case["dtype"] == "fp8":
        for name in ("k_scale", "v_scale"):
            s[name] = (0.75 + 0.5 * torch.rand(hk, device=DEV, generator=g)) / 64.0
    return s


def _prepare_adapters(case, g):
    T, h, n, r = case["T"], case["hidden"], case["count"], case["rank"]
    if case["runs"]:  # requests of unequal lengths, the adapters in turn; one in nine without
        turn = (torch.arange(T, device=DEV).float() / T).pow(1.5).mul(n + max(1, n // 8)).long()
        ids = torch.where(turn < n, turn, -1)
    else:
        ids = torch.arange(T, device=DEV)[torch.randperm(T, device=DEV, generator=g)] % n
        ids = torch.where(torch.rand(T, device=DEV, generator=g) < 0.05, -1, ids)
    wide = (case["q"], case["k"])
    return {"op": "adapters", "x": _normal(g, T, h).to(torch.bfloat16), "ids": ids.int(),
            "a": [(_normal(g, n, r, h) * h ** -0.5).to(torch.bfloat16) for _ in wide],
            "b": [(_normal(g, n, d, r) * (0.3 * r ** -0.5)).to(torch.bfloat16) for d in wide],
            "scale": 0.5 + torch.rand(n, device=DEV, generator=g),
            "base": [_normal(g, T, d).to(torch.bfloat16) for d in wide],
            "y": [torch.empty(T, d, device=DEV, dtype=torch.bfloat16) for d in wide],
            "sums": [torch.empty(T, device=DEV) for _ in wide]}


# ------------------------------------------------------------------ the calls

def run(s):
    if own:
        return {"rope": _own_rope, "attn": _own_attn, "adapters": _own_adapters}[s["op"]](s)
    return {"rope": _plain_rope, "attn": _plain_attn, "adapters": _plain_adapters}[s["op"]](s)


def _call(s, make):
    """The call with its arguments marshalled once, as a serving loop keeps it."""
    if "call" not in s:
        s["call"] = make()
    s["call"]()


def _own_rope(s):
    import paper_2608_09160_amd as qkn

    def make():
        def seg(i, x, y=None):
            more = {"w": s["gamma"][i], "partials": s["sums"][i], "d_full": s["d_full"][i]} if s["tp"] else {}
            return qkn.RopeSeg(x=x, y=y, **more)
        return qkn.PreparedRopeCache(s["table"], s["pos"], s["D"], q=seg(0, s["q"], s["y"]), k=seg(1, s["k"]), v=s["v"],
                                     cache=qkn.KVCache(s["k_pool"], s["v_pool"]), slots=s["slots"],
                                     interleaved=s["interleaved"], eps=EPS)
    _call(s, make)
    return {"q": s["y"], "k": s["k_pool"], "v": s["v_pool"]}


def _own_attn(s):
    import paper_2608_09160_amd as qkn
    _call(s, lambda: qkn.PreparedAttn(
        s["q"], qkn.KVCache(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"]), s["block_table"], s["q_start"],
        s["kv_len"], max_q=s["max_q"], max_kv=s["max_kv"], scale=s["scale"], window=s["window"], out=s["out"],
        lse=s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def _own_adapters(s):
    import paper_2608_09160_amd as qkn
    _call(s, lambda: qkn.PreparedAdapters(
        s["x"], [qkn.AdapterSeg(a=a, b=b, y=y, partials=p, base=base)
                 for a, b, y, p, base in zip(s["a"], s["b"], s["y"], s["sums"], s["base"])],
        s["ids"], s["scale"]))
    return {"y": s["y"], "sums": s["sums"]}


# ------------------------------------------------------------------ plain forms, in 32 bits

def _rotate(x, cos, sin, rot, interleaved):
    """x [T, heads, D], cos and sin [T, 1, rot / 2]."""
    turn, rest = x[..., :rot], x[..., rot:]
    a, b = (turn[..., 0::2], turn[..., 1::2]) if interleaved else (turn[..., : rot // 2], turn[..., rot // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turn = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turn, rest], -1)


def _write(pool, slots, rows):
    page = pool.shape[2]
    if pool.dtype == FP8:
        pool, rows = pool.view(torch.uint8), rows.clamp(-448.0, 448.0).to(FP8).view(torch.uint8)
    pool[slots // page, :, slots % page] = rows.to(pool.dtype)


def _plain_rope(s):
    D = s["D"]
    cos, sin = (t[:, None] for t in s["table"][s["pos"].long()].unbind(-1))
    rows = []
    for i, x in enumerate((s["q"], s["k"])):
        x = x.float()
        if s["tp"]:
            x = x * s["gamma"][i] * torch.rsqrt(s["sums"][i].sum(0) / s["d_full"][i] + EPS)[:, None]
        rows.append(_rotate(x.view(x.shape[0], -1, D), cos, sin, s["rot"], s["interleaved"]))
    s["y"].copy_(rows[0].flatten(1))
    _write(s["k_pool"], s["slots"], rows[1])
    _write(s["v_pool"], s["slots"], s["v"].float().view(rows[1].shape))
    return {"q": s["y"], "k": s["k_pool"], "v": s["v_pool"]}


def _gathered(pool, table, n, scale):
    """The first n rows of every sequence: [B, kv_heads, n, D] in 32 bits."""
    page = pool.shape[2]
    j = torch.arange(n, device=DEV)
    x = (pool.view(torch.uint8) if pool.dtype == FP8 else pool)[table[:, j // page].long(), :, j % page]
    x = x.view(pool.dtype).float().transpose(1, 2)
    return (x if scale is None else x * scale[:, None, None]).contiguous()


def _plain_attn(s):
    D, kv_heads = s["D"], s["k_pool"].shape[1]
    T, group = s["q"].shape[0], s["q"].shape[1] // (D * kv_heads)
    start, kv_len = s["q_start"].long(), s["kv_len"].long()
    B, nq, nkv = kv_len.numel(), s["max_q"], s["max_kv"]
    k = _gathered(s["k_pool"], s["block_table"], nkv, s["k_scale"])
    v = _gathered(s["v_pool"], s["block_table"], nkv, s["v_scale"])
    i, j = torch.arange(nq, device=DEV), torch.arange(nkv, device=DEV)
    rows = (start[:-1, None] + i).clamp_(max=T - 1)
    q = s["q"].float()[rows].view(B, nq, kv_heads, group, D).permute(0, 2, 1, 3, 4).reshape(B, kv_heads, nq * group, D)
    at = (kv_len - (start[1:] - start[:-1]))[:, None] + i  # [B, nq]: the cache position of each new token
    seen = (j <= at[..., None]) & (j < kv_len[:, None, None])
    if s["window"]:
        seen &= j > at[..., None] - s["window"]
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


def _plain_adapters(s):
    x, ids, n = s["x"].float(), s["ids"].long(), s["scale"].numel()
    pick = (ids[:, None] == torch.arange(n, device=DEV)).float() * s["scale"]
    for i in range(2):
        a, b = s["a"][i].float(), s["b"][i].float()
        inner = (x @ a.flatten(0, 1).t()).view(-1, n, a.shape[1]) * pick[:, :, None]
        delta = inner.flatten(1) @ b.transpose(1, 2).flatten(0, 1)
        s["y"][i].copy_(s["base"][i].float() + delta)
        torch.sum(s["y"][i].float().square(), 1, out=s["sums"][i])
    return {"y": s["y"], "sums": s["sums"]}


# ------------------------------------------------------------------ the definitions, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attn": _exact_attn, "adapters": _exact_adapters}[case["op"]](case, s)


def _exact_rope(case, s):
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
        heads.append(x)
    k, v = s["k_pool"].double(), s["v_pool"].double()
    page, row = s["slots"] // case["page"], s["slots"] % case["page"]
    k[page, :, row] = heads[1]
    v[page, :, row] = s["v"].double().reshape(T, -1, D)
    return {"q": heads[0].flatten(1), "k": k, "v": v}


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
            allowed &= ahead > -case["window"]
        for h in range(case["heads"]):
            k = s["k_pool"][pages, h // group].double().reshape(-1, D)[:m]
            v = s["v_pool"][pages, h // group].double().reshape(-1, D)[:m]
            if s["k_scale"] is not None:
                k, v = k * s["k_scale"][h // group].double(), v * s["v_scale"][h // group].double()
            cols = slice(h * D, (h + 1) * D)
            score = s["q"][t:t + n, cols].double() @ k.t() / math.sqrt(D)
            norm = torch.logsumexp(score.masked_fill(~allowed, -math.inf), 1)
            out[t:t + n, cols] = torch.where(allowed, (score - norm[:, None]).exp(), 0.0) @ v
            if lse is not None:
                lse[t:t + n, h] = norm
        t += n
    return {"out": out, "lse": lse}


def _exact_adapters(case, s):
    ys, sums = [], []
    for i in range(2):
        y = s["base"][i].double()
        for n in range(case["count"]):
            rows = (s["ids"] == n).nonzero()[:, 0]
            inner = s["x"][rows].double() @ s["a"][i][n].double().t()
            y[rows] += s["scale"][n].double() * (inner @ s["b"][i][n].double().t())
        ys.append(y)
        sums.append(y.to(torch.bfloat16).double().square().sum(1))  # of the stored values
    return {"y": ys, "sums": sums}
