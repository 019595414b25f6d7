"""The attention block of one rank: every step against the definition in 64 bits on what the step before it stored,
and a replayed graph against eager calls."""
import numpy as np
import pytest
import torch

import paper_2608_09160_amd as qkn
from oracle import block as O
from paper_2608_09160_amd import block

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HIDDEN, HEADS, KV, D, PAGE = 256, 4, 2, 64, 16
EPS = 1e-6


def _host(t):
    return t.detach().double().cpu().numpy()


def _setup(seed, sequences, longest, fp8, rank=16, adapters=3):
    g = torch.Generator().manual_seed(seed)

    def mat(*shape):
        return (torch.randn(*shape, generator=g) * shape[-1] ** -0.5).to(torch.bfloat16).to(DEV)

    n_q, n_kv = HEADS * D, KV * D
    w = block.Weights(mat(n_q, HIDDEN), mat(n_kv, HIDDEN), mat(n_kv, HIDDEN), mat(HIDDEN, n_q),
                      (torch.rand(n_q, generator=g) + 0.5).to(DEV), (torch.rand(n_kv, generator=g) + 0.5).to(DEV),
                      tuple((mat(adapters, rank, HIDDEN), mat(adapters, d, rank)) for d in (n_q, n_kv, n_kv)),
                      (torch.rand(adapters, generator=g) + 0.5).to(DEV))
    pages = block.Pages(sequences, longest, PAGE, DEV)
    shape = (pages.count, KV, PAGE, D)
    if fp8:
        pools = [torch.zeros(shape, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2)]
        cache = qkn.KVCache(*pools, *((torch.rand(KV, generator=g) * 0.02 + 0.01).to(DEV) for _ in range(2)))
    else:
        cache = qkn.KVCache(*(torch.zeros(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    return g, w, pages, cache, qkn.qkn_rope_table(longest, D, device=DEV)


def _batch(g, pages, news, befores, adapters=3):
    n, m = torch.tensor(news), torch.tensor(befores)
    seq = torch.repeat_interleave(torch.arange(len(news)), n)
    pos = torch.cat([torch.arange(b, b + a) for a, b in zip(news, befores)]).int()
    x = torch.randn(len(seq), HIDDEN, generator=g).to(torch.bfloat16).to(DEV)
    start = torch.cat([torch.zeros(1, dtype=torch.long), n.cumsum(0)]).int()
    seq, pos = seq.to(DEV), pos.to(DEV)
    return block.Batch(x, pos, pages.slots(seq, pos), start.to(DEV), (n + m).int().to(DEV), pages.table, max(news),
                       max(a + b for a, b in zip(news, befores)), (seq % (adapters + 1)).int())  # one has none


def _cached(pool, scale, table, b, m):
    pages = table[b, :(m + PAGE - 1) // PAGE].long().cpu().numpy()
    x = _host(pool)[pages]
    if scale is not None:
        x = x * _host(scale)[None, :, None, None]
    return x.transpose(0, 2, 1, 3).reshape(-1, KV, D)[:m]


def _check(step, w, cache, b, tp=1, rank=0):
    """The stages' outputs, each from its own stored inputs. Runs the stages one after the other."""
    x, ids = _host(b.x), b.ids.cpu().numpy()
    ids = np.where(ids < 3, ids, -1)
    for p in step.projections:
        p()
    bases = [_host(t).copy() for t in (step.q, step.k, step.v)]
    for base, weight in zip(bases, (w.wq, w.wk, w.wv)):
        dots = np.abs(x) @ np.abs(_host(weight)).T
        O.check_rounded(base, x @ _host(weight).T, (HIDDEN / 32 + 24) * 2.0 ** -24 * dots, "bf16", "projection")
    step.adapters()
    for y, base, (a, bm) in zip((step.q, step.k, step.v), bases, w.adapters):
        ref, size = O.adapted(base, x, _host(a), _host(bm), ids, _host(w.adapter_scale))
        error = ((HIDDEN / 32 + a.shape[1] + 24) * 2.0 ** -24 + 2.0 ** -22) * size
        error[ids < 0] = 0.0
        O.check_rounded(_host(y), ref, error, "bf16", "adapters")
    if tp > 1:
        step.exchange(step.stat_q, step.stat_k, rank)
    q, k, v = (_host(t).copy() for t in (step.q, step.k, step.v))
    for stat, rows in ((step.stat_q, q), (step.stat_k, k)):
        own = (rows ** 2).sum(1)
        assert np.all(np.abs(_host(stat)[rank] - own) <= 1e-5 * own)
    step.rope()
    pos, table = b.pos.cpu().numpy(), _host(step.rope._keep[0])
    slots = b.slots.cpu().numpy()
    for name, rows, gamma, stat in (("q", q, w.gq, step.stat_q), ("k", k, w.gk, step.stat_k)):
        z = O.normed(rows, _host(gamma), _host(stat), tp * rows.shape[1], EPS)
        ref, size = O.rotated(z, table, pos, D, D, False)
        if name == "q":
            O.check_rounded(_host(step.q), ref, 2.0 ** -20 * size, "bf16", "rotated q")
        else:
            stored_k = (ref, size)
    for name, pool, scale, (ref, size) in (("k", cache.k, cache.k_scale, stored_k),
                                           ("v", cache.v, cache.v_scale, (v, np.abs(v) * 0))):
        got = _host(pool)[slots // PAGE, :, slots % PAGE]
        f = _host(scale)[None, :, None] if scale is not None else 1.0
        ref, size = (z.reshape(-1, KV, D) / f for z in (ref, size))
        error = 2.0 ** -20 * size + (2.0 ** -22 * np.abs(ref) if scale is not None else 0.0)
        O.check_rounded(got, ref, error, "fp8" if scale is not None else "bf16", f"cached {name}")
    step.attn()
    out, start, qr = _host(step.attn.out), b.q_start.cpu().numpy(), _host(step.q)
    for s, m in enumerate(b.kv_len.cpu().numpy()):
        kc, vc = (_cached(p, f, b.block_table, s, m) for p, f in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        rows = slice(start[s], start[s + 1])
        for h in range(HEADS):
            kh, vh, qh = kc[:, h * KV // HEADS], vc[:, h * KV // HEADS], qr[rows, h * D:(h + 1) * D]
            ref, _ = O.attention(qh, kh, vh, D ** -0.5)
            size, _ = O.attention(qh, kh, np.abs(vh), D ** -0.5)
            reach = D ** 0.5 * np.abs(qh).max() * np.abs(kh).max()
            e = 2.0 ** -20 * (reach + np.log2(m + 2) + 4)
            O.check_rounded(out[rows, h * D:(h + 1) * D], ref, (2.0 ** -8 + 2 * e) * size, "bf16", "attention")
    step.output()
    dots = np.abs(out) @ np.abs(_host(w.wo)).T
    O.check_rounded(_host(step.out), out @ _host(w.wo).T, (HEADS * D / 32 + 24) * 2.0 ** -24 * dots, "bf16", "output")


@pytest.mark.parametrize("fp8", [False, True])
def test_every_stage(fp8):
    g, w, pages, cache, table = _setup(1, 4, 120, fp8)
    prompts = [37, 1, 64, 90]
    b = _batch(g, pages, prompts, [0] * 4)
    _check(block.Step(w, cache, table, b, eps=EPS), w, cache, b)
    b = _batch(g, pages, [1, 17, 1, 1], prompts)  # three single tokens and a chunk
    _check(block.Step(w, cache, table, b, eps=EPS), w, cache, b)


def test_second_rank_of_two():
    """The first rank's statistics come from outside; this rank's row stays its own."""
    g, w, pages, cache, table = _setup(2, 2, 64, False)
    b = _batch(g, pages, [20, 33], [0, 0])
    other = [(torch.rand(53, generator=g) * 100 + 200).to(DEV) for _ in range(2)]

    def exchange(stat_q, stat_k, rank):
        stat_q[1 - rank].copy_(other[0])
        stat_k[1 - rank].copy_(other[1])
    step = block.Step(w, cache, table, b, tp=2, rank=1, eps=EPS, exchange=exchange)
    _check(step, w, cache, b, tp=2, rank=1)
    staged, step.out[:] = step.out.clone(), 0
    assert torch.equal(step(), staged)


def test_replayed_graph_follows_its_inputs():
    prompts = [40, 3, 100]
    outs = {}
    for replayed in (False, True):
        g, w, pages, cache, table = _setup(3, 3, 120, False)
        first = _batch(g, pages, prompts, [0] * 3)
        block.Step(w, cache, table, first)()
        b = _batch(g, pages, [1] * 3, prompts)
        b.max_kv = 120
        step = block.Step(w, cache, table, b)
        step()
        torch.cuda.synchronize()
        if replayed:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        outs[replayed] = []
        for i in range(6):
            if replayed:
                graph.replay()
            else:
                step()
            torch.cuda.synchronize()
            outs[replayed].append(step.out.clone())
            b.x.copy_(step.out)
            b.pos += 1
            b.kv_len += 1
            b.slots.copy_(pages.slots(torch.arange(3, device=DEV), b.pos))
    for eager, replay in zip(outs[False], outs[True]):
        assert torch.equal(eager, replay) and torch.isfinite(eager).all()


def test_example(capsys):
    out = block.main(prompts=(70, 1, 33), tokens=4, hidden=512, heads=4, kv_heads=2, head_dim=64)
    assert out.shape == (3, 512) and torch.isfinite(out).all()
    assert "us a step" in capsys.readouterr().out


def test_refusals():
    g, w, pages, cache, table = _setup(4, 1, 16, False)
    b = _batch(g, pages, [2], [0])
    with pytest.raises(ValueError):
        block.Step(w, cache, table, b, tp=2)
    with pytest.raises(ValueError):
        block.Step(w, cache, table, b, tp=2, rank=2, exchange=lambda *a: None)
    b.ids = None
    with pytest.raises(ValueError):
        block.Step(w, cache, table, b)


@pytest.mark.parametrize("as_handle", [False, True])
def test_one_call_on_a_given_stream(monkeypatch, as_handle):
    """What a call allocates belongs to the stream that it runs on, and the results are those of the current one."""
    from paper_2608_09160_amd import _serve
    g, w, pages, cache, table = _setup(5, 2, 300, False)
    b = _batch(g, pages, [1, 1], [260, 290])
    for pool in (cache.k, cache.v):
        pool.copy_(torch.randn(pool.shape, generator=g).to(torch.bfloat16))
    q = torch.randn(2, HEADS * D, generator=g).to(torch.bfloat16).to(DEV)
    side, streams, real = torch.cuda.Stream(), [], _serve._workspace

    def recorded(*args):
        streams.append(torch.cuda.current_stream().cuda_stream)
        return real(*args)
    monkeypatch.setattr(_serve, "_workspace", recorded)

    def calls(stream):
        base = torch.zeros(2, HEADS * D, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        out = qkn.qkn_attn(q, cache, b.block_table, b.q_start, b.kv_len, 1, b.max_kv, stream=stream)
        y = qkn.qkn_adapters_add(b.x, [qkn.AdapterSeg(*w.adapters[0], base=base)], b.ids, stream=stream)[0][0]
        turned = qkn.qkn_rope_cache(table, b.pos, D, qkn.RopeSeg(q), stream=stream)
        angles = qkn.qkn_rope_table(9, D, stream=stream)
        torch.cuda.synchronize()
        return out, y, turned, angles
    want = calls(None)
    assert streams == [torch.cuda.current_stream().cuda_stream] * 2
    got = calls(side.cuda_stream if as_handle else side)
    assert streams[2:] == [side.cuda_stream] * 2
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_replayed_graph_of_a_batch_that_loses_sequences():
    """The step's shape stays, the sequences that are left come first: the live rows are those of the full batch, the
    padding's are zeros, and nothing of the padding reaches the cache."""
    prompts = [150, 3, 400, 90]
    g, w, pages, cache, table = _setup(6, 4, 700, False)
    block.Step(w, cache, table, _batch(g, pages, prompts, [0] * 4))()
    b = _batch(g, pages, [1] * 4, prompts)
    b.max_kv = 700  # enough to split keys; those of up to 512 stay whole, so that no result depends on the others' lengths
    step = block.Step(w, cache, table, b)
    assert step.attn.workspace.numel() > 16  # split keys
    full = step().clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    pools = cache.k.clone(), cache.v.clone()
    for live in (4, 2, 1, 3, 0, 4):
        b.q_start.copy_(torch.arange(5).clamp(max=live).int())
        b.kv_len.copy_(torch.tensor([(m + 1) * (i < live) for i, m in enumerate(prompts)], dtype=torch.int32))
        b.slots.copy_(torch.where(torch.arange(4, device=DEV) < live,
                                  pages.slots(torch.arange(4, device=DEV), b.pos), -1))
        step.attn.workspace.fill_(0x7F)  # as if other calls had used it
        step.out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert step.attn.out[live:].count_nonzero() == 0 and step.out[live:].count_nonzero() == 0
        assert torch.equal(step.out[:live], full[:live])
        assert torch.equal(cache.k, pools[0]) and torch.equal(cache.v, pools[1])


def test_prepared_calls_keep_their_tensors():
    """A prepared call holds the addresses of its tensors: they live as long as it does, whatever becomes of the objects
    that named them."""
    import gc
    import weakref
    g, w, pages, cache, table = _setup(7, 2, 64, True)
    b = _batch(g, pages, [1, 1], [20, 30])

    def rows(width=HEADS * D, dtype=torch.bfloat16):
        return torch.zeros(2, width, dtype=dtype, device=DEV)
    q, k = (qkn.RopeSeg(rows(n), torch.ones(n, device=DEV), torch.ones(1, 2, device=DEV), n, rows(n))
            for n in (HEADS * D, KV * D))
    pools = qkn.KVCache(cache.k.clone(), cache.v.clone(), cache.k_scale.clone(), cache.v_scale.clone())
    seg = qkn.AdapterSeg(w.adapters[0][0].clone(), w.adapters[0][1].clone(), rows(), torch.ones(2, device=DEV), rows())
    calls = [qkn.PreparedRopeCache(table, b.pos, D, q, k, rows(KV * D), pools, b.slots),
             qkn.PreparedAttn(rows(), pools, b.block_table, b.q_start, b.kv_len, 1, 64, lse=rows(HEADS, torch.float32)),
             qkn.PreparedAdapters(rows(HIDDEN), [seg], b.ids.clone())]
    refs = [weakref.ref(t) for holder in (q, k, pools, seg) for t in vars(holder).values() if torch.is_tensor(t)]
    assert len(refs) == 4 + 4 + 4 + 5
    for holder in (q, k, pools, seg):
        for name, t in vars(holder).items():
            if torch.is_tensor(t):
                setattr(holder, name, None)
    del t
    gc.collect()
    assert all(r() is not None for r in refs)
    for call in calls:
        call()
    torch.cuda.synchronize()
    calls.clear()
    del call
    gc.collect()
    assert all(r() is None for r in refs)
