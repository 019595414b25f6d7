"""The attention block over a 4-bit cache whose pages the device hands out: the operators together, as they are served."""
import numpy as np
import pytest
import torch

import paper_2608_09160_amd as qkn
from oracle import block as B
from oracle import cache4 as O
from oracle import pages as P
from paper_2608_09160_amd import block

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HIDDEN, HEADS, KV, D, PAGE = 256, 4, 2, 64, 16


def _host(t):
    return t.detach().double().cpu().numpy()


def _ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def _weights(g):
    def mat(*shape):
        return (torch.randn(*shape, generator=g) * shape[-1] ** -0.5).to(torch.bfloat16).to(DEV)
    n_q, n_kv = HEADS * D, KV * D
    return block.Weights(mat(n_q, HIDDEN), mat(n_kv, HIDDEN), mat(n_kv, HIDDEN), mat(HIDDEN, n_q),
                         (torch.rand(n_q, generator=g) + 0.5).to(DEV), (torch.rand(n_kv, generator=g) + 0.5).to(DEV))


def _check_attention(step, cache, b, window, sinks):
    """Attention's rows against the definition over what the cache holds now."""
    out, start, q = _host(step.attn.out), b.q_start.cpu().numpy(), _host(step.q)
    for s, m in enumerate(b.kv_len.cpu().numpy()):
        j = torch.arange(m, device=DEV)
        slots = b.block_table[s, j // PAGE].long() * PAGE + j % PAGE
        k, v = (_host(t).reshape(m, KV, D) for t in qkn.qkn_cache4_load(cache, slots))
        rows = slice(start[s], start[s + 1])
        for h in range(HEADS):
            kh, vh, qh = k[:, h * KV // HEADS], v[:, h * KV // HEADS], q[rows, h * D:(h + 1) * D]
            ref, _, size = O.attention(qh, kh, vh, D ** -0.5, window, sinks)
            reach = D ** 0.5 * np.abs(qh).max(initial=0) * np.abs(kh).max(initial=0)
            e = 2.0 ** -20 * (reach + np.log2(m + 2) + 4)
            B.check_rounded(out[rows, h * D:(h + 1) * D], ref, (2.0 ** -8 + 2 * e) * size, "bf16", "attention")


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_prompts_branches_and_single_tokens(window, sinks):
    g = torch.Generator().manual_seed(window)
    w, longest, rows = _weights(g), 160, 5
    book, cache = qkn.PageBook.empty(60, rows, longest, PAGE, DEV), qkn.KVCache4.empty(60, KV, PAGE, D, DEV)
    table = qkn.qkn_rope_table(longest, D, device=DEV)

    def run(counts, which):
        """Grows the rows, which are ascending, and steps over all rows' new tokens."""
        T = sum(counts)
        slots, pos = torch.empty(T, dtype=torch.int64, device=DEV), torch.empty(T, dtype=torch.int32, device=DEV)
        qkn.qkn_pages_grow(book, _ints(counts), _ints(which), slots, pos)
        new = np.zeros(rows, dtype=int)
        new[which] = counts
        x = torch.randn(T, HIDDEN, generator=g).to(torch.bfloat16).to(DEV)
        b = block.Batch(x, pos, slots, _ints(np.concatenate([[0], new.cumsum()])), book.kv_len, book.table, max(counts), longest)
        step = block.Step(w, cache, table, b, window=window, sinks=sinks)
        step()
        # the rows as they were written: the norm and the rotation of what the projections stored
        k, v = (_host(p.clone()) for p in (step.k, step.v))
        z = B.normed(k, _host(w.gk), _host(step.stat_k), KV * D, 1e-6)
        ref, size = B.rotated(z, _host(table), pos.cpu().numpy(), D, D, False)
        at = slots.cpu().numpy()
        def stored(pool):
            return pool.cpu().numpy()[at // PAGE, :, at % PAGE]
        O.check_stored(stored(cache.k), stored(cache.k_exp), ref.reshape(T, KV, D), 2.0 ** -20 * size.reshape(T, KV, D), "k")
        codes, exps = O.quantised(v.reshape(T, KV, D))
        assert np.array_equal(stored(cache.v), codes) and np.array_equal(stored(cache.v_exp), exps)
        _check_attention(step, cache, b, window, sinks)
        P.Book(*(t.cpu().numpy() for t in (book.refs, book.table, book.kv_len)), PAGE).check()

    run([37, 90], [0, 2])
    qkn.qkn_pages_fork(book, _ints([0, 2, 0]), _ints([1, 3, 4]), [cache])
    run([1, 1, 1, 1, 1], range(5))
    run([1, 20, 1, 1, 17], range(5))
    qkn.qkn_pages_free(book, _ints([0, 3]))
    src, dst = _ints([0] * 60), _ints([0] * 60)
    qkn.qkn_pages_compact(book, src, dst, [cache])
    assert src[0] >= 0  # something moved
    run([1, 1, 1], [1, 2, 4])
    run([25, 1, 1, 1], [0, 1, 2, 4])


def test_branches_served_from_a_graph():
    out, book, cache = block.branches(prompt=75, count=5, tokens=40, hidden=HIDDEN, heads=HEADS, kv_heads=KV, head_dim=D,
                                      window=30, sinks=3)
    again, _, _ = block.branches(prompt=75, count=5, tokens=40, hidden=HIDDEN, heads=HEADS, kv_heads=KV, head_dim=D,
                                 window=30, sinks=3)
    assert torch.equal(out, again) and out.isfinite().all()
    assert book.kv_len.tolist() == [115, 115, 115, 0, 0]
    assert out[3:].count_nonzero() == 0  # padding
    assert len({tuple(r.tolist()) for r in out[:3]}) == 3
    P.Book(*(t.cpu().numpy() for t in (book.refs, book.table, book.kv_len)), PAGE).check()
    shared = 75 // PAGE
    assert all(torch.equal(book.table[r, :shared], book.table[0, :shared]) for r in (1, 2))
    assert (book.refs == 3).sum() == shared
