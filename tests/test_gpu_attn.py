"""Attention over the paged cache, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_09160_amd as qkn
from oracle import block as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _host(t):
    return t.detach().double().cpu().numpy()


class Batch:
    """A batch of sequences with shuffled pages; what no token sees is filled with NaN."""

    def __init__(self, seed, lens, hq, hk, D, page=16, fp8=False, spread=1.0, order="heads first", pad=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.hq, self.hk, self.D, self.page, self.fp8 = lens, hq, hk, D, page, fp8
        self.T = sum(n for n, _ in lens)
        counts = [(m + page - 1) // page for _, m in lens]
        pages = sum(counts) + 2
        perm = torch.randperm(pages, generator=g)
        width = max(counts + [1])
        self.table = torch.full((len(lens), width), pages + 7, dtype=torch.int32)  # unused entries: no such page
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = perm[at:at + c].int()
            at += c
        used = torch.zeros(pages, page, dtype=torch.bool)
        for b, (n, m) in enumerate(lens):
            for j in range(m):
                used[self.table[b, j // page], j % page] = True
        pools = []
        for _ in range(2):
            x = torch.randn(pages, hk, page, D, generator=g) * spread
            x = x.to(torch.float8_e4m3fn).float() if fp8 else x.to(torch.bfloat16).float()
            x = torch.where(used[:, None, :, None], x, torch.nan)
            pools.append(x)
        self.k, self.v = pools
        self.scales = [torch.rand(hk, generator=g) + 0.5 if fp8 else None for _ in range(2)]
        self.q = (torch.randn(self.T, hq * D, generator=g) * spread).to(torch.bfloat16)
        self.order, self.pad = order, pad
        self.q_start = torch.tensor(np.concatenate([[0], np.cumsum([n for n, _ in lens])]), dtype=torch.int32)
        self.kv_len = torch.tensor([m for _, m in lens], dtype=torch.int32)

    def _pool(self, x):
        x = x.to(torch.float8_e4m3fn if self.fp8 else torch.bfloat16).to(DEV)
        if self.order == "rows first":
            raw = x.view(torch.uint8 if self.fp8 else torch.int16)
            x = raw.transpose(1, 2).contiguous().transpose(1, 2).view(x.dtype)
        return x

    def run(self, lse=True, **kw):
        q = torch.zeros(self.T, self.hq * self.D + self.pad, dtype=torch.bfloat16, device=DEV)[:, :self.hq * self.D]
        q.copy_(self.q)
        s = [z.to(DEV) if z is not None else None for z in self.scales]
        lse = torch.full((self.T, self.hq), 7.0, device=DEV) if lse else None
        kw = {"max_q": max([n for n, _ in self.lens] + [0]), "max_kv": max([m for _, m in self.lens] + [0]), **kw}
        out = qkn.qkn_attn(q, qkn.KVCache(self._pool(self.k), self._pool(self.v), *s), self.table.to(DEV),
                           self.q_start.to(DEV), self.kv_len.to(DEV), lse=lse, **kw)
        torch.cuda.synchronize()
        return out, lse

    def sequence(self, b, h):
        """q, k, v of one sequence and query head, in 64 bits."""
        n, m = self.lens[b]
        pages = self.table[b, :(m + self.page - 1) // self.page].long()
        g = h // (self.hq // self.hk)
        k, v = (z[pages, g].reshape(-1, self.D)[:m].double().numpy() * (float(s[g]) if s is not None else 1.0)
                for z, s in ((self.k, self.scales[0]), (self.v, self.scales[1])))
        t = int(self.q_start[b])
        return self.q[t:t + n, h * self.D:(h + 1) * self.D].double().numpy(), k, v

    def check(self, out, lse, scale=None, causal=True, window=0):
        out, lse = _host(out), _host(lse)
        scale = self.D ** -0.5 if scale is None else scale
        for b, (n, m) in enumerate(self.lens):
            t = int(self.q_start[b])
            for h in range(self.hq):
                q, k, v = self.sequence(b, h)
                ref, ref_lse = O.attention(q, k, v, scale, causal, window)
                size, _ = O.attention(q, k, np.abs(v), scale, causal, window)
                # fp32 scores: sums of 32 products at a time (16 roundings at most) and the exponent's argument, relative to
                # the largest terms
                reach = scale * np.abs(q).max(initial=0) * np.abs(k).max(initial=0) * self.D
                e = 2.0 ** -20 * (reach + np.log2(m + 2) + 4)
                # weights rounded to bf16 (2^-8 at most, half of it their share of the sum apart), then the result
                got = out[t:t + n, h * self.D:(h + 1) * self.D]
                O.check_rounded(got, ref, (2.0 ** -8 + 2 * e) * size, "bf16", f"sequence {b} head {h}")
                empty = np.isneginf(ref_lse)
                assert np.array_equal(np.isneginf(lse[t:t + n, h]), empty)
                bad = np.isnan(ref_lse)
                assert np.array_equal(np.isnan(lse[t:t + n, h]), bad)
                ok = ~empty & ~bad
                assert np.all(np.abs(lse[t:t + n, h][ok] - ref_lse[ok]) <= e + 2.0 ** -22 * np.abs(ref_lse[ok]))


LENGTHS = {
    "one token, one key": [(1, 1)],
    "single tokens": [(1, 1), (1, 15), (1, 16), (1, 17), (1, 31), (1, 32), (1, 33), (1, 64), (1, 130), (1, 700)],
    "prompt": [(67, 67)],
    "chunk": [(33, 300)],
    "mixed": [(1, 200), (0, 0), (70, 70), (1, 1), (0, 50), (19, 128), (5, 6)],
    "long chunk": [(200, 523)],
}


@pytest.mark.parametrize("lens", list(LENGTHS))
@pytest.mark.parametrize("hq,hk,D,page,fp8", [(1, 1, 64, 16, False), (4, 1, 128, 16, False), (5, 1, 128, 32, True),
                                              (6, 2, 64, 64, True), (8, 2, 256, 16, False), (4, 4, 256, 128, True),
                                              (8, 1, 96, 16, False), (2, 2, 8, 16, False), (24, 1, 32, 16, True)])
def test_against_the_definition(lens, hq, hk, D, page, fp8):
    batch = Batch(len(lens) * 100 + D, LENGTHS[lens], hq, hk, D, page, fp8)
    batch.check(*batch.run())


@pytest.mark.parametrize("window", [1, 2, 16, 33, 100, 10000])
@pytest.mark.parametrize("hq,hk", [(2, 2), (16, 1), (40, 1)])
def test_windows(window, hq, hk):
    batch = Batch(window, [(1, 300), (40, 40), (3, 90), (65, 210)], hq, hk, 64)
    batch.check(*batch.run(window=window), window=window)


@pytest.mark.parametrize("hq,hk", [(2, 2), (16, 1), (40, 1)])
def test_not_causal(hq, hk):
    batch = Batch(5, [(1, 300), (40, 40), (3, 90), (20, 7)], hq, hk, 64)
    batch.check(*batch.run(causal=False), causal=False)


@pytest.mark.parametrize("hq,hk", [(1, 1), (16, 1), (40, 1)])
def test_rows_that_see_nothing(hq, hk):
    """More new tokens than the cache holds: the first ones are before its first token."""
    batch = Batch(8, [(20, 7), (9, 0), (3, 3), (80, 1)], hq, hk, 128)
    out, lse = batch.run()
    batch.check(out, lse)
    assert out[:13].abs().max() == 0 and lse[:13].isneginf().all() and out[20:29].abs().max() == 0


@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("max_kv", [1, 500, 4000])
def test_hints_do_not_change_what_is_computed(few, max_kv):
    """max_q and max_kv choose the kernel and the splits; lengths beyond them stay right."""
    batch = Batch(11, [(1, 900), (70, 300), (2, 33)], 8, 2, 128)
    batch.check(*batch.run(max_q=1 if few else 4096, max_kv=max_kv))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("order,pad", [("rows first", 8), ("heads first", 16)])
def test_strides(order, pad, fp8):
    batch = Batch(12, [(1, 70), (50, 99)], 4, 2, 64, 32, fp8, order=order, pad=pad)
    batch.check(*batch.run())


@pytest.mark.parametrize("hq", [4, 80])
@pytest.mark.parametrize("spread", [0.05, 6.0, 30.0])
def test_flat_and_peaked_weights(hq, spread):
    batch = Batch(13, [(1, 1000), (30, 400)], hq, 1, 128, spread=spread)
    batch.check(*batch.run(max_kv=1000), scale=None)


def test_rising_scores_move_the_bound():
    """Each key's score is far above all before it: every tile rescales what came before."""
    batch = Batch(14, [(1, 600), (3, 600), (40, 600)], 4, 1, 64)
    steps = torch.arange(600).float() * 0.25
    for b in range(3):
        pages = batch.table[b, :38].long()
        for j in range(600):
            batch.k[pages[j // 16], 0, j % 16] = (torch.ones(64) * steps[j]).to(torch.bfloat16).float()
    batch.q = torch.full_like(batch.q, 1.0)
    batch.check(*batch.run())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,window", [(4, 0), (40, 0), (2, 20), (40, 20), (130, 20)])
@pytest.mark.parametrize("value", ["nan", "inf"])
def test_unseen_infinities_and_nan_reach_no_row(fp8, hq, window, value):
    """A key's NaN or infinity, in K or in V, is in the result of the tokens that see the key and of no other."""
    if fp8 and value == "inf":
        pytest.skip("e4m3fn has no infinity")
    n, m = 37, 150
    batch = Batch(15, [(n, m), (1, 64)], hq, 1, 64, 16, fp8)
    clean_out, clean_lse = batch.run(window=window)
    for pool, element in (("v", 5), ("v", 63), ("k", 9)):
        for j in (m - n - 3, m - n + 4, m - 20, m - 1):
            bad = Batch(15, [(n, m), (1, 64)], hq, 1, 64, 16, fp8)
            getattr(bad, pool)[int(bad.table[0, j // 16]), 0, j % 16, element] = float(value)
            out, _ = bad.run(window=window)
            at = torch.arange(m - n, m)
            sees = (at >= j) & ((at < j + window) if window else torch.tensor(True))
            same = out[:n].view(n, hq, 64) == clean_out[:n].view(n, hq, 64)
            assert same[~sees].all(), (pool, element, j)
            assert torch.equal(out[n:], clean_out[n:])
            if pool == "v":
                hit = out[:n].view(n, hq, 64)[..., element]
                assert (hit[sees].isnan() if value == "nan" else hit[sees] == float("inf")).all()
                same[..., element] = True
                assert same.all()


def test_table_entries_and_lengths_outside_their_ranges_stay_inside_the_buffers():
    batch = Batch(16, [(1, 40), (20, 60)], 4, 1, 64)
    batch.table[0, 1], batch.table[1, 2] = -5, 1 << 30
    batch.kv_len[1] = 1 << 30
    batch.q_start[0] = -3
    out, _ = batch.run(max_kv=64)
    assert out.shape == (21, 256)
    zero = Batch(16, [(1, 40)], 4, 1, 64)
    zero.table[0, :] = -1  # no page: keys and values of zero
    out, lse = zero.run()
    assert out.abs().max() == 0 and torch.allclose(lse, torch.full_like(lse, float(np.log(40.0))), atol=1e-5)


def test_repeats_graphs_and_streams_agree():
    batch = Batch(17, [(1, 1500), (1, 20), (1, 800)], 8, 2, 128)
    want, want_lse = batch.run()
    for _ in range(3):
        out, lse = batch.run()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    kv_len = batch.kv_len.to(DEV)
    lse = torch.empty(3, 8, device=DEV)
    call = qkn.PreparedAttn(batch.q.to(DEV), qkn.KVCache(batch._pool(batch.k), batch._pool(batch.v)),
                            batch.table.to(DEV), batch.q_start.to(DEV), kv_len, max_q=1, max_kv=1500, lse=lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert torch.equal(call.out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):  # a replay reads the lengths that the device holds then
        for lens in ((1500, 20, 800), (1499, 7, 1)):
            kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
            call.out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            batch.lens = [(1, m) for m in lens]
            batch.check(call.out, lse)


def test_no_tokens():
    batch = Batch(18, [(0, 0), (0, 30)], 2, 1, 64)
    out, _ = batch.run()
    assert out.shape == (0, 128)


@pytest.mark.parametrize("hq,hk,D,fp8,n,m", [(16, 4, 128, False, 777, 3000), (5, 1, 128, True, 1, 20000),
                                             (8, 2, 64, False, 1024, 1024), (4, 1, 256, True, 300, 2100)])
def test_long(hq, hk, D, fp8, n, m):
    batch = Batch(19, [(n, m)], hq, hk, D, 64, fp8)
    out, lse = batch.run()
    rows = sorted({0, min(1, n - 1), n // 3, n // 2, n - 1})
    for h in (0, hq - 1):
        q, k, v = batch.sequence(0, h)
        for i in rows:
            ref, ref_lse = O.attention(q[i:i + 1], k[:m - n + i + 1], v[:m - n + i + 1], D ** -0.5)
            size, _ = O.attention(q[i:i + 1], k[:m - n + i + 1], np.abs(v[:m - n + i + 1]), D ** -0.5)
            e = 2.0 ** -20 * (D ** -0.5 * np.abs(q[i]).max() * np.abs(k).max() * D + 20)
            O.check_rounded(_host(out)[i, h * D:(h + 1) * D], ref[0], (2.0 ** -8 + 2 * e) * size[0], "bf16", f"{i} {h}")
            assert abs(_host(lse)[i, h] - ref_lse[0]) <= e + 2.0 ** -22 * abs(ref_lse[0])


def _padded_batch(which):
    """(batch, q_start, tokens of a sequence): a batch among tokens that no sequence has, NaN in their rows of q."""
    if which == "behind":  # a replayed batch of single tokens whose last sequences are gone
        batch = Batch(20, [(1, 1500), (1, 20), (1, 800)] + [(0, 0)] * 5, 8, 2, 128)
        start, T = [0, 1, 2, 3, 3, 3, 3, 3, 3], 8
    elif which == "before and behind":
        batch = Batch(21, [(1, 1300), (0, 40), (2, 900)], 8, 2, 128)
        start, T = [5, 6, 6, 8], 70
    elif which == "chunk":
        batch = Batch(22, [(40, 900), (33, 33)], 8, 2, 128)
        start, T = [3, 43, 76], 150
    else:  # no sequence has a token
        batch = Batch(23, [(0, 900), (0, 0)], 8, 2, 128)
        start, T = [2, 2, 2], 9
    q = torch.full((T, 8 * 128), float("nan"), dtype=torch.bfloat16)
    q[start[0]:start[-1]] = batch.q
    batch.q, batch.T = q, T
    batch.q_start = torch.tensor(start, dtype=torch.int32)
    return batch, range(start[0], start[-1])


@pytest.mark.parametrize("fill", [0, 0x7F, 0xFF])
@pytest.mark.parametrize("max_kv", [16, 1500])  # whole and split keys
@pytest.mark.parametrize("which", ["behind", "before and behind", "chunk", "nothing"])
def test_tokens_of_no_sequence_are_zeros(which, max_kv, fill):
    """Whatever the workspace held before."""
    batch, own = _padded_batch(which)
    workspace = torch.full((1 << 26,), fill, dtype=torch.uint8, device=DEV)
    out = torch.full((batch.T, 8 * 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    _, lse = batch.run(max_q=40 if which == "chunk" else 1, max_kv=max_kv, out=out, workspace=workspace)
    batch.check(out, lse)
    rest = [t for t in range(batch.T) if t not in own]
    assert rest and out[rest].count_nonzero() == 0 and lse[rest].isneginf().all()


@pytest.mark.parametrize("hq", [8, 80])
def test_no_sequence_at_all(hq):
    """T tokens and a batch of none."""
    empty = torch.empty(0, dtype=torch.int32, device=DEV)
    pool = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    q = torch.ones(5, hq * 64, dtype=torch.bfloat16, device=DEV)
    lse = torch.ones(5, hq, device=DEV)
    out = qkn.qkn_attn(q, qkn.KVCache(pool, pool.clone()), empty.view(0, 4), torch.zeros(1, dtype=torch.int32, device=DEV),
                       empty, lse=lse)
    assert out.count_nonzero() == 0 and lse.isneginf().all()


@pytest.mark.parametrize("fill", [0, 0x7F, 0xFF])
@pytest.mark.parametrize("start", [[0, 40, 20, 60], [60, 30, 10, 0], [0, 0, 1 << 30, 3], [50, 20, 60, -7]])
def test_descending_starts_stay_inside_the_buffers(start, fill):
    """Rows beside q, out and lse keep what they hold; the workspace's rest does too."""
    batch = Batch(24, [(20, 900), (20, 700), (20, 1500)], 8, 2, 128)
    batch.q_start = torch.tensor(start, dtype=torch.int32)
    whole = torch.full((62, 1024), 3.0, dtype=torch.bfloat16, device=DEV)
    sums = torch.full((62, 8), 3.0, device=DEV)
    for max_q in (1, 20):
        room = torch.full((1 << 26,), fill, dtype=torch.uint8, device=DEV)
        call = qkn.PreparedAttn(batch.q.to(DEV), qkn.KVCache(batch._pool(batch.k), batch._pool(batch.v)),
                                batch.table.to(DEV), batch.q_start.to(DEV), batch.kv_len.to(DEV), max_q=max_q, max_kv=1500,
                                out=whole[1:61], lse=sums[1:61], workspace=room)
        call()
        torch.cuda.synchronize()
        assert (whole[[0, 61]] == 3).all() and (sums[[0, 61]] == 3).all()
        assert (room[1 << 25:] == fill).all()


@pytest.mark.parametrize("hq,window", [(4, 0), (40, 0), (2, 20), (40, 20), (130, 20)])
@pytest.mark.parametrize("fp8,value", [(False, "nan"), (False, "inf"), (False, "-inf"), (True, "nan")])  # no infinity in e4m3fn
def test_infinities_and_nan_of_a_key_are_in_the_rows_that_see_it(fp8, hq, window, value):
    """A NaN, or a score of +infinity, makes the row NaN; a score of -infinity is a weight of 0."""
    n, m = 37, 150
    for j in (m - n - 3, m - n + 4, m - 20, m - 1):
        bad = Batch(25, [(n, m), (1, 64)], hq, 1, 64, 16, fp8)
        bad.k[int(bad.table[0, j // 16]), 0, j % 16, 9] = float(value)
        out, lse = (_host(t) for t in bad.run(window=window))
        largest = np.abs(_host(bad.k)[np.isfinite(_host(bad.k))]).max()
        for b, (new, kept) in enumerate(bad.lens):
            for h in range(hq):
                q, k, v = bad.sequence(b, h)
                ref, ref_lse = O.attention(q, k, v, 0.125, window=window)
                size, _ = O.attention(q, k, np.abs(v), 0.125, window=window)
                e = 2.0 ** -20 * (0.125 * np.abs(q).max() * largest * 2.0 * 64 + np.log2(kept + 2) + 4)  # scales: up to 1.5
                rows = slice(n * b, n * b + new)
                O.check_rounded(out[rows, 64 * h:64 * h + 64], ref, (2.0 ** -8 + 2 * e) * size, "bf16", f"{j} {b} {h}")
                assert np.array_equal(np.isnan(lse[rows, h]), np.isnan(ref_lse))
                ok = np.isfinite(ref_lse)
                assert np.all(np.abs(lse[rows, h][ok] - ref_lse[ok]) <= e + 2.0 ** -22 * np.abs(ref_lse[ok]))
                if b == 0:
                    at = np.arange(m - n, m)
                    sees = (at >= j) & ((at < j + window) if window else True)
                    hit = sees if value == "nan" else sees & (q[:, 9] * float(value) == np.inf)
                    assert np.array_equal(np.isnan(ref_lse), hit)  # the reference says so too


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window", [1, 100, 700, 3000])
@pytest.mark.parametrize("hq,hk", [(2, 2), (16, 1), (48, 1)])
def test_windows_of_single_tokens_with_split_keys(window, hq, hk, fp8):
    """Few rows, more keys than one part of them has: parts begin where the window does."""
    batch = Batch(26, [(1, 2000), (1, 30), (0, 0), (1, 5000), (1, 1)], hq, hk, 128, 64, fp8)
    batch.check(*batch.run(window=window), window=window)


@pytest.mark.parametrize("window", [0, 300])
@pytest.mark.parametrize("value", ["nan", "inf"])
def test_infinities_and_nan_in_split_keys(value, window):
    batch = Batch(27, [(1, 2100), (3, 1900)], 4, 1, 64)
    for b, j in ((0, 5), (0, 2098), (1, 1896), (1, 1899)):
        batch.v[int(batch.table[b, j // 16]), 0, j % 16, 40] = float(value)
    clean = Batch(27, [(1, 2100), (3, 1900)], 4, 1, 64)
    (out, lse), (want, want_lse) = batch.run(window=window), clean.run(window=window)
    assert torch.equal(lse, want_lse)
    out, want = out.view(4, 4, 64), want.view(4, 4, 64)
    same = out == want
    same[..., 40] = True
    assert same.all()
    hit = out[..., 40].isnan() if value == "nan" else out[..., 40] == float("inf")
    # tokens at 2099 of the first sequence; 1897, 1898, 1899 of the second: 1899 is seen by the last one alone
    assert hit.all()
    batch.v[int(batch.table[1, 1896 // 16]), 0, 1896 % 16, 40] = 0.0
    out = batch.run(window=window)[0].view(4, 4, 64)
    assert out[1:3, :, 40].isfinite().all() and not out[3, :, 40].isfinite().any()
