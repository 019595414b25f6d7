"""Attention with a window and first tokens, and over the 4-bit cache, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_09160_amd as qkn
from oracle import block as B
from oracle import cache4 as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _host(t):
    return t.detach().double().cpu().numpy()


class Batch:
    """A batch of sequences with shuffled pages; what no token sees is filled with NaN."""

    def __init__(self, seed, lens, hq, hk, D, page=16, fmt="fp4", spread=1.0, order="heads first", pad=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.hq, self.hk, self.D, self.page, self.fmt = lens, hq, hk, D, page, fmt
        self.T = sum(n for n, _ in lens)
        counts = [(m + page - 1) // page for _, m in lens]
        pages = sum(counts) + 2
        perm = torch.randperm(pages, generator=g)
        self.table = torch.full((len(lens), max(counts + [1])), pages + 7, dtype=torch.int32)  # unused: no such page
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = perm[at:at + c].int()
            at += c
        used = torch.zeros(pages, page, dtype=torch.bool)
        for b, (n, m) in enumerate(lens):
            for j in range(m):
                used[self.table[b, j // page], j % page] = True
        self.values, self.bytes = [], []  # K's and V's, without scales
        for _ in range(2):
            x = torch.randn(pages, hk, page, D, generator=g) * spread
            if fmt == "fp4":
                codes, exps = O.quantised(x.double().numpy())
                exps = np.where(used.numpy()[:, None, :, None], exps, 255).astype(np.uint8)
                self.bytes.append([codes, exps])
                self.values.append(O.values(codes, exps))
            else:
                x = torch.where(used[:, None, :, None], x, torch.nan)
                self.values.append((x.to(torch.float8_e4m3fn) if fmt == "fp8" else x.to(torch.bfloat16)).double().numpy())
        self.scales = [torch.rand(hk, generator=g) + 0.5 if fmt == "fp8" else None for _ in range(2)]
        self.q = (torch.randn(self.T, hq * D, generator=g) * spread).to(torch.bfloat16)
        self.order, self.pad = order, pad
        self.q_start = torch.tensor(np.concatenate([[0], np.cumsum([n for n, _ in lens])]), dtype=torch.int32)
        self.kv_len = torch.tensor([m for _, m in lens], dtype=torch.int32)

    def put(self, which, b, j, g, element, value):
        """A NaN (or, in bf16, an infinity) at one place of K (0) or V (1); in 4 bits its block of 32 becomes NaN."""
        page, row = int(self.table[b, j // self.page]), j % self.page
        if self.fmt == "fp4":
            self.bytes[which][1][page, g, row, element // 32] = 255
            self.values[which] = O.values(*self.bytes[which])
        else:
            self.values[which][page, g, row, element] = value

    def cache(self):
        def pool(x):
            x = x.to(DEV)
            return x if self.order == "heads first" else x.transpose(1, 2).contiguous().transpose(1, 2)
        if self.fmt == "fp4":
            (kc, ke), (vc, ve) = self.bytes
            return qkn.KVCache4(*(pool(torch.from_numpy(x.copy())) for x in (kc, vc, ke, ve)))
        to = torch.float8_e4m3fn if self.fmt == "fp8" else torch.bfloat16
        raw = torch.uint8 if self.fmt == "fp8" else torch.int16
        pools = [pool(torch.from_numpy(x).float().to(to).view(raw)).view(to) for x in self.values]
        return qkn.KVCache(*pools, *(s.to(DEV) if s is not None else None for s in self.scales))

    def arguments(self, **kw):
        q = torch.zeros(self.T, self.hq * self.D + self.pad, dtype=torch.bfloat16, device=DEV)[:, :self.hq * self.D]
        q.copy_(self.q)
        lse = torch.full((self.T, self.hq), 7.0, device=DEV)
        kw = {"max_q": max([n for n, _ in self.lens] + [0]), "max_kv": max([m for _, m in self.lens] + [0]), "lse": lse, **kw}
        return (q, self.cache(), self.table.to(DEV), self.q_start.to(DEV), self.kv_len.to(DEV)), kw

    def run(self, **kw):
        a, kw = self.arguments(**kw)
        out = qkn.qkn_attn(*a, **kw)
        torch.cuda.synchronize()
        return out, kw["lse"]

    def sequence(self, b, h):
        n, m = self.lens[b]
        pages = self.table[b, :(m + self.page - 1) // self.page].long().numpy()
        g = h // (self.hq // self.hk)
        k, v = (z[pages, g].reshape(-1, self.D)[:m] * (float(s[g]) if s is not None else 1.0)
                for z, s in zip(self.values, self.scales))
        t = int(self.q_start[b])
        return self.q[t:t + n, h * self.D:(h + 1) * self.D].double().numpy(), k, v

    def check(self, out, lse, window=0, sinks=0, heads=None):
        out, lse, scale = _host(out), _host(lse), self.D ** -0.5
        for b, (n, m) in enumerate(self.lens):
            t = int(self.q_start[b])
            for h in range(self.hq) if heads is None else heads:
                q, k, v = self.sequence(b, h)
                ref, ref_lse, size = O.attention(q, k, v, scale, window, sinks)
                # fp32 scores: sums of 32 products at a time (16 roundings at most) and the exponent's argument, relative
                # to the largest terms
                reach = scale * np.abs(q).max(initial=0) * np.nan_to_num(np.abs(k)).max(initial=0) * self.D
                e = 2.0 ** -20 * (reach + np.log2(m + 2) + 4)
                # weights rounded to bf16 (2^-8 at most, half of it their share of the sum apart), then the result
                # a weight is relative to a key's of 1 or more, in 32 bits: below 2^-126, the least normal number, it may
                # be taken as 0, for each of m keys
                lost = m * 2.0 ** -126 * np.nan_to_num(np.abs(v)).max(initial=0)
                B.check_rounded(out[t:t + n, h * self.D:(h + 1) * self.D], ref, (2.0 ** -8 + 2 * e) * size + lost, "bf16",
                                f"sequence {b} head {h}")
                empty, bad = np.isneginf(ref_lse), np.isnan(ref_lse)
                got = lse[t:t + n, h]
                assert np.array_equal(np.isneginf(got), empty) and np.array_equal(np.isnan(got), bad)
                ok = ~empty & ~bad
                assert np.all(np.abs(got[ok] - ref_lse[ok]) <= e + 2.0 ** -22 * np.abs(ref_lse[ok]))


LENGTHS = {
    "one token, one key": [(1, 1)],
    "single tokens": [(1, 1), (1, 15), (1, 16), (1, 17), (1, 31), (1, 32), (1, 33), (1, 64), (1, 130), (1, 700)],
    "prompt": [(67, 67)],
    "chunk": [(33, 300)],
    "mixed": [(1, 200), (0, 0), (70, 70), (1, 1), (0, 50), (19, 128), (5, 6)],
    "long chunk": [(200, 523)],
    "rows that see nothing": [(20, 7), (9, 0), (3, 3), (80, 1)],
}
HEADS4 = [(1, 1, 64, 16), (4, 1, 128, 16), (5, 1, 128, 32), (6, 2, 64, 64), (8, 2, 256, 16), (4, 4, 256, 128), (8, 1, 96, 16),
          (24, 1, 32, 16), (3, 1, 160, 32), (40, 1, 64, 16), (60, 2, 128, 16)]


@pytest.mark.parametrize("lens", list(LENGTHS))
@pytest.mark.parametrize("hq,hk,D,page", HEADS4)
def test_4_bits_against_the_definition(lens, hq, hk, D, page):
    batch = Batch(len(lens) * 100 + D, LENGTHS[lens], hq, hk, D, page)
    batch.check(*batch.run())


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("window,sinks", [(1, 1), (1, 40), (2, 16), (16, 4), (33, 70), (100, 1), (64, 128), (10000, 5), (20, 10000)])
@pytest.mark.parametrize("hq,hk", [(2, 2), (16, 1), (40, 1)])
def test_windows_with_first_tokens(window, sinks, hq, hk, fmt):
    batch = Batch(window + sinks, [(1, 300), (40, 40), (3, 90), (65, 210), (30, 9)], hq, hk, 64, fmt=fmt)
    batch.check(*batch.run(window=window, sinks=sinks), window=window, sinks=sinks)


@pytest.mark.parametrize("fmt,D", [("bf16", 128), ("fp8", 128), ("fp4", 128), ("bf16", 256), ("fp4", 256), ("fp8", 16)])
@pytest.mark.parametrize("hq", [3, 20, 50])
def test_windows_with_first_tokens_of_other_heads(hq, fmt, D):
    batch = Batch(D + hq, [(1, 400), (50, 300), (2, 70)], hq, 1, D, 32, fmt)
    batch.check(*batch.run(window=50, sinks=20), window=50, sinks=20)


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("window,sinks", [(1, 1), (100, 4), (700, 300), (64, 2500), (3000, 128), (33, 1100)])
@pytest.mark.parametrize("hq,hk", [(2, 2), (48, 1)])
def test_single_tokens_with_split_keys(window, sinks, hq, hk, fmt):
    """Few rows, more keys than one part of them has; first tokens and window more than 64 pages of 16 apart, and first
    tokens on more pages than that."""
    batch = Batch(26, [(1, 2000), (1, 30), (0, 0), (1, 6000), (1, 1)], hq, hk, 128, 16, fmt)
    batch.check(*batch.run(window=window, sinks=sinks), window=window, sinks=sinks)


@pytest.mark.parametrize("window,sinks", [(0, 0), (4100, 3), (50, 4)])
@pytest.mark.parametrize("hq,hk,D,most", [(8, 8, 64, 5000), (16, 8, 128, 4500), (8, 8, 256, 4100), (40, 8, 128, 4096)])
def test_many_sequences_of_unequal_lengths(hq, hk, D, most, window, sinks):
    """More tiles than fill half the chip's places with few workgroups to a CU, split to make unequal sequences even; also
    where max_q says less than the sequences have."""
    lens = [(1 + b % 3, (b * 37) % 150) for b in range(30 if D == 256 else 40)]
    lens[0], lens[3], lens[17], lens[-1] = (3, most), (0, 0), (1, 2077), (2, 1024)
    batch = Batch(most + hq, lens, hq, hk, D)
    for max_q in (3, 1):
        batch.check(*batch.run(window=window, sinks=sinks, max_q=max_q), window=window, sinks=sinks, heads=[0, hq - 1])


@pytest.mark.parametrize("window,sinks", [(64, 4090), (1, 4500), (2000, 2100), (100, 100000)])
@pytest.mark.parametrize("hq,hk,D", [(8, 8, 64), (16, 8, 128)])
def test_many_sequences_with_many_first_tokens(hq, hk, D, window, sinks):
    """As above: first tokens and a short window together are as many keys as are split."""
    lens = [(1 + b % 3, (b * 37) % 150) for b in range(40)]
    lens[0], lens[3], lens[17], lens[-1] = (3, 5000), (0, 0), (1, 4777), (2, 1024)
    batch = Batch(hq + sinks, lens, hq, hk, D)
    for max_q in (3, 1):
        batch.check(*batch.run(window=window, sinks=sinks, max_q=max_q), window=window, sinks=sinks, heads=[0, hq - 1])


@pytest.mark.parametrize("window,sinks", [(0, 0), (2500, 3), (50, 4)])
def test_many_chunks_of_unequal_lengths(window, sinks):
    """As above, of more rows."""
    lens = [(64 - b % 5, 64 + 9 * b) for b in range(16)]
    lens[2], lens[15] = (60, 3001), (61, 2048)
    batch = Batch(window, lens, 16, 4, 128)
    batch.check(*batch.run(window=window, sinks=sinks), window=window, sinks=sinks, heads=[0, 6, 15])


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("hq,hk,D,n,m,window,sinks", [(16, 4, 128, 777, 5000, 1000, 30), (16, 2, 64, 300, 4000, 64, 1300),
                                                      (8, 8, 256, 200, 2500, 200, 4)])
def test_chunks_far_behind_their_first_tokens(hq, hk, D, n, m, window, sinks, fmt):
    batch = Batch(27, [(n, m), (1, 2100)], hq, hk, D, 16, fmt)
    batch.check(*batch.run(window=window, sinks=sinks), window=window, sinks=sinks, heads=(0, hq - 1))


@pytest.mark.parametrize("hq", [2, 16, 80])
@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
def test_what_first_tokens_do_not_change(fmt, hq):
    """None of them, or no window: the bits of the call without; first tokens that all rows see anyway: those of no window
    in value."""
    batch = Batch(31, [(1, 300), (40, 40), (65, 210)], hq, 1, 64, fmt=fmt)
    plain, window = batch.run(), batch.run(window=50)
    assert all(torch.equal(a, b) for a, b in zip(plain, batch.run(sinks=100)))
    assert all(torch.equal(a, b) for a, b in zip(window, batch.run(window=50, sinks=0)))
    batch.check(*batch.run(window=50, sinks=300))
    batch.check(*batch.run(window=50, sinks=2 ** 31 - 1))


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("order,pad", [("rows first", 8), ("heads first", 16)])
def test_strides(order, pad, fmt):
    batch = Batch(12, [(1, 70), (50, 99)], 4, 2, 64, 32, fmt, order=order, pad=pad)
    batch.check(*batch.run(window=20, sinks=5), window=20, sinks=5)


@pytest.mark.parametrize("hq", [4, 80])
@pytest.mark.parametrize("spread", [0.05, 6.0, 30.0])
def test_flat_and_peaked_weights(hq, spread):
    batch = Batch(13, [(1, 1000), (30, 400)], hq, 1, 128, spread=spread)
    batch.check(*batch.run(max_kv=1000))


@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("max_kv", [1, 500, 4000])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 10)])
def test_hints_do_not_change_what_is_computed(few, max_kv, window, sinks):
    batch = Batch(11, [(1, 900), (70, 300), (2, 33)], 8, 2, 128)
    batch.check(*batch.run(max_q=1 if few else 4096, max_kv=max_kv, window=window, sinks=sinks), window=window, sinks=sinks)


@pytest.mark.parametrize("hq", [2, 40, 130])
@pytest.mark.parametrize("fmt,value", [("bf16", "nan"), ("bf16", "inf"), ("fp8", "nan"), ("fp4", "nan")])
def test_unseen_infinities_and_nan_reach_no_row(fmt, value, hq):
    """A key's NaN or infinity, in V or in K, is in the result of the tokens that see the key and of no other."""
    n, m, window, sinks = 37, 150, 20, 6
    lens = [(n, m), (1, 64)]
    clean, _ = Batch(15, lens, hq, 1, 64, 16, fmt).run(window=window, sinks=sinks)
    for which, element in ((1, 5), (1, 63), (0, 9)):
        for j in (0, 5, 6, m - n - 3, m - n + 4, m - 20, m - 1):
            bad = Batch(15, lens, hq, 1, 64, 16, fmt)
            bad.put(which, 0, j, 0, element, float(value))
            out, _ = bad.run(window=window, sinks=sinks)
            at = torch.arange(m - n, m)
            sees = (at >= j) & ((at < j + window) | torch.tensor(j < sinks))
            same = out[:n].view(n, hq, 64) == clean[:n].view(n, hq, 64)
            assert same[~sees].all(), (which, element, j)
            assert torch.equal(out[n:], clean[n:])
            if which:
                near = slice(element // 32 * 32, element // 32 * 32 + 32) if fmt == "fp4" else slice(element, element + 1)
                hit = out[:n].view(n, hq, 64)[..., near]
                assert (hit[sees].isnan() if value == "nan" else hit[sees] == float("inf")).all()
                same[..., near] = True
                assert same.all()


@pytest.mark.parametrize("hq", [2, 16, 40, 130])
@pytest.mark.parametrize("exponent", [0, 1, 252, 253, 254, 255])
def test_what_lies_behind_a_sequence_in_its_last_page(exponent, hq):
    """Rows that were never written hold any bytes: exponents whose values are beyond bf16 too."""
    lens = [(1, 70), (1, 1), (37, 150), (20, 20)]
    batch = Batch(33, lens, hq, 1, 64, 32)
    want, want_lse = batch.run(window=40, sinks=3)
    unused = [np.repeat(e == 255, 16, -1) for _, e in batch.bytes]
    for (codes, exps), bad in zip(batch.bytes, unused):
        codes[bad] = np.random.default_rng(1).integers(0, 256, int(bad.sum()))
        exps[exps == 255] = exponent
    out, lse = batch.run(window=40, sinks=3)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("hq", [2, 16, 40, 130])
@pytest.mark.parametrize("exponent", [253, 254, 255])
@pytest.mark.parametrize("which", [0, 1])
def test_a_nan_block_is_in_the_rows_that_see_it(which, exponent, hq):
    n, m, window, sinks = 37, 150, 20, 6
    for j in (5, m - n - 3, m - 20):
        batch = Batch(34, [(n, m), (1, 64)], hq, 1, 64, 16)
        page, row = int(batch.table[0, j // 16]), j % 16
        batch.bytes[which][1][page, 0, row, 1] = exponent
        batch.values[which] = O.values(*batch.bytes[which])
        batch.check(*batch.run(window=window, sinks=sinks), window=window, sinks=sinks)


def test_table_entries_and_lengths_outside_their_ranges_stay_inside_the_buffers():
    batch = Batch(16, [(1, 40), (20, 60)], 4, 1, 64)
    batch.table[0, 1], batch.table[1, 2] = -5, 1 << 30
    batch.kv_len[1] = 1 << 30
    batch.q_start[0] = -3
    for kw in ({}, dict(window=7, sinks=30)):
        assert batch.run(max_kv=64, **kw)[0].shape == (21, 256)
    zero = Batch(16, [(1, 40)], 4, 1, 64)
    zero.table[0, :] = -1  # no page: keys and values of zero
    out, lse = zero.run()
    assert out.abs().max() == 0 and torch.allclose(lse, torch.full_like(lse, float(np.log(40.0))), atol=1e-5)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
def test_repeats_graphs_and_streams_agree(fmt):
    batch = Batch(17, [(1, 1500), (1, 20), (1, 800)], 8, 2, 128, fmt=fmt)
    kw = dict(window=200, sinks=10)
    want, want_lse = batch.run(**kw)
    for _ in range(3):
        out, lse = batch.run(**kw)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    a, more = batch.arguments(**kw)
    call, kv_len, lse = qkn.PreparedAttn(*a, **more), a[4], more["lse"]
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
            batch.check(call.out, lse, **kw)


@pytest.mark.parametrize("fmt", ["bf16", "fp4"])
@pytest.mark.parametrize("max_q,max_kv", [(1, 16), (1, 1500), (40, 1500)])
def test_tokens_of_no_sequence_are_zeros(max_q, max_kv, fmt):
    batch = Batch(21, [(1, 1300), (0, 40), (2, 900)], 8, 2, 128, fmt=fmt)
    q = torch.full((70, 8 * 128), float("nan"), dtype=torch.bfloat16)
    q[5:8] = batch.q
    batch.q, batch.T, batch.q_start = q, 70, torch.tensor([5, 6, 6, 8], dtype=torch.int32)
    out = torch.full((70, 8 * 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    _, lse = batch.run(max_q=max_q, max_kv=max_kv, out=out, window=300, sinks=40)
    batch.check(out, lse, window=300, sinks=40)
    rest = list(range(5)) + list(range(8, 70))
    assert out[rest].count_nonzero() == 0 and lse[rest].isneginf().all()


def test_no_tokens():
    out, _ = Batch(18, [(0, 0), (0, 30)], 2, 1, 64).run(window=3, sinks=2)
    assert out.shape == (0, 128)
