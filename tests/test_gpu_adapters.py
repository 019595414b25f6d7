"""Low-rank adapters beside the projection, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_09160_amd as qkn
from oracle import block as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _host(t):
    return t.detach().double().cpu().numpy()


def _bf16(g, *shape, scale=1.0, pad=0):
    x = torch.randn(*shape[:-1], shape[-1] + pad, generator=g) * scale
    return x.to(torch.bfloat16).to(DEV)[..., :shape[-1]]


def _ids(kind, T, count, g):
    if kind == "runs":
        return (torch.arange(T) * (count + 1) // T).int()  # the last run's id is past the adapters
    if kind == "one":
        return torch.full((T,), count - 1, dtype=torch.int32)
    if kind == "none":
        return torch.tensor([-1, count, 1 << 30])[torch.arange(T) % 3].int()
    return torch.randint(-1, count, (T,), generator=g).int()


def _check(x, segs, bases, ids, scale, what):
    n = ids.cpu().numpy()
    count, rank, hidden = segs[0].a.shape
    n = np.where((n >= 0) & (n < count), n, -1)
    factor = _host(scale) if scale is not None else np.ones(count)
    for i, (s, base) in enumerate(zip(segs, bases)):
        ref, size = O.adapted(_host(base), _host(x), _host(s.a), _host(s.b), n, factor)
        # fp32 sums of 32 products at a time, the parts' and wavefronts' sums, and the rounding of scale * (A x)
        error = ((hidden / 32 + rank + 24) * 2.0 ** -24 + 2.0 ** -22) * size
        error[n < 0] = 0.0
        y = _host(s.y)
        O.check_rounded(y, ref, error, "bf16", f"{what} segment {i}")
        if s.partials is not None:
            stored = (y ** 2).sum(1)
            assert np.all(np.abs(_host(s.partials) - stored) <= 1e-5 * stored), f"{what} segment {i} statistic"


@pytest.mark.parametrize("kind", ["random", "runs", "one", "none"])
@pytest.mark.parametrize("T,hidden,widths,count,rank", [
    (1, 64, (64,), 1, 8), (5, 1024, (128, 64), 3, 16), (64, 4096, (256, 64), 32, 16), (130, 520, (72, 8, 200), 7, 24),
    (300, 256, (1032,), 2, 128), (512, 128, (64, 64), 5, 8), (513, 192, (64, 128), 5, 64), (1500, 64, (136,), 9, 40),
    (2000, 320, (64, 64, 64), 3, 32),
])
def test_against_the_definition(kind, T, hidden, widths, count, rank):
    g = torch.Generator().manual_seed(T + hidden + rank)
    x = _bf16(g, T, hidden, pad=8)
    scale = (torch.rand(count, generator=g) + 0.5).to(DEV)
    segs, bases = [], []
    for i, d in enumerate(widths):
        bases.append(_bf16(g, T, d, pad=8 * i))
        segs.append(qkn.AdapterSeg(a=_bf16(g, count, rank, hidden, scale=hidden ** -0.5, pad=16 * i),
                                   b=_bf16(g, count, d, rank, scale=rank ** -0.5, pad=8), base=bases[-1],
                                   partials=torch.empty(T, device=DEV)))
    ids = _ids(kind, T, count, g).to(DEV)
    qkn.qkn_adapters_add(x, segs, ids, scale)
    _check(x, segs, bases, ids, scale, kind)


def test_in_place_without_scale_and_statistic():
    g = torch.Generator().manual_seed(1)
    x, y = _bf16(g, 40, 256), _bf16(g, 40, 128)
    base = y.clone()
    seg = qkn.AdapterSeg(a=_bf16(g, 4, 16, 256, scale=0.06), b=_bf16(g, 4, 128, 16, scale=0.25), y=y)
    ids = _ids("random", 40, 4, g).to(DEV)
    qkn.qkn_adapters_add(x, [seg], ids)
    _check(x, [seg], [base], ids, None, "in place")


def test_no_adapters_at_all():
    g = torch.Generator().manual_seed(2)
    x, base = _bf16(g, 9, 64), _bf16(g, 9, 64)
    seg = qkn.AdapterSeg(a=torch.empty(0, 8, 64, dtype=torch.bfloat16, device=DEV),
                         b=torch.empty(0, 64, 8, dtype=torch.bfloat16, device=DEV), base=base,
                         partials=torch.empty(9, device=DEV))
    qkn.qkn_adapters_add(x, [seg], torch.zeros(9, dtype=torch.int32, device=DEV))
    assert torch.equal(seg.y, base)


@pytest.mark.parametrize("T", [30, 700])
def test_a_request_does_not_change_another(T):
    """NaN and infinities in one request's input, base or adapter stay in its own rows; the others keep their bits."""
    g = torch.Generator().manual_seed(3)
    x, base = _bf16(g, T, 128), _bf16(g, T, 64)
    a, b = _bf16(g, 3, 16, 128, scale=0.1), _bf16(g, 3, 64, 16, scale=0.25)
    ids = (torch.arange(T, dtype=torch.int32) % 3).to(DEV)

    def rows():
        return qkn.qkn_adapters_add(x, [qkn.AdapterSeg(a=a, b=b, base=base)], ids)[0][0]
    clean = rows().clone()
    others = ids != 1
    for hurt in (a[1], b[1]):
        keep = hurt.clone()
        for value in (float("nan"), float("inf")):
            hurt[3, 5] = value
            y = rows()
            assert torch.equal(y[others], clean[others]) and not torch.isfinite(y[~others]).all()
            hurt.copy_(keep)
    for hurt in (x, base):
        keep = hurt.clone()
        hurt[4, 7] = float("nan")
        y = rows()
        same = torch.arange(T, device=DEV) != 4
        assert torch.equal(y[same], clean[same]) and y[4].isnan().any()
        hurt.copy_(keep)


def test_graph_and_repeats_agree():
    g = torch.Generator().manual_seed(4)
    x, base = _bf16(g, 64, 512), _bf16(g, 64, 192)
    seg = qkn.AdapterSeg(a=_bf16(g, 6, 8, 512), b=_bf16(g, 6, 192, 8), base=base, partials=torch.empty(64, device=DEV))
    ids = _ids("random", 64, 6, g).to(DEV)
    call = qkn.PreparedAdapters(x, [seg], ids)
    call()
    torch.cuda.synchronize()
    want, want_sum = seg.y.clone(), seg.partials.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        seg.y.zero_()
        seg.partials.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(seg.y, want) and torch.equal(seg.partials, want_sum)


def test_after_the_projection_before_the_norm():
    """The statistic replaces the projection's: the norm's Phases B+C of the adapted rows equal the whole norm."""
    g = torch.Generator().manual_seed(5)
    T, h, d = 33, 256, 128
    x, w = _bf16(g, T, h), _bf16(g, d, h, scale=h ** -0.5)
    gamma = torch.rand(d, generator=g).to(DEV) + 0.5
    seg = qkn._lib.ProjSeg(w=w)
    qkn._lib.qkn_proj_partial(x, [seg])
    ad = qkn.AdapterSeg(a=_bf16(g, 2, 8, h, scale=0.06), b=_bf16(g, 2, d, 8, scale=0.3), y=seg.y, partials=seg.partials)
    qkn.qkn_adapters_add(x, [ad], _ids("random", T, 2, g).to(DEV))
    got = qkn.qkn_apply(seg.y, gamma, seg.partials.view(1, T), d, 1e-6).float()
    z = seg.y.double()
    want = z * gamma.double() / (z.square().mean(1, keepdim=True) + 1e-6).sqrt()
    assert ((got.double() - want).abs() <= 8e-3 * want.abs()).all()


def test_no_tokens():
    seg = qkn.AdapterSeg(a=torch.empty(1, 8, 64, dtype=torch.bfloat16, device=DEV),
                         b=torch.empty(1, 64, 8, dtype=torch.bfloat16, device=DEV),
                         base=torch.empty(0, 64, dtype=torch.bfloat16, device=DEV))
    y, _ = qkn.qkn_adapters_add(torch.empty(0, 64, dtype=torch.bfloat16, device=DEV), [seg],
                                torch.empty(0, dtype=torch.int32, device=DEV))[0]
    assert y.shape == (0, 64)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("T", [3, 200, 1100])
def test_rows_without_an_adapter_keep_their_bits(T, in_place):
    """Negative zeros and NaN payloads among them."""
    g = torch.Generator().manual_seed(6)
    bits = torch.randint(-2 ** 15, 2 ** 15, (T, 64), generator=g, dtype=torch.int16).to(DEV)
    bits[:, :4] = torch.tensor([-0x8000, 0x7F81, -0x7F, 0], dtype=torch.int16, device=DEV)  # -0, NaN, NaN, 0
    base = bits.view(torch.bfloat16)
    y = base if in_place else torch.zeros_like(base)
    ids = torch.where(torch.arange(T) % 3 == 1, torch.arange(T) % 2, -1).int().to(DEV)
    a, b = _bf16(g, 2, 8, 128, scale=0.1), _bf16(g, 2, 64, 8, scale=0.3)
    want = bits.clone()
    qkn.qkn_adapters_add(_bf16(g, T, 128), [qkn.AdapterSeg(a=a, b=b, y=y, base=base)], ids)
    assert torch.equal(y.view(torch.int16)[ids < 0], want[ids < 0])
