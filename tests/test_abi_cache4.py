"""The C ABI of the 4-bit cache and of first tokens beside a window, without a GPU: struct layout, refusals, overlap rules,
path choice. Pointers are fake addresses that nothing dereferences ("validate_only" is set, or the call is refused)."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2608_09160_amd import _lib as L
from paper_2608_09160_amd import _serve as S

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
BASE, MB = 0x7f0000000000, 1 << 20
DRY = L.QKN_EDRYRUN


@pytest.fixture
def dry():
    lib = S.load()
    assert lib.qkn_set_option(b"validate_only", 1) == 0
    yield lib
    assert lib.qkn_set_option(b"validate_only", 0) == 0


def cache(D=128, **kw):
    c, e = D // 2, D // 32
    base = dict(k=BASE + 1000 * MB, v=BASE + 1200 * MB, k_exp=BASE + 1400 * MB, v_exp=BASE + 1500 * MB, num_pages=64,
                page_size=16, n_kv=2, head_dim=D)
    for pool, w in (("k", c), ("v", c), ("ke", e), ("ve", e)):
        base.update({pool + "_token": w, pool + "_head": 16 * w, pool + "_page": 32 * w})
    base.update(kw)
    return S.QknCache4(**base)


def args(**kw):
    base = dict(q=BASE, ldq=1024, out=BASE + 100 * MB, ldo=1024, lse=BASE + 200 * MB, q_start=BASE + 210 * MB,
                kv_len=BASE + 220 * MB, block_table=BASE + 230 * MB, ld_table=256, T=64, batch=64, n_q=8, max_q=1,
                max_kv=4096, causal=1, window=0, scale=0.1)
    base.update(kw)
    return S.QknAttnArgs(**base)


def attn4(lib, a=None, c=None, sinks=0, ws=BASE + 4000 * MB, ws_bytes=1 << 32):
    a, c = args() if a is None else a, cache() if c is None else c
    return lib.qkn_attn4(ctypes.byref(a), sinks, ctypes.byref(c), ws, ws_bytes, None)


def seg(at, heads, D=128, **kw):
    base = dict(x=BASE + at * MB, ldx=heads * D, w=BASE + (at + 100) * MB, partials=BASE + (at + 110) * MB,
                d_full=heads * 2 * D, y=BASE + (at + 120) * MB, ldy=heads * D, heads=heads)
    base.update(kw)
    return S.QknRopeSeg(**base)


def rope4(lib, **kw):
    D = kw.get("D", 128)
    a = dict(q=seg(0, 8, D), k=seg(300, 2, D), v=BASE + 600 * MB, ldv=2 * D, T=64, D=D, rot=D, inter=0,
             table=BASE + 700 * MB, n_pos=4096, pos=BASE + 800 * MB, slots=BASE + 810 * MB, cache=cache(D), tp=2,
             eps=1e-6)
    a.update(kw)
    ref = [ctypes.byref(a[n]) if a[n] is not None else None for n in ("q", "k", "cache")]
    return lib.qkn_rope_cache4(ref[0], ref[1], a["v"], a["ldv"], a["T"], a["D"], a["rot"], a["inter"], a["table"],
                               a["n_pos"], a["pos"], a["slots"], ref[2], a["tp"], ctypes.c_float(a["eps"]), None)


def load4(lib, c=None, **kw):
    a = dict(slots=BASE, T=64, k=BASE + 100 * MB, ldk=256, v=BASE + 200 * MB, ldv=256)
    a.update(kw)
    c = cache() if c is None else c
    return lib.qkn_cache4_load(ctypes.byref(c), a["slots"], a["T"], a["k"], a["ldk"], a["v"], a["ldv"], None)


def test_accepted(dry):
    assert attn4(dry) == DRY and attn4(dry, sinks=4) == DRY and attn4(dry, args(window=100), sinks=2 ** 31 - 1) == DRY
    assert attn4(dry, args(T=0, q=None, out=None)) == L.QKN_OK
    assert attn4(dry, c=cache(num_pages=0, k=None, v=None, k_exp=None, v_exp=None)) == DRY
    assert rope4(dry) == DRY and rope4(dry, T=0) == L.QKN_OK and rope4(dry, q=None) == DRY and rope4(dry, k=None) == DRY
    assert rope4(dry, v=None) == DRY and rope4(dry, k=seg(300, 2, y=None)) == DRY
    assert rope4(dry, k=None, cache=cache(k=None, k_exp=None)) == DRY  # V alone: K's pools are not touched
    assert load4(dry) == DRY and load4(dry, v=None) == DRY and load4(dry, T=0) == L.QKN_OK


@pytest.mark.parametrize("max_q,n_q,D,name", [
    (1, 8, 128, "attn<128,16>/fp4"), (1, 34, 128, "attn<128,32>/fp4"), (16, 8, 128, "attn<128,64>/fp4"),
    (17, 8, 128, "attn<128,64,shared>/fp4"), (4096, 8, 128, "attn<128,128,shared>/fp4"), (1, 8, 32, "attn<64,16>/fp4"),
    (1, 8, 96, "attn<128,16>/fp4"), (9, 8, 256, "attn<256,64,shared>/fp4"),
])
def test_attention_kernels(dry, max_q, n_q, D, name):
    a = args(max_q=max_q, n_q=n_q, ldq=n_q * D, ldo=n_q * D, T=max(64, max_q), max_kv=4096 + max_q)
    assert attn4(dry, a, cache(D)) == DRY
    assert L.qkn_last_launch()["kernel"] == name


def test_first_tokens_choose_the_kernel_only_beside_a_window(dry):
    c = S.QknCache(k=BASE + 1000 * MB, v=BASE + 2000 * MB, num_pages=4096, page_size=16, n_kv=2, head_dim=128, fp8=0,
                   k_page=4096, k_head=2048, k_token=128, v_page=4096, v_head=2048, v_token=128)
    for window, sinks, name in ((0, 0, "attn<128,16>/bf16"), (0, 9, "attn<128,16>/bf16"), (9, 0, "attn<128,16>/bf16"),
                                (9, 9, "attn<128,16>/bf16+sinks")):
        a = args(window=window)
        assert dry.qkn_attn_sinks(ctypes.byref(a), sinks, ctypes.byref(c), BASE + 4000 * MB, 1 << 32, None) == DRY
        assert L.qkn_last_launch()["kernel"] == name
    a = args(window=9)
    assert dry.qkn_attn_sinks(ctypes.byref(a), -1, ctypes.byref(c), BASE + 4000 * MB, 1 << 32, None) == L.QKN_EINVAL
    assert dry.qkn_attn_sinks(ctypes.byref(a), 1, None, BASE + 4000 * MB, 1 << 32, None) == L.QKN_EINVAL
    assert dry.qkn_attn_sinks(None, 1, ctypes.byref(c), BASE + 4000 * MB, 1 << 32, None) == L.QKN_EINVAL
    # qkn_attn's workspace is enough for every window and number of first tokens
    for T, batch, max_q, max_kv in ((64, 64, 1, 4096), (777, 1, 777, 12001), (300, 4, 200, 30000)):
        a = args(T=T, batch=batch, max_q=max_q, max_kv=max_kv)
        need = dry.qkn_attn_workspace_bytes(ctypes.byref(a), ctypes.byref(c))
        for window in (1, 100, 1 << 30):
            for sinks in (0, 1, 4096, 2 ** 31 - 1):
                a = args(T=T, batch=batch, max_q=max_q, max_kv=max_kv, window=window)
                assert dry.qkn_attn_sinks(ctypes.byref(a), sinks, ctypes.byref(c), BASE + 4000 * MB, need, None) == DRY


def test_workspace(dry):
    a, c = args(), cache()
    need = dry.qkn_attn4_workspace_bytes(ctypes.byref(a), ctypes.byref(c))
    assert need > 0 and attn4(dry, ws_bytes=need) == DRY and attn4(dry, ws_bytes=need - 1) == L.QKN_EINVAL
    assert attn4(dry, args(window=64), sinks=9, ws_bytes=need) == DRY
    # a layer's without a window is enough for its windows, whichever tiles are split
    for T, batch, max_q, n_kv in ((64, 64, 1, 8), (40, 40, 1, 8), (400, 100, 4, 8), (1000, 64, 60, 1), (9000, 2, 4096, 1)):
        for max_kv in (1, 511, 2048, 4095, 4096, 100000):
            c = cache(n_kv=n_kv, num_pages=8, k_page=16 * 64 * n_kv, v_page=16 * 64 * n_kv, ke_page=64 * n_kv, ve_page=64 * n_kv)
            whole = args(T=T, batch=batch, max_q=max_q, max_kv=max_kv)
            need = dry.qkn_attn4_workspace_bytes(ctypes.byref(whole), ctypes.byref(c))
            for window in (0, 1, 4095, 4096, 1 << 20):
                a = args(T=T, batch=batch, max_q=max_q, max_kv=max_kv, window=window)
                assert dry.qkn_attn4_workspace_bytes(ctypes.byref(a), ctypes.byref(c)) == need
                assert attn4(dry, a, c, ws_bytes=need) == DRY
    assert dry.qkn_attn4_workspace_bytes(None, ctypes.byref(c)) == L.QKN_EINVAL
    assert dry.qkn_attn4_workspace_bytes(ctypes.byref(a), None) == L.QKN_EINVAL


@pytest.mark.parametrize("T,batch,max_q,n_kv,keys", [(64, 64, 1, 8, 4096), (40, 40, 1, 8, 4096), (1500, 20, 64, 4, 2048)])
def test_first_tokens_count_where_long_keys_are_split(dry, T, batch, max_q, n_kv, keys):
    """A row reads its first tokens besides its window: with that many together the keys are split (into a workspace) where
    a window of as many would be."""
    c = cache(n_kv=n_kv, num_pages=8, k_page=16 * 64 * n_kv, v_page=16 * 64 * n_kv, ke_page=64 * n_kv, ve_page=64 * n_kv)
    for window, sinks, split in ((keys, 0, True), (keys - 1, 0, False), (64, keys - 64, True), (64, keys - 65, False),
                                 (1, 2 ** 31 - 1, True), (2 ** 31 - 1, 2 ** 31 - 1, True)):
        a = args(T=T, batch=batch, max_q=max_q, max_kv=16384, ld_table=1024, window=window)
        assert attn4(dry, a, c, sinks, ws=None, ws_bytes=0) == (L.QKN_EINVAL if split else DRY), (window, sinks)
        need = dry.qkn_attn4_workspace_bytes(ctypes.byref(a), ctypes.byref(c))
        assert attn4(dry, a, c, sinks, ws_bytes=need) == DRY
        # as many keys as the sequences have at most
        a = args(T=T, batch=batch, max_q=max_q, max_kv=keys - 1, ld_table=1024, window=window)
        assert attn4(dry, a, c, sinks, ws=None, ws_bytes=0) == DRY


def test_attention_of_2_32_threads_is_refused(dry):
    """As QKN_ENOTSUP by the validation, not as QKN_EHIP by a launch: 16 rows to a workgroup of 256 threads, a workgroup more for
    the sequence, 8 heads of keys; and the joining of split keys, 8 rows to one."""
    c = dict(n_kv=8, k_page=8 * 512, v_page=8 * 512, ke_page=8 * 32, ve_page=8 * 32)
    far = dict(q=1 << 40, ldq=512, out=1 << 41, ldo=512, lse=None, n_q=8, max_q=1)
    most = 16 * ((1 << 21) - 2) + 15
    for T, want in ((most, DRY), (most + 1, L.QKN_ENOTSUP)):
        assert attn4(dry, args(T=T, batch=1, max_kv=16, **far), cache(64, **c)) == want  # few keys: not split
    most = (1 << 24) - 1  # 8 rows a token
    for T, want in ((most, DRY), (most + 1, L.QKN_ENOTSUP)):
        a = args(T=T, batch=1, max_kv=1 << 16, ld_table=1 << 12, **far)
        need = dry.qkn_attn4_workspace_bytes(ctypes.byref(a), ctypes.byref(cache(64, **c)))
        assert need > 0 and attn4(dry, a, cache(64, **c), ws_bytes=need) == want


MALFORMED = [dict(num_pages=-1), dict(page_size=24), dict(page_size=0), dict(n_kv=0), dict(head_dim=0), dict(head_dim=48),
             dict(k_token=63), dict(v_head=0), dict(ke_token=3), dict(ve_page=-4), dict(k_page=(1 << 40) + 1)]


@pytest.mark.parametrize("kw", MALFORMED)
def test_malformed_caches(dry, kw):
    assert attn4(dry, c=cache(**kw)) == L.QKN_EINVAL
    assert rope4(dry, cache=cache(**kw)) == L.QKN_EINVAL
    assert load4(dry, cache(**kw)) == L.QKN_EINVAL


@pytest.mark.parametrize("pool", ["k", "v", "k_exp", "v_exp"])
def test_missing_pools(dry, pool):
    assert attn4(dry, c=cache(**{pool: None})) == L.QKN_EINVAL
    assert rope4(dry, cache=cache(**{pool: None})) == L.QKN_EINVAL
    assert load4(dry, cache(**{pool: None})) == L.QKN_EINVAL


@pytest.mark.parametrize("kw", [dict(T=-1), dict(scale=0.0), dict(window=-1), dict(causal=0, window=3), dict(n_q=7), dict(q=None)])
def test_attention_refusals(dry, kw):
    assert attn4(dry, args(**kw)) == L.QKN_EINVAL
    assert attn4(dry, sinks=-1) == L.QKN_EINVAL


@pytest.mark.parametrize("c", [dict(page_size=8), dict(k=BASE + 1000 * MB + 8), dict(v_token=72), dict(k_page=2052),
                               dict(ke_token=1 << 27)])
def test_attention_not_supported(dry, c):
    assert attn4(dry, c=cache(**c)) == L.QKN_ENOTSUP
    assert attn4(dry, args(n_q=2, ldq=1024), cache(288)) == L.QKN_ENOTSUP


@pytest.mark.parametrize("a", [dict(out=BASE + 1000 * MB), dict(out=BASE + 1200 * MB), dict(out=BASE + 1400 * MB),
                               dict(lse=BASE + 1500 * MB), dict(out=BASE), dict(lse=BASE + 4000 * MB)])
def test_attention_overlap(dry, a):
    assert attn4(dry, args(**a)) == L.QKN_EOVERLAP


@pytest.mark.parametrize("kw", [dict(q=None, k=None, v=None), dict(k=None, v=None), dict(cache=None), dict(slots=None), dict(pos=None),
                                dict(table=None), dict(D=64), dict(rot=130), dict(rot=3), dict(T=-1), dict(tp=0), dict(eps=-1.0),
                                dict(ldv=255), dict(cache=cache(n_kv=3)), dict(cache=cache(D=64))])
def test_write_refusals(dry, kw):
    if kw.get("D"):  # the caches' other head size
        kw = dict(D=64, cache=cache(128), q=seg(0, 8, 64), k=seg(300, 2, 64), rot=64)
    assert rope4(dry, **kw) == L.QKN_EINVAL


@pytest.mark.parametrize("kw", [dict(cache=cache(k_exp=BASE + 600 * MB)), dict(cache=cache(v=BASE + 300 * MB)),
                                dict(cache=cache(v_exp=BASE + 420 * MB)), dict(cache=cache(v=BASE + 1000 * MB)),
                                dict(cache=cache(k_exp=BASE + 1000 * MB)), dict(slots=BASE + 1400 * MB)])
def test_write_overlap(dry, kw):
    assert rope4(dry, **kw) == L.QKN_EOVERLAP


@pytest.mark.parametrize("kw,kernel", [
    (dict(), "rope<8>/fp4"), (dict(rot=64), "rope<8>/fp4"), (dict(rot=32), "rope4/elements"), (dict(rot=32, inter=1), "rope<8>/fp4"),
    (dict(rot=16, inter=1), "rope4/elements"), (dict(rot=0, table=None, pos=None), "rope<8>/fp4"),
    (dict(D=32), "rope4/elements"), (dict(D=32, inter=1), "rope<8>/fp4"), (dict(D=96, rot=64), "rope4/elements"),
    (dict(ldv=257), "rope4/elements"), (dict(cache=cache(v_token=65, v_head=1040, v_page=2080)), "rope4/elements"),
    (dict(cache=cache(ke_token=5, ke_head=80, ke_page=161)), "rope<8>/fp4"),
])
def test_write_paths(dry, kw, kernel):
    assert rope4(dry, **kw) == DRY
    assert L.qkn_last_launch()["kernel"] == kernel


def test_writes_of_2_32_threads_are_refused(dry):
    """As QKN_ENOTSUP before anything is written: half a wavefront takes 32 elements, and a wavefront a token's rows."""
    far = dict(q=None, v=None, ldv=0, table=1 << 50, pos=1 << 51, slots=1 << 52, tp=1, rot=32)
    k = dict(x=1 << 40, w=None, partials=None, d_full=0)
    for T, want in (((1 << 24) - 1, DRY), (1 << 24, L.QKN_ENOTSUP)):  # 8 blocks a token, 8 to a workgroup
        assert rope4(dry, T=T, k=seg(300, 2, y=None, **k), **far) == want
        if want == DRY:
            assert L.qkn_last_launch()["kernel"] == "rope4/elements"
    # one block a token, and rows besides: the second launch's limit, found before the first
    k.update(x=1 << 40, ldx=32)
    c = cache(32, n_kv=1)
    far.update(D=32, cache=c)
    most = 4 * ((1 << 24) - 1)
    for T, want in ((most, DRY), (most + 1, L.QKN_ENOTSUP)):
        assert rope4(dry, T=T, k=seg(300, 1, 32, y=1 << 45, **k), **far) == want
    # rows that are not written need no second launch
    for T, want in ((2 * most, DRY), (2 * most + 8, L.QKN_ENOTSUP)):
        assert rope4(dry, T=T, k=seg(300, 1, 32, y=None, **k), **far) == want


def test_reading_back(dry):
    assert load4(dry, k=None, v=None) == L.QKN_EINVAL
    assert load4(dry, slots=None) == L.QKN_EINVAL and load4(dry, T=-1) == L.QKN_EINVAL
    assert load4(dry, ldk=255) == L.QKN_EINVAL and load4(dry, ldv=0) == L.QKN_EINVAL
    assert dry.qkn_cache4_load(None, BASE, 4, BASE + MB, 256, None, 0, None) == L.QKN_EINVAL
    assert load4(dry, T=1 << 27) == L.QKN_ENOTSUP
    for kw in (dict(k=BASE), dict(k=BASE + 1000 * MB), dict(v=BASE + 1500 * MB), dict(v=BASE + 100 * MB)):
        assert load4(dry, **kw) == L.QKN_EOVERLAP
    assert load4(dry) == DRY and L.qkn_last_launch()["kernel"] == "cache4_load<8>"
    for kw in (dict(ldk=257), dict(k=BASE + 100 * MB + 2), dict(c=cache(k_token=65, k_head=1040, k_page=2080))):
        assert load4(dry, **kw) == DRY and L.qkn_last_launch()["kernel"] == "cache4_load<1>"


def test_struct_layout_matches_header(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    lines = ['printf("qkn_cache4 %zu\\n", sizeof(qkn_cache4));']
    lines += [f'printf("{f} %zu\\n", offsetof(qkn_cache4, {f}));' for f, _ in S.QknCache4._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "qkn_cache4.h"\nint main(void) {'
                   + "\n".join(lines) + "return 0; }")
    subprocess.run(["gcc", "-std=c99", "-I", INCLUDE, str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines():
        name, value = line.split()
        want = ctypes.sizeof(S.QknCache4) if name == "qkn_cache4" else getattr(S.QknCache4, name).offset
        assert int(value) == want, name


def test_bindings_checks():
    c = S.KVCache4.empty(2, 1, 16, 64, device="cpu")
    assert [tuple(t.shape) for t in (c.k, c.v, c.k_exp, c.v_exp)] == [(2, 1, 16, 32)] * 2 + [(2, 1, 16, 2)] * 2
    assert c.head_dim == 64
    with pytest.raises(ValueError):
        c.struct()  # not on a GPU
    with pytest.raises(TypeError):
        S.KVCache4(c.k.to(torch.int8), c.v, c.k_exp, c.v_exp).struct()
    for bad in (dict(v=c.v[:1]), dict(k_exp=c.k_exp[..., :1]), dict(k=c.k[0]), dict(v_exp=c.v_exp[:, :, :8])):
        pools = dict(k=c.k, v=c.v, k_exp=c.k_exp, v_exp=c.v_exp)
        pools.update(bad)
        with pytest.raises(ValueError):
            S.KVCache4(**pools).struct()


@pytest.mark.parametrize("sinks", [-1, 2 ** 31, 2 ** 32])
def test_first_tokens_that_no_32_bits_hold(sinks, monkeypatch):
    """Refused, not taken modulo 2^32."""
    monkeypatch.setattr(S, "_rows", lambda t, what, *a: (BASE, 128, t.shape[0], t.shape[1]))
    monkeypatch.setattr(S, "_index", lambda t, what, dtype, n: BASE)
    monkeypatch.setattr(S.KVCache4, "struct", lambda self: cache(64))
    ints = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="sinks"):
        S.PreparedAttn(torch.empty(1, 128), S.KVCache4.empty(1, 2, 16, 64, device="cpu"), ints.view(1, 2), ints, ints[:1],
                       window=4, sinks=sinks, out=torch.empty(1, 128))
