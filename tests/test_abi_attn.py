"""The paged attention's C ABI without a GPU: struct layout, refusals, overlap rules, kernel choice, workspace."""
import ctypes
import os
import shutil
import subprocess

import pytest

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


def args(**kw):
    base = dict(q=BASE, ldq=1024, out=BASE + 100 * MB, ldo=1024, lse=BASE + 200 * MB, q_start=BASE + 210 * MB,
                kv_len=BASE + 220 * MB, block_table=BASE + 230 * MB, ld_table=256, T=64, batch=64, n_q=8, max_q=1,
                max_kv=4096, causal=1, window=0, scale=0.1)
    base.update(kw)
    return S.QknAttnArgs(**base)


def cache(**kw):
    base = dict(k=BASE + 1000 * MB, v=BASE + 2000 * MB, num_pages=4096, page_size=16, n_kv=2, head_dim=128, fp8=0,
                k_page=4096, k_head=2048, k_token=128, v_page=4096, v_head=2048, v_token=128)
    base.update(kw)
    return S.QknCache(**base)


def call(lib, a=None, c=None, ws=BASE + 4000 * MB, ws_bytes=1 << 32):
    a, c = args() if a is None else a, cache() if c is None else c
    return lib.qkn_attn(ctypes.byref(a), ctypes.byref(c), ws, ws_bytes, None)


def need(lib, a=None, c=None):
    a, c = args() if a is None else a, cache() if c is None else c
    return lib.qkn_attn_workspace_bytes(ctypes.byref(a), ctypes.byref(c))


def test_accepted(dry):
    assert call(dry) == DRY
    assert call(dry, args(lse=None)) == DRY
    assert call(dry, args(window=100)) == DRY
    assert call(dry, args(T=0)) == L.QKN_OK
    assert call(dry, args(T=0, batch=0, q=None, out=None, q_start=None, kv_len=None, block_table=None)) == L.QKN_OK
    assert call(dry, args(ld_table=0, block_table=None)) == DRY
    assert call(dry, c=cache(num_pages=0, k=None, v=None)) == DRY


@pytest.mark.parametrize("max_q,n_q,D,fp8,name", [
    (1, 8, 128, 0, "attn<128,16>/bf16"), (1, 32, 128, 0, "attn<128,16>/bf16"), (1, 34, 128, 0, "attn<128,32>/bf16"),
    (5, 8, 128, 1, "attn<128,32>/fp8"), (16, 8, 128, 1, "attn<128,64>/fp8"), (17, 8, 128, 1, "attn<128,64,shared>/fp8"),
    (4096, 8, 128, 0, "attn<128,128,shared>/bf16"),
    (1, 8, 64, 0, "attn<64,16>/bf16"), (1, 8, 8, 0, "attn<64,16>/bf16"), (1, 8, 72, 0, "attn<128,16>/bf16"),
    (9, 8, 256, 0, "attn<256,64,shared>/bf16"), (0, 8, 256, 0, "attn<256,16>/bf16"),
])
def test_kernel_choice(dry, max_q, n_q, D, fp8, name):
    a = args(max_q=max_q, n_q=n_q, ldq=n_q * D, ldo=n_q * D, T=max(64, max_q), max_kv=4096 + max_q)
    c = cache(head_dim=D, fp8=fp8, k_token=D, v_token=D, k_head=16 * D, v_head=16 * D, k_page=32 * D, v_page=32 * D)
    assert call(dry, a, c) == DRY
    assert L.qkn_last_launch()["kernel"] == name


def test_workspace(dry):
    n = need(dry)
    # a part of every workgroup that the chip holds (two a CU, 16 rows each), and where each row's parts are
    assert n == 512 * 16 * (4 * 128 + 8) + 64 * 8 * 8
    assert call(dry, ws_bytes=n) == DRY
    assert call(dry, ws_bytes=n - 1) == L.QKN_EINVAL
    assert call(dry, ws=None) == L.QKN_EINVAL
    assert call(dry, ws=BASE + 4000 * MB + 8) == L.QKN_ENOTSUP
    assert need(dry, args(max_kv=16)) == 0  # nothing to split
    assert call(dry, args(max_kv=16), ws=None, ws_bytes=0) == DRY
    assert need(dry, args(T=0)) == 0
    assert need(dry, args(n_q=7)) == L.QKN_EINVAL
    assert need(dry, c=cache(page_size=8)) == L.QKN_ENOTSUP


@pytest.mark.parametrize("kw", [
    dict(T=-1), dict(batch=-1), dict(max_q=-1), dict(max_kv=-1), dict(n_q=0), dict(n_q=7), dict(ldq=1016), dict(ldo=1016),
    dict(ld_table=-1), dict(window=-1), dict(causal=0, window=4), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=float("inf")), dict(scale=float("nan")), dict(q=None), dict(out=None), dict(q_start=None),
    dict(kv_len=None), dict(block_table=None),
])
def test_refused_arguments(dry, kw):
    assert call(dry, args(**kw)) == L.QKN_EINVAL


@pytest.mark.parametrize("kw", [
    dict(k=None), dict(v=None), dict(page_size=24), dict(n_kv=0), dict(n_kv=3), dict(head_dim=0), dict(k_token=64),
    dict(num_pages=-1), dict(v_scale=BASE),
])
def test_refused_caches(dry, kw):
    assert call(dry, c=cache(**kw)) == L.QKN_EINVAL


def test_null_structs(dry):
    c = cache()
    assert dry.qkn_attn(None, ctypes.byref(c), None, 0, None) == L.QKN_EINVAL
    assert dry.qkn_attn(ctypes.byref(args()), None, None, 0, None) == L.QKN_EINVAL
    assert dry.qkn_attn_workspace_bytes(None, ctypes.byref(c)) == L.QKN_EINVAL


@pytest.mark.parametrize("a,c", [
    (dict(q=BASE + 8), {}), (dict(out=BASE + 100 * MB + 2), {}), (dict(ldq=1028), {}), (dict(ldo=1028), {}),
    ({}, dict(page_size=8)), ({}, dict(k=BASE + 1000 * MB + 8)), ({}, dict(k_page=4100)), ({}, dict(v_token=132)),
    ({}, dict(fp8=1, k_head=2056)), (dict(n_q=2, ldq=520, ldo=520), dict(head_dim=260, k_token=260, v_token=260)),
    (dict(n_q=2), dict(head_dim=12)), (dict(n_q=2), dict(head_dim=24, fp8=1)), (dict(T=1 << 28), {}),
    (dict(ld_table=1 << 27), {}), ({}, dict(k_token=1 << 27)),
])
def test_not_supported(dry, a, c):
    assert call(dry, args(**a), cache(**c)) == L.QKN_ENOTSUP


@pytest.mark.parametrize("a,c", [
    (dict(out=BASE), {}), (dict(out=BASE + 1000 * MB), {}), (dict(out=BASE + 210 * MB), {}), (dict(lse=BASE), {}),
    (dict(lse=BASE + 100 * MB), {}), (dict(lse=BASE + 4000 * MB), {}), (dict(block_table=BASE + 100 * MB), {}),
    (dict(kv_len=BASE + 200 * MB), {}), ({}, dict(v=BASE + 4000 * MB)),
    ({}, dict(fp8=1, k_scale=BASE + 100 * MB)),
])
def test_overlap(dry, a, c):
    assert call(dry, args(**a), cache(**c)) == L.QKN_EOVERLAP


def test_pools_may_share_an_allocation(dry):
    assert call(dry, c=cache(v=BASE + 1000 * MB + 8192, k_page=8192, v_page=8192)) == DRY


def test_struct_layout_matches_header(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    lines = ['printf("qkn_attn_args %zu\\n", sizeof(qkn_attn_args));']
    lines += [f'printf("{f} %zu\\n", offsetof(qkn_attn_args, {f}));' for f, _ in S.QknAttnArgs._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "qkn_attn.h"\nint main(void) {'
                   + "\n".join(lines) + "return 0; }")
    subprocess.run(["gcc", "-std=c99", "-I", INCLUDE, str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines():
        name, value = line.split()
        want = ctypes.sizeof(S.QknAttnArgs) if name == "qkn_attn_args" else getattr(S.QknAttnArgs, name).offset
        assert int(value) == want, name


@pytest.mark.parametrize("T,batch,n_q,D,max_q,max_kv", [
    (1024, 1, 16, 128, 1024, 16384), (777, 1, 16, 128, 777, 12001), (300, 4, 16, 64, 200, 30000), (64, 64, 16, 128, 1, 4096),
    (90, 3, 16, 256, 60, 9000),
])
def test_one_workspace_serves_every_window(dry, T, batch, n_q, D, max_q, max_kv):
    """Layers of one model differ in window and mask: the size depends on neither, and is enough for all."""
    c = cache(n_kv=4, head_dim=D, k_token=D, v_token=D, k_head=16 * D, v_head=16 * D, k_page=64 * D, v_page=64 * D)
    sizes = dict(T=T, batch=batch, n_q=n_q, ldq=n_q * D, ldo=n_q * D, max_q=max_q, max_kv=max_kv)
    layers = [dict(causal=1, window=w) for w in (0, 1, 128, 1024, 1 << 30)] + [dict(causal=0)]
    bytes_of = {need(dry, args(**sizes, **layer), c) for layer in layers}
    assert len(bytes_of) == 1
    for layer in layers:
        assert call(dry, args(**sizes, **layer), c, ws_bytes=bytes_of.copy().pop()) == DRY


def test_pools_beyond_the_address_space(dry):
    """Page strides whose extent no address space has: the extent is the overlap test's, and must not wrap around."""
    wide = dict(k_page=1 << 40, v_page=1 << 40)
    assert call(dry, c=cache(num_pages=(1 << 24) + 1, **wide)) == L.QKN_EINVAL
    assert call(dry, c=cache(num_pages=1 << 31, k_page=1 << 40)) == L.QKN_EINVAL
    assert call(dry, c=cache(num_pages=1 << 31, v_page=1 << 40)) == L.QKN_EINVAL
    assert call(dry, c=cache(num_pages=1, **wide)) == DRY  # the stride of one page is not used
    far = cache(num_pages=33, k_page=1 << 28, v_page=1 << 28, v=BASE + (1 << 40))  # 16 GiB of k, read up to its last page
    assert call(dry, args(out=BASE + 1000 * MB + (1 << 33)), far) == L.QKN_EOVERLAP
