"""The rotary pass's C ABI without a GPU: struct layout, refusals, overlap rules, path choice. Pointers are fake
addresses that nothing dereferences ("validate_only" is set, or the call is refused)."""
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


def seg(at, heads, **kw):
    base = dict(x=BASE + at * MB, ldx=heads * 128, w=BASE + (at + 100) * MB, partials=BASE + (at + 110) * MB,
                d_full=heads * 256, y=BASE + (at + 120) * MB, ldy=heads * 128, heads=heads)
    base.update(kw)
    return S.QknRopeSeg(**base)


def cache(**kw):
    base = dict(k=BASE + 1000 * MB, v=BASE + 1200 * MB, num_pages=64, page_size=16, n_kv=2, head_dim=128, fp8=0,
                k_page=4096, k_head=2048, k_token=128, v_page=4096, v_head=2048, v_token=128)
    base.update(kw)
    return S.QknCache(**base)


def call(lib, **kw):
    a = dict(q=seg(0, 8), k=seg(300, 2), v=BASE + 600 * MB, ldv=256, T=64, D=128, rot=128, inter=0,
             table=BASE + 700 * MB, n_pos=4096, pos=BASE + 800 * MB, slots=BASE + 810 * MB, cache=cache(), tp=2,
             eps=1e-6)
    a.update(kw)
    ref = [ctypes.byref(a[n]) if a[n] is not None else None for n in ("q", "k", "cache")]
    return lib.qkn_rope_cache(ref[0], ref[1], a["v"], a["ldv"], a["T"], a["D"], a["rot"], a["inter"], a["table"],
                              a["n_pos"], a["pos"], a["slots"], ref[2], a["tp"], ctypes.c_float(a["eps"]), None)


def test_accepted(dry):
    assert call(dry) == DRY
    assert L.qkn_last_launch()["kernel"] == "rope<8>/bf16"
    assert call(dry, T=0) == L.QKN_OK
    assert call(dry, T=0, table=None, pos=None, slots=None, v=None) == L.QKN_OK
    assert call(dry, q=None) == DRY
    assert call(dry, k=None, v=None, cache=None) == DRY
    assert call(dry, k=seg(300, 2, y=None)) == DRY
    assert call(dry, rot=0, table=None, pos=None) == DRY
    assert call(dry, q=seg(0, 8, w=None, partials=None, d_full=0)) == DRY
    assert call(dry, k=None) == DRY  # V alone into the cache


@pytest.mark.parametrize("kw,name", [
    (dict(D=128, rot=24), "rope<1>/bf16"),
    (dict(q=seg(0, 8, x=BASE + 2)), "rope<1>/bf16"),
    (dict(q=seg(0, 8, ldy=1028)), "rope<1>/bf16"),
    (dict(v=BASE + 600 * MB + 8), "rope<1>/bf16"),
    (dict(cache=cache(k_token=132, k_head=2112, k_page=4224)), "rope<1>/bf16"),
    (dict(cache=cache(fp8=1, k=BASE + 1000 * MB + 8)), "rope<8>/fp8"),
    (dict(cache=cache(fp8=1, k=BASE + 1000 * MB + 4)), "rope<1>/fp8"),
])
def test_path(dry, kw, name):
    assert call(dry, **kw) == DRY
    assert L.qkn_last_launch()["kernel"] == name


@pytest.mark.parametrize("kw", [
    dict(q=None, k=None), dict(T=-1), dict(D=0), dict(rot=127), dict(rot=-2), dict(rot=130), dict(tp=0),
    dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")), dict(cache=None), dict(table=None), dict(pos=None),
    dict(slots=None), dict(n_pos=-1), dict(ldv=255),
    dict(q=seg(0, 8, x=None)), dict(q=seg(0, 8, y=None)), dict(q=seg(0, 8, partials=None)), dict(q=seg(0, 0)),
    dict(q=seg(0, 8, ldx=1023)), dict(q=seg(0, 8, ldy=1023)), dict(q=seg(0, 8, d_full=1023)),
    dict(k=seg(300, 1)), dict(k=seg(300, 2, y=None), v=None, cache=None), dict(k=None, v=None),
    dict(cache=cache(head_dim=64)), dict(cache=cache(page_size=0)), dict(cache=cache(page_size=24)),
    dict(cache=cache(page_size=1 << 17)), dict(cache=cache(num_pages=-1)), dict(cache=cache(n_kv=0)),
    dict(cache=cache(k_token=127)), dict(cache=cache(v_page=0)), dict(cache=cache(k=None)), dict(cache=cache(v=None)),
    dict(cache=cache(k_scale=BASE)),  # a bf16 cache has no scale
])
def test_refused(dry, kw):
    assert call(dry, **kw) == L.QKN_EINVAL


def test_size_limits(dry):
    wide = (1 << 23) + 1
    assert call(dry, q=seg(0, wide, ldx=wide * 128, ldy=wide * 128, w=None)) == L.QKN_ENOTSUP
    assert call(dry, T=1 << 31, q=seg(0, 8, w=None, x=1 << 20, y=1 << 46), k=None, v=None, cache=None, table=1 << 50,
                pos=1 << 51) == L.QKN_ENOTSUP


def test_launches_of_2_32_threads_are_refused(dry):
    """As QKN_ENOTSUP by the validation, not as QKN_EHIP by the launch: four wavefronts a workgroup, one a token."""
    most = 4 * ((1 << 24) - 1)
    for T, want in ((most, DRY), (most + 1, L.QKN_ENOTSUP)):
        q = seg(0, 8, w=None, partials=None, d_full=0, x=1 << 40, y=1 << 42)
        assert call(dry, T=T, q=q, k=None, v=None, cache=None, table=1 << 50, pos=1 << 51) == want


@pytest.mark.parametrize("kw", [
    dict(q=seg(0, 8, y=BASE + 2)),                     # y one element into x
    dict(q=seg(0, 8, y=BASE + 300 * MB)),              # Q's output on K's input
    dict(q=seg(0, 8, y=BASE + 420 * MB)),              # both outputs
    dict(q=seg(0, 8, w=BASE + 420 * MB)),              # an output on gamma
    dict(pos=BASE + 120 * MB), dict(table=BASE + 120 * MB), dict(slots=BASE + 120 * MB), dict(v=BASE + 120 * MB),
    dict(cache=cache(k=BASE)), dict(cache=cache(v=BASE + 300 * MB)), dict(cache=cache(v=BASE + 1000 * MB)),
    dict(cache=cache(fp8=1, v_scale=BASE + 1000 * MB)),
])
def test_overlap(dry, kw):
    assert call(dry, **kw) == L.QKN_EOVERLAP


def test_in_place_and_interleaved_pools_are_not_overlaps(dry):
    assert call(dry, q=seg(0, 8, y=BASE)) == DRY
    assert call(dry, cache=cache(v=BASE + 1000 * MB + 8192, k_page=8192, v_page=8192)) == DRY


def test_table_validation(dry):
    def table(n=16, rot=64, out=BASE, **kw):
        sc = S.QknRopeScaling(*{**dict(base=1e4, factor=1.0, low=0.0, high=0.0, original=0.0, magnitude=1.0), **kw}.values())
        return dry.qkn_rope_table(out, n, rot, ctypes.byref(sc), None)
    assert table() == DRY and table(n=0, out=None) == L.QKN_OK
    assert table(factor=4.0, low=1.0, high=32.0, original=4096.0) == DRY
    assert dry.qkn_rope_table(BASE, 16, 64, None, None) == L.QKN_EINVAL
    for bad in (dict(n=-1), dict(rot=63), dict(rot=0), dict(out=None), dict(base=0.0), dict(base=float("nan")),
                dict(factor=0.5), dict(low=2.0, high=1.0, original=8.0), dict(low=-1.0, high=1.0, original=8.0),
                dict(low=1.0, high=2.0), dict(magnitude=float("inf"))):
        assert table(**bad) == L.QKN_EINVAL, bad


def test_struct_layouts_match_header(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    classes = {"qkn_cache": S.QknCache, "qkn_rope_seg": S.QknRopeSeg, "qkn_rope_scaling": S.QknRopeScaling}
    lines = []
    for name, cls in classes.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "qkn_rope.h"\nint main(void) {'
                   + "\n".join(lines) + "return 0; }")
    subprocess.run(["gcc", "-std=c99", "-I", INCLUDE, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    for line in out.splitlines():
        name, value = line.split()
        cls, _, field = name.partition(".")
        want = getattr(classes[cls], field).offset if field else ctypes.sizeof(classes[cls])
        assert int(value) == want, name


def test_empty_pools_are_not_an_overlap(dry):
    """A cache without pages has no pool to overlap: both may be NULL, as empty tensors are, or one address."""
    assert call(dry, cache=cache(num_pages=0, k=None, v=None)) == DRY
    assert call(dry, cache=cache(num_pages=0, k=BASE + 1000 * MB, v=BASE + 1000 * MB)) == DRY
    assert call(dry, cache=cache(num_pages=0, k=None, v=None, fp8=1), k=seg(300, 2, y=None)) == DRY
