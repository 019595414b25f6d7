"""The adapters' C ABI without a GPU: struct layout, refusals, overlap rules, workspace."""
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


def seg(at=0, **kw):
    base = dict(a=BASE + (at + 1000) * MB, a_adapter=16 * 512, lda=512, b=BASE + (at + 1100) * MB, b_adapter=128 * 16,
                ldb=16, base=BASE + (at + 1200) * MB, ldbase=128, y=BASE + (at + 1300) * MB, ldy=128,
                partials=BASE + (at + 1400) * MB, d_local=128)
    base.update(kw)
    return S.QknAdapterSeg(**base)


def call(lib, segs=None, **kw):
    a = dict(x=BASE, ldx=512, T=64, hidden=512, nseg=None, rank=16, count=4, ids=BASE + 100 * MB,
             scale=BASE + 110 * MB, ws=BASE + 200 * MB, ws_bytes=100 * MB)
    a.update(kw)
    segs = [seg()] if segs is None else segs
    arr = (S.QknAdapterSeg * max(1, len(segs)))(*segs)
    nseg = len(segs) if a["nseg"] is None else a["nseg"]
    return lib.qkn_adapters_add(a["x"], a["ldx"], a["T"], a["hidden"], arr, nseg, a["rank"], a["count"], a["ids"],
                                a["scale"], a["ws"], a["ws_bytes"], None)


def test_accepted(dry):
    assert call(dry) == DRY and L.qkn_last_launch()["kernel"] == "adapters<gather>"
    assert call(dry, T=513) == DRY and L.qkn_last_launch()["kernel"] == "adapters<tiles>"
    assert call(dry, [seg(), seg(1000), seg(2000)]) == DRY
    assert call(dry, [seg(partials=None)], scale=None) == DRY
    assert call(dry, [seg(base=BASE + 1300 * MB)]) == DRY  # in place
    assert call(dry, [seg(a=None, b=None)], count=0, scale=None) == DRY
    assert call(dry, [seg(a_adapter=0, b_adapter=0)]) == DRY  # one matrix for all
    assert call(dry, T=0, x=None, ids=None, ws=None, ws_bytes=0) == L.QKN_OK


def test_workspace(dry):
    need = dry.qkn_adapters_workspace_bytes(64, 512, 16, 1)
    assert need == 2 * 64 * 16 * 4  # two parts of 256
    assert call(dry, ws_bytes=need) == DRY and call(dry, ws_bytes=need - 1) == L.QKN_EINVAL
    assert call(dry, ws=None) == L.QKN_EINVAL and call(dry, ws=BASE + 200 * MB + 4) == L.QKN_ENOTSUP
    assert dry.qkn_adapters_workspace_bytes(0, 512, 16, 1) == 0
    for bad in ((-1, 512, 16, 1), (1, 0, 16, 1), (1, 512, 0, 1), (1, 512, 16, 0), (1, 512, 16, 4)):
        assert dry.qkn_adapters_workspace_bytes(*bad) == L.QKN_EINVAL


@pytest.mark.parametrize("kw", [dict(x=None), dict(ids=None), dict(T=-1), dict(hidden=0), dict(rank=0), dict(nseg=0),
                                dict(nseg=4), dict(count=-1), dict(ldx=511)])
def test_refused(dry, kw):
    assert call(dry, **kw) == L.QKN_EINVAL


@pytest.mark.parametrize("kw", [dict(a=None), dict(b=None), dict(base=None), dict(y=None), dict(d_local=0),
                                dict(lda=504), dict(ldb=8), dict(ldbase=120), dict(ldy=120), dict(a_adapter=-8),
                                dict(b_adapter=-8)])
def test_refused_segments(dry, kw):
    assert call(dry, [seg(**kw)]) == L.QKN_EINVAL


@pytest.mark.parametrize("s,kw", [
    ({}, dict(x=BASE + 8)), ({}, dict(ldx=516)), ({}, dict(hidden=508)), ({}, dict(rank=12)), (dict(ldb=136), dict(rank=136)),
    (dict(ldbase=132), {}), (dict(ldy=132), {}), (dict(y=BASE + 1300 * MB + 8), {}), (dict(base=BASE + 2), {}),
    (dict(a=BASE + 1000 * MB + 8), {}), (dict(b=BASE + 1100 * MB + 8), {}), (dict(lda=516), {}), (dict(ldb=20), {}),
    (dict(a_adapter=8196), {}), (dict(b_adapter=2052), {}), (dict(d_local=124), {}), ({}, dict(T=(1 << 24) + 1)),
])
def test_not_supported(dry, s, kw):
    assert call(dry, [seg(**s)], **kw) == L.QKN_ENOTSUP


@pytest.mark.parametrize("s,kw", [
    (dict(y=BASE), {}), (dict(y=BASE + 1200 * MB + 16), {}), (dict(y=BASE + 1200 * MB, ldy=136), {}),
    (dict(y=BASE + 1000 * MB), {}), (dict(y=BASE + 1100 * MB), {}), (dict(partials=BASE + 1300 * MB), {}),
    (dict(partials=BASE + 100 * MB), {}), ({}, dict(ws=BASE + 1300 * MB)), ({}, dict(ws=BASE)),
    ({}, dict(scale=BASE + 1400 * MB)),
])
def test_overlap(dry, s, kw):
    assert call(dry, [seg(**s)], **kw) == L.QKN_EOVERLAP


def test_outputs_of_two_segments_overlap(dry):
    assert call(dry, [seg(), seg(1000, y=BASE + 1300 * MB)]) == L.QKN_EOVERLAP


def test_struct_layout_matches_header(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    lines = ['printf("qkn_adapter_seg %zu\\n", sizeof(qkn_adapter_seg));']
    lines += [f'printf("{f} %zu\\n", offsetof(qkn_adapter_seg, {f}));' for f, _ in S.QknAdapterSeg._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "qkn_adapters.h"\nint main(void) {'
                   + "\n".join(lines) + "return 0; }")
    subprocess.run(["gcc", "-std=c99", "-I", INCLUDE, str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines():
        name, value = line.split()
        want = ctypes.sizeof(S.QknAdapterSeg) if name == "qkn_adapter_seg" else getattr(S.QknAdapterSeg, name).offset
        assert int(value) == want, name
