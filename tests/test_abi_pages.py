"""The C ABI of the book of pages without a GPU: struct layout, refusals, overlap rules, the copies' vectors. Pointers are
fake addresses that nothing dereferences ("validate_only" is set, or the call is refused)."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2608_09160_amd import _lib as L
from paper_2608_09160_amd import _pages as P
from paper_2608_09160_amd import _serve as S

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
BASE, MB = 0x7f0000000000, 1 << 20
DRY = L.QKN_EDRYRUN


@pytest.fixture
def dry():
    lib = P.load()
    assert lib.qkn_set_option(b"validate_only", 1) == 0
    yield lib
    assert lib.qkn_set_option(b"validate_only", 0) == 0


def book(at=0, **kw):
    base = dict(refs=BASE + at * MB, table=BASE + (at + 10) * MB, kv_len=BASE + (at + 20) * MB, num_pages=4096, ld_table=64,
                rows=128, page_size=16)
    base.update(kw)
    return P.QknPages(**base)


def calls(lib, b, n=8, T=8, which=BASE + 100 * MB, a=BASE + 110 * MB, s=BASE + 120 * MB, d=BASE + 130 * MB, done=BASE + 140 * MB,
          ws=BASE + 150 * MB, ws_bytes=1 << 20, out=None):
    """Statuses of grow, fork, free, compact."""
    p = ctypes.byref(b) if b is not None else None
    o = ctypes.byref(out) if out is not None else None
    return (lib.qkn_pages_grow(p, which, a, n, T, s, d, done, None), lib.qkn_pages_fork(p, a, which, n, s, d, done, None),
            lib.qkn_pages_free(p, which, n, None), lib.qkn_pages_compact(p, o, s, d, n, ws, ws_bytes, None))


def test_accepted(dry):
    assert calls(dry, book()) == (DRY,) * 4
    assert calls(dry, book(), out=book(200)) == (DRY,) * 4
    p = ctypes.byref(book())
    assert dry.qkn_pages_grow(p, None, BASE + 110 * MB, 8, 0, None, None, BASE + 140 * MB, None) == DRY
    assert dry.qkn_pages_free(p, None, 8, None) == DRY
    assert calls(dry, book(), n=0, T=0)[:3] == (L.QKN_OK,) * 3
    # in place in part: the book's refs, another table
    assert calls(dry, book(), out=book(table=BASE + 300 * MB))[3] == DRY


@pytest.mark.parametrize("kw", [dict(num_pages=-1), dict(num_pages=(1 << 24) + 1), dict(rows=-1), dict(ld_table=-1), dict(page_size=0),
                                dict(page_size=24), dict(page_size=1 << 17), dict(ld_table=1 << 27), dict(refs=None), dict(table=None),
                                dict(kv_len=None)])
def test_malformed_books(dry, kw):
    assert calls(dry, book(**kw)) == (L.QKN_EINVAL,) * 4
    assert calls(dry, None) == (L.QKN_EINVAL,) * 4
    sizes = {k: v for k, v in kw.items() if k not in ("refs", "table", "kv_len")}
    assert (dry.qkn_pages_compact_workspace_bytes(ctypes.byref(book(**kw))) < 0) == bool(sizes)


def test_refusals(dry):
    e = L.QKN_EINVAL
    assert calls(dry, book(), n=-1) == (e,) * 4
    assert calls(dry, book(), n=1025)[:3] == (L.QKN_ENOTSUP,) * 3 and calls(dry, book(), n=1025)[3] == DRY
    assert calls(dry, book(), n=(1 << 24) + 1)[3] == L.QKN_ENOTSUP
    p = ctypes.byref(book())
    g = [BASE + 100 * MB, BASE + 110 * MB, 8, 8, BASE + 120 * MB, BASE + 130 * MB, BASE + 140 * MB, None]
    for i, v, rc in ((1, None, e), (6, None, e), (3, -1, e), (3, 1 << 31, L.QKN_ENOTSUP)):
        assert dry.qkn_pages_grow(p, *[v if k == i else x for k, x in enumerate(g)]) == rc
    f = [BASE + 100 * MB, BASE + 110 * MB, 8, BASE + 120 * MB, BASE + 130 * MB, BASE + 140 * MB, None]
    for i in (0, 1, 3, 4, 5):
        assert dry.qkn_pages_fork(p, *[None if k == i else x for k, x in enumerate(f)]) == e
    assert calls(dry, book(), s=None)[3] == e and calls(dry, book(), d=None)[3] == e
    for other in (dict(num_pages=4095), dict(rows=127), dict(ld_table=63), dict(page_size=32), dict(refs=None), dict(table=None)):
        assert calls(dry, book(), out=book(200, **other))[3] == e
    need = dry.qkn_pages_compact_workspace_bytes(p)
    assert need == 4 * (4096 + 1 + 1) and calls(dry, book(), ws_bytes=need)[3] == DRY
    assert calls(dry, book(), ws_bytes=need - 1)[3] == e and calls(dry, book(), ws=None)[3] == e
    assert calls(dry, book(), ws=BASE + 150 * MB + 4)[3] == L.QKN_ENOTSUP


def test_moves_of_2_32_threads_are_refused(dry):
    """As QKN_ENOTSUP, before a list of moves is written that no launch then carries out: a thread a page and a table entry."""
    far = dict(refs=1 << 40, table=1 << 41, kv_len=1 << 50, num_pages=256, page_size=1, rows=(1 << 16) - 1)
    for ld, want in ((1 << 16, DRY), ((1 << 16) + 1, L.QKN_ENOTSUP), (1 << 30, L.QKN_ENOTSUP)):
        assert (256 + ld * far["rows"] < 1 << 32) == (want == DRY)
        assert calls(dry, book(ld_table=ld, **far))[3] == want


def test_overlap(dry):
    o = L.QKN_EOVERLAP
    for at in (0, 10, 20):  # the book's arrays
        here = BASE + at * MB
        assert calls(dry, book(), which=here)[:3] == (o,) * 3
        assert calls(dry, book(), s=here) == (o, o, DRY, o)
        assert calls(dry, book(), d=here) == (o, o, DRY, o)
        assert calls(dry, book(), ws=here)[3] == o
    assert calls(dry, book(), s=BASE + 130 * MB)[0::3] == (o, o)
    assert calls(dry, book(), done=BASE + 110 * MB)[:2] == (o, o)
    assert calls(dry, book(table=BASE + 64)) == (o,) * 4
    assert calls(dry, book(), out=book(200, table=BASE))[3] == o  # the table over the book's refs
    assert calls(dry, book(), out=book(200, refs=BASE + 4))[3] == o


def cache(**kw):
    base = dict(k=BASE + 1000 * MB, v=BASE + 2000 * MB, num_pages=64, page_size=16, n_kv=2, head_dim=128, fp8=0,
                k_page=4096, k_head=2048, k_token=128, v_page=4096, v_head=2048, v_token=128)
    base.update(kw)
    return S.QknCache(**base)


def copy(lib, *caches, n=8, src=BASE, dst=BASE + MB):
    arr = (S.QknCache * len(caches))(*caches)
    return lib.qkn_pages_copy(arr, len(caches), src, dst, n, None)


def test_copies(dry):
    assert copy(dry, cache()) == DRY and L.qkn_last_launch()["kernel"] == "pages_copy<16>"
    assert copy(dry, cache(), n=0) == L.QKN_OK and copy(dry) == L.QKN_OK
    assert copy(dry, *[cache() for _ in range(50)]) == DRY
    for kw, unit in ((dict(head_dim=20, k_token=20, v_token=20, k_head=320, v_head=320), 16), (dict(k=BASE + 1000 * MB + 4), 4),
                     (dict(k_page=4098), 4), (dict(v_token=129, v_head=2064, v_page=4128), 2),
                     (dict(fp8=1, v=BASE + 2000 * MB + 1), 1)):
        assert copy(dry, cache(**kw)) == DRY
        assert L.qkn_last_launch()["kernel"] == f"pages_copy<{unit}>", kw
    e, o = L.QKN_EINVAL, L.QKN_EOVERLAP
    assert copy(dry, cache(), n=-1) == e and copy(dry, cache(), src=None) == e and copy(dry, cache(), dst=None) == e
    assert copy(dry, cache(k=None)) == e and copy(dry, cache(v=None)) == e and copy(dry, cache(), cache(page_size=3)) == e
    assert copy(dry, cache(num_pages=0, k=None, v=None)) == L.QKN_OK
    assert dry.qkn_pages_copy(None, 1, BASE, BASE + MB, 8, None) == e and dry.qkn_pages_copy(None, -1, BASE, BASE + MB, 8, None) == e
    assert copy(dry, cache(), n=(1 << 24) + 1) == L.QKN_ENOTSUP
    assert copy(dry, cache(head_dim=1 << 20, k_token=1 << 20, v_token=1 << 20, k_head=1 << 24, v_head=1 << 24, k_page=1 << 27,
                           v_page=1 << 27, n_kv=64)) == L.QKN_ENOTSUP
    assert copy(dry, cache(), src=BASE + 1000 * MB) == o and copy(dry, cache(), dst=BASE + 2000 * MB) == o


def test_copies_of_4_bits(dry):
    base = dict(k=BASE + 1000 * MB, v=BASE + 1200 * MB, k_exp=BASE + 1400 * MB, v_exp=BASE + 1500 * MB, num_pages=64,
                page_size=16, n_kv=2, head_dim=128)
    for pool, w in (("k", 64), ("v", 64), ("ke", 4), ("ve", 4)):
        base.update({pool + "_token": w, pool + "_head": 16 * w, pool + "_page": 32 * w})
    def call(**kw):
        arr = (S.QknCache4 * 2)(S.QknCache4(**base), S.QknCache4(**{**base, **kw}))
        return dry.qkn_pages_copy4(arr, 2, BASE, BASE + MB, 8, None)
    assert call() == DRY and L.qkn_last_launch()["kernel"] == "pages_copy<16>"
    assert call(ke_token=5, ke_head=80, ke_page=160) == DRY and L.qkn_last_launch()["kernel"] == "pages_copy<1>"
    assert call(head_dim=100) == L.QKN_EINVAL and call(v_exp=None) == L.QKN_EINVAL and call(v_exp=BASE) == L.QKN_EOVERLAP


def test_struct_layout_matches_header(tmp_path):
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    lines = ['printf("qkn_pages %zu\\n", sizeof(qkn_pages));']
    lines += [f'printf("{f} %zu\\n", offsetof(qkn_pages, {f}));' for f, _ in P.QknPages._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "qkn_pages.h"\nint main(void) {'
                   + "\n".join(lines) + "return 0; }")
    subprocess.run(["gcc", "-std=c99", "-I", INCLUDE, str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines():
        name, value = line.split()
        want = ctypes.sizeof(P.QknPages) if name == "qkn_pages" else getattr(P.QknPages, name).offset
        assert int(value) == want, name


def test_bindings_checks():
    b = P.PageBook.empty(10, 3, 100, 16, device="cpu")
    assert b.table.shape == (3, 7) and b.refs.shape == (10,) and b.kv_len.shape == (3,)
    with pytest.raises(ValueError):
        b.struct()  # not on a GPU
    with pytest.raises(TypeError):
        P.PreparedPagesCopy([S.KVCache(b.refs, b.refs), S.KVCache4(*[b.refs] * 4)], b.refs, b.refs)


def test_freeing_without_a_list_is_of_every_row(dry, monkeypatch):
    monkeypatch.setattr(P.PageBook, "struct", lambda self: book(rows=self.table.shape[0]))
    for rows, want in ((0, L.QKN_OK), (1, DRY), (1024, DRY), (1025, L.QKN_ENOTSUP)):
        free = P.PreparedPagesFree(P.PageBook.empty(4, rows, 16, 16, device="cpu"))
        assert free._args[1:] == (None, rows)
        assert free._fn(*free._args, None) == want
