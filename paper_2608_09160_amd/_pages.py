"""ctypes binding of the book of a cache's pages (include/qkn_pages.h): argument marshalling only, as in ``_serve``.

Each call has a ``Prepared...`` class, whose arguments are checked and marshalled once (for serving loops and HIP graphs,
the tensors stay referenced), and a function that makes the call at once.
"""
from __future__ import annotations

import copy
import ctypes
from dataclasses import dataclass
from typing import Optional, Sequence, Union

import torch

from ._lib import _c_i64, _check, _stream, _vp, load as _load
from ._serve import KVCache, KVCache4, QknCache, QknCache4, _index, _on, _workspace

_i32 = ctypes.c_int32


class QknPages(ctypes.Structure):
    _fields_ = [("refs", _vp), ("table", _vp), ("kv_len", _vp), ("num_pages", _c_i64), ("ld_table", _c_i64),
                ("rows", _i32), ("page_size", _i32)]


def load() -> ctypes.CDLL:
    """The library with these entry points' signatures declared."""
    lib = _load()
    if lib.qkn_pages_grow.argtypes is None:
        book = ctypes.POINTER(QknPages)
        lib.qkn_pages_grow.argtypes = [book, _vp, _vp, _i32, _c_i64, _vp, _vp, _vp, _vp]
        lib.qkn_pages_fork.argtypes = [book, _vp, _vp, _i32, _vp, _vp, _vp, _vp]
        lib.qkn_pages_free.argtypes = [book, _vp, _i32, _vp]
        lib.qkn_pages_compact_workspace_bytes.argtypes = [book]
        lib.qkn_pages_compact_workspace_bytes.restype = _c_i64
        lib.qkn_pages_compact.argtypes = [book, book, _vp, _vp, _i32, _vp, _c_i64, _vp]
        lib.qkn_pages_copy.argtypes = [ctypes.POINTER(QknCache), _i32, _vp, _vp, _i32, _vp]
        lib.qkn_pages_copy4.argtypes = [ctypes.POINTER(QknCache4), _i32, _vp, _vp, _i32, _vp]
    return lib


@dataclass
class PageBook:
    """Which pages each row (sequence) of a batch has, on the device: refs int32 [pages] (rows that have the page, 0:
    free), table int32 [rows, pages of a row], kv_len int32 [rows]. table and kv_len are what PreparedAttn takes."""

    refs: torch.Tensor
    table: torch.Tensor
    kv_len: torch.Tensor
    page_size: int

    @classmethod
    def empty(cls, pages: int, rows: int, max_tokens: int, page_size: int, device="cuda") -> "PageBook":
        """A book of `rows` empty rows, each of up to max_tokens tokens."""
        per = (max_tokens + page_size - 1) // page_size
        return cls(*(torch.zeros(*shape, dtype=torch.int32, device=device) for shape in ((pages,), (rows, per), (rows,))),
                   page_size)

    def struct(self) -> QknPages:
        if self.table.dim() != 2 or self.refs.dim() != 1 or tuple(self.kv_len.shape) != self.table.shape[:1]:
            raise ValueError("book: expected refs [pages], table [rows, pages of a row], kv_len [rows]")
        rows, per = self.table.shape
        return QknPages(_index(self.refs, "book.refs", torch.int32, 0), _index(self.table, "book.table", torch.int32, 0),
                        _index(self.kv_len, "book.kv_len", torch.int32, 0), self.refs.numel(), per, rows, self.page_size)


class _Call:
    """A prepared call: `_keep` has what its arguments point at."""

    _name = ""

    def _prepare(self, book, *args, keep=()):
        self.book = copy.copy(book)
        self._keep = keep
        self._args = args
        self._fn = getattr(load(), self._name)

    def _run(self, stream):
        _check(self._fn(*self._args, _stream(stream)), self._name)


def _list(t: Optional[torch.Tensor], what: str, n: int) -> Optional[int]:
    if t is not None and t.numel() != n:
        raise ValueError(f"{what}: expected {n} elements, got {t.numel()}")
    return None if t is None else _index(t, what, torch.int32, n)


class PreparedPagesGrow(_Call):
    """qkn_pages_grow: counts[i] (int32) more tokens for row which[i] (int32; None: row i), with their pages. slots
    (int64) and pos (int32), or None, receive where the new tokens go, in the order of the list, done (int32, allocated
    if None) the rows' tokens or -1 where the pool or the row has no room."""

    _name = "qkn_pages_grow"

    def __init__(self, book: PageBook, counts: torch.Tensor, which: Optional[torch.Tensor] = None,
                 slots: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None,
                 done: Optional[torch.Tensor] = None):
        n = counts.numel()
        if done is None:
            done = torch.empty(n, dtype=torch.int32, device=counts.device)
        if slots is not None and pos is not None and slots.numel() != pos.numel():
            raise ValueError("slots and pos must be of one length")
        T = slots.numel() if slots is not None else pos.numel() if pos is not None else 0
        self.counts, self.which, self.slots, self.pos, self.done = counts, which, slots, pos, done
        b = book.struct()
        self._prepare(book, ctypes.byref(b), _list(which, "which", n), _list(counts, "counts", n), n, T,
                      None if slots is None else _index(slots, "slots", torch.int64, T), _list(pos, "pos", T),
                      _list(done, "done", n), keep=(b,))

    def __call__(self, stream=None) -> torch.Tensor:
        self._run(stream)
        return self.done


class PreparedPagesFork(_Call):
    """qkn_pages_fork: the empty rows `to` (int32) become copies of the rows `parents` (int32). Whole pages are shared; src
    and dst (int32, allocated if None) receive the partly full ones and their copies' pages, -1 where there is none, for
    PreparedPagesCopy; done the rows' tokens, or -1."""

    _name = "qkn_pages_fork"

    def __init__(self, book: PageBook, parents: torch.Tensor, to: torch.Tensor, src: Optional[torch.Tensor] = None,
                 dst: Optional[torch.Tensor] = None, done: Optional[torch.Tensor] = None):
        n = parents.numel()
        src, dst, done = (torch.empty(n, dtype=torch.int32, device=parents.device) if t is None else t
                          for t in (src, dst, done))
        self.parents, self.to, self.src, self.dst, self.done = parents, to, src, dst, done
        b = book.struct()
        self._prepare(book, ctypes.byref(b), _list(parents, "parents", n), _list(to, "to", n), n, _list(src, "src", n),
                      _list(dst, "dst", n), _list(done, "done", n), keep=(b,))

    def __call__(self, stream=None) -> torch.Tensor:
        self._run(stream)
        return self.done


class PreparedPagesFree(_Call):
    """qkn_pages_free: empties the rows `which` (int32; None: every row of the book)."""

    _name = "qkn_pages_free"

    def __init__(self, book: PageBook, which: Optional[torch.Tensor] = None):
        b = book.struct()
        n = b.rows if which is None else which.numel()
        self.which = which
        self._prepare(book, ctypes.byref(b), _list(which, "which", n), n, keep=(b,))

    def __call__(self, stream=None) -> None:
        self._run(stream)


class PreparedPagesCompact(_Call):
    """qkn_pages_compact: pages in use move to the front of the pools, as many as src and dst (int32) have room for; they
    receive the moves, for PreparedPagesCopy. out: a book of the same sizes that receives table and refs (None: in
    place). Calls share the workspace: on one stream at a time."""

    _name = "qkn_pages_compact"

    def __init__(self, book: PageBook, src: torch.Tensor, dst: torch.Tensor, out: Optional[PageBook] = None,
                 workspace: Optional[torch.Tensor] = None):
        b, n = book.struct(), src.numel()
        o = None if out is None else out.struct()
        lib = load()
        need = lib.qkn_pages_compact_workspace_bytes(ctypes.byref(b))
        if need < 0:
            _check(int(need), "qkn_pages_compact_workspace_bytes")
        self.src, self.dst, self.out = src, dst, copy.copy(book if out is None else out)
        self.workspace = _workspace(workspace, need, src.device)
        self._prepare(book, ctypes.byref(b), None if o is None else ctypes.byref(o), _list(src, "src", n),
                      _list(dst, "dst", n), n, self.workspace.data_ptr(), self.workspace.numel(), keep=(b, o))

    def __call__(self, stream=None):
        self._run(stream)
        return self.src, self.dst


class PreparedPagesCopy(_Call):
    """qkn_pages_copy (4-bit caches: qkn_pages_copy4): page src[i] to page dst[i] (int32) in every cache of the list."""

    def __init__(self, caches: Sequence[Union[KVCache, KVCache4]], src: torch.Tensor, dst: torch.Tensor):
        caches, n = list(caches), src.numel()
        four = [isinstance(c, KVCache4) for c in caches]
        if any(four) and not all(four):
            raise TypeError("caches: 4-bit ones and others in calls of their own")
        self._name = "qkn_pages_copy4" if caches and four[0] else "qkn_pages_copy"
        structs = ((QknCache4 if caches and four[0] else QknCache) * len(caches))(*(c.struct() for c in caches))
        self.caches, self.src, self.dst = [copy.copy(c) for c in caches], src, dst
        self._prepare(None, structs, len(caches), _list(src, "src", n), _list(dst, "dst", n), n, keep=())

    def __call__(self, stream=None) -> None:
        self._run(stream)


def qkn_pages_grow(book, counts, which=None, slots=None, pos=None, done=None, stream=None) -> torch.Tensor:
    """PreparedPagesGrow made and called once."""
    with _on(stream):
        return PreparedPagesGrow(book, counts, which, slots, pos, done)()


def qkn_pages_fork(book, parents, to, caches=(), src=None, dst=None, stream=None) -> torch.Tensor:
    """PreparedPagesFork made and called once, and the pages copied in `caches`."""
    with _on(stream):
        fork = PreparedPagesFork(book, parents, to, src, dst)
        done = fork()
        if caches:
            PreparedPagesCopy(caches, fork.src, fork.dst)()
        return done


def qkn_pages_free(book, which=None, stream=None) -> None:
    """PreparedPagesFree made and called once."""
    with _on(stream):
        PreparedPagesFree(book, which)()


def qkn_pages_compact(book, src, dst, caches=(), out=None, workspace=None, stream=None):
    """PreparedPagesCompact made and called once, and the pages moved in `caches`; returns (src, dst)."""
    with _on(stream):
        moves = PreparedPagesCompact(book, src, dst, out, workspace)()
        if caches:
            PreparedPagesCopy(caches, src, dst)()
        return moves


def qkn_pages_copy(caches, src, dst, stream=None) -> None:
    """PreparedPagesCopy made and called once."""
    with _on(stream):
        PreparedPagesCopy(caches, src, dst)()
