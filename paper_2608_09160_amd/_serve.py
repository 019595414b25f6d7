"""ctypes binding of the attention block's entry points (include/qkn_rope.h, qkn_attn.h, qkn_adapters.h, qkn_cache.h, qkn_cache4.h):
argument marshalling only, as in ``_lib``.

Row tensors are 2-D with a contiguous last dimension and any row stride; heads follow each other in a row, as
the projection writes them. Each operator has a ``Prepared...`` class, whose arguments are checked and marshalled
once (for serving loops and HIP graphs, the tensors stay referenced), and a function that makes the call at once.
"""
from __future__ import annotations

import contextlib
import copy
import ctypes
from dataclasses import dataclass
from typing import Optional, Union

import torch

from ._lib import _c_i64, _check, _f32, _rows, _stream, _vp, load as _load

_int = ctypes.c_int


class QknCache(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("num_pages", _c_i64),
                ("page_size", ctypes.c_int32), ("n_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("fp8", ctypes.c_int32), ("k_page", _c_i64), ("k_head", _c_i64), ("k_token", _c_i64),
                ("v_page", _c_i64), ("v_head", _c_i64), ("v_token", _c_i64)]


class QknCache4(ctypes.Structure):
    _fields_ = ([(n, _vp) for n in ("k", "v", "k_exp", "v_exp")] + [("num_pages", _c_i64)] +
                [(n, ctypes.c_int32) for n in ("page_size", "n_kv", "head_dim")] +
                [(f"{pool}_{n}", _c_i64) for pool in ("k", "v", "ke", "ve") for n in ("page", "head", "token")])


class QknRopeScaling(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("base", "factor", "low", "high", "original", "magnitude")]


class QknRopeSeg(ctypes.Structure):
    _fields_ = [("x", _vp), ("ldx", _c_i64), ("w", _vp), ("partials", _vp), ("d_full", _c_i64), ("y", _vp),
                ("ldy", _c_i64), ("heads", ctypes.c_int32)]


class QknAttnArgs(ctypes.Structure):
    _fields_ = [("q", _vp), ("ldq", _c_i64), ("out", _vp), ("ldo", _c_i64), ("lse", _vp), ("q_start", _vp),
                ("kv_len", _vp), ("block_table", _vp), ("ld_table", _c_i64), ("T", _c_i64),
                ("batch", ctypes.c_int32), ("n_q", ctypes.c_int32), ("max_q", ctypes.c_int32),
                ("max_kv", ctypes.c_int32), ("causal", ctypes.c_int32), ("window", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class QknAdapterSeg(ctypes.Structure):
    _fields_ = [("a", _vp), ("a_adapter", _c_i64), ("lda", _c_i64), ("b", _vp), ("b_adapter", _c_i64),
                ("ldb", _c_i64), ("base", _vp), ("ldbase", _c_i64), ("y", _vp), ("ldy", _c_i64), ("partials", _vp),
                ("d_local", _c_i64)]


def load() -> ctypes.CDLL:
    """The library with these entry points' signatures declared."""
    lib = _load()
    if lib.qkn_rope_cache.argtypes is None:
        lib.qkn_rope_table.argtypes = [_vp, _c_i64, _int, ctypes.POINTER(QknRopeScaling), _vp]
        lib.qkn_rope_cache.argtypes = [ctypes.POINTER(QknRopeSeg), ctypes.POINTER(QknRopeSeg), _vp, _c_i64, _c_i64,
                                       _int, _int, _int, _vp, _c_i64, _vp, _vp, ctypes.POINTER(QknCache), _int,
                                       ctypes.c_float, _vp]
        lib.qkn_rope_cache4.argtypes = [ctypes.POINTER(QknCache4) if a is ctypes.POINTER(QknCache) else a
                                        for a in lib.qkn_rope_cache.argtypes]
        lib.qkn_attn_sinks.argtypes = [ctypes.POINTER(QknAttnArgs), ctypes.c_int32, ctypes.POINTER(QknCache), _vp, _c_i64,
                                       _vp]
        lib.qkn_attn4_workspace_bytes.argtypes = [ctypes.POINTER(QknAttnArgs), ctypes.POINTER(QknCache4)]
        lib.qkn_attn4_workspace_bytes.restype = _c_i64
        lib.qkn_attn4.argtypes = [ctypes.POINTER(QknAttnArgs), ctypes.c_int32, ctypes.POINTER(QknCache4), _vp, _c_i64, _vp]
        lib.qkn_cache4_load.argtypes = [ctypes.POINTER(QknCache4), _vp, _c_i64, _vp, _c_i64, _vp, _c_i64, _vp]
        lib.qkn_attn_workspace_bytes.argtypes = [ctypes.POINTER(QknAttnArgs), ctypes.POINTER(QknCache)]
        lib.qkn_attn_workspace_bytes.restype = _c_i64
        lib.qkn_attn.argtypes = [ctypes.POINTER(QknAttnArgs), ctypes.POINTER(QknCache), _vp, _c_i64, _vp]
        lib.qkn_adapters_workspace_bytes.argtypes = [_c_i64, _c_i64, _int, _int]
        lib.qkn_adapters_workspace_bytes.restype = _c_i64
        lib.qkn_adapters_add.argtypes = [_vp, _c_i64, _c_i64, _c_i64, ctypes.POINTER(QknAdapterSeg), _int, _int, _c_i64,
                                         _vp, _vp, _vp, _c_i64, _vp]
    return lib


def _on(stream):
    """Makes `stream` (None: as it is; a stream or its handle) the current one: what a call allocates for itself then
    belongs to it and is not handed out again before the call's kernels have run."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream)
                             else torch.cuda.ExternalStream(_stream(stream)))


_CACHE_DTYPES = {torch.bfloat16: 0, torch.float8_e4m3fn: 1, torch.uint8: 1}


def _index(t: torch.Tensor, what: str, dtype: torch.dtype, numel: int) -> int:
    if t.dtype != dtype or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous {dtype} GPU tensor")
    if t.numel() < numel:
        raise ValueError(f"{what}: needs {numel} elements, has {t.numel()}")
    return t.data_ptr()


def _pool_strides(name: str, t: torch.Tensor) -> list:
    """Strides of a page, a head and a token."""
    D = t.shape[3]
    if not t.is_cuda or (D > 1 and t.stride(3) != 1):
        raise ValueError(f"cache.{name}: expected a GPU tensor with a contiguous last dimension")
    # the stride of a dimension of one is never used
    return [max(t.stride(i), D) if t.shape[i] == 1 else t.stride(i) for i in (0, 1, 2)]


@dataclass
class KVCache:
    """Pools of pages [pages, kv heads, page size, head dim], of any strides with a contiguous last dimension
    (a permuted view of another order works): bf16, or float8_e4m3fn (uint8 codes) with fp32 scales per KV head."""

    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None

    @property
    def head_dim(self) -> int:
        return self.k.shape[3]

    def struct(self) -> QknCache:
        if self.k.dtype not in _CACHE_DTYPES or self.k.dtype != self.v.dtype:
            raise TypeError(f"cache: expected two pools in bf16 or float8_e4m3fn, got {self.k.dtype}, {self.v.dtype}")
        if self.k.dim() != 4 or self.k.shape != self.v.shape:
            raise ValueError("cache: pools must be [pages, kv heads, page size, head dim], alike")
        pages, n_kv, page, D = self.k.shape
        strides = _pool_strides("k", self.k) + _pool_strides("v", self.v)
        return QknCache(self.k.data_ptr(), self.v.data_ptr(), _f32(self.k_scale, "k_scale", n_kv),
                        _f32(self.v_scale, "v_scale", n_kv), pages, page, n_kv, D, _CACHE_DTYPES[self.k.dtype], *strides)


@dataclass
class KVCache4:
    """Pools of a cache in 4 bits, uint8: codes [pages, kv heads, page size, head dim / 2], two to a byte, and exponents
    [pages, kv heads, page size, head dim / 32] (include/qkn_cache4.h has the format); any strides with a contiguous last
    dimension. Takes a KVCache's place in PreparedRopeCache and PreparedAttn; qkn_cache4_load reads rows back."""

    k: torch.Tensor
    v: torch.Tensor
    k_exp: torch.Tensor
    v_exp: torch.Tensor

    @classmethod
    def empty(cls, pages: int, kv_heads: int, page_size: int, head_dim: int, device="cuda") -> "KVCache4":
        """Pools of that size, not cleared."""
        return cls(*(torch.empty(pages, kv_heads, page_size, head_dim // n, dtype=torch.uint8, device=device)
                     for n in (2, 2, 32, 32)))

    @property
    def head_dim(self) -> int:
        return 2 * self.k.shape[3]

    def struct(self) -> QknCache4:
        pools = (self.k, self.v, self.k_exp, self.v_exp)
        if any(t.dtype != torch.uint8 for t in pools):
            raise TypeError(f"cache: expected four uint8 pools, got {[t.dtype for t in pools]}")
        if self.k.dim() != 4 or self.k.shape[3] % 16:
            raise ValueError("cache: codes must be [pages, kv heads, page size, head dim / 2], head dim a multiple of 32")
        pages, n_kv, page, half = self.k.shape
        if self.v.shape != self.k.shape or any(tuple(t.shape) != (pages, n_kv, page, half // 16) for t in pools[2:]):
            raise ValueError("cache: pools must be of the same pages, heads and rows, exponents [.., head dim / 32]")
        strides = [s for name, t in zip(("k", "v", "k_exp", "v_exp"), pools) for s in _pool_strides(name, t)]
        return QknCache4(*(t.data_ptr() for t in pools), pages, page, n_kv, 2 * half, *strides)


@dataclass
class RopeSeg:
    """Q or K rows for the rotary pass; with w and partials (fp32 [tp, T]) the norm's Phases B+C come first."""

    x: torch.Tensor                           # bf16 [T, heads * head_dim]
    w: Optional[torch.Tensor] = None          # fp32 [heads * head_dim]
    partials: Optional[torch.Tensor] = None   # fp32 [tp, T]
    d_full: int = 0
    y: Optional[torch.Tensor] = None          # bf16 [T, heads * head_dim]; Q's is allocated if None


def qkn_rope_table(n_pos: int, rot_dim: int, base: float = 10000.0, factor: float = 1.0, low: float = 0.0,
                   high: float = 0.0, original: float = 0.0, magnitude: float = 1.0,
                   out: Optional[torch.Tensor] = None, device="cuda", stream=None) -> torch.Tensor:
    """cos and sin of every position and pair, fp32 [n_pos, rot_dim / 2, 2]; see qkn_rope_scaling for the
    scaling to long contexts."""
    with _on(stream):
        if out is None:
            out = torch.empty(n_pos, max(rot_dim, 0) // 2, 2, dtype=torch.float32, device=device)
        sc = QknRopeScaling(base, factor, low, high, original, magnitude)
        _check(load().qkn_rope_table(_f32(out, "out", n_pos * (rot_dim // 2) * 2), n_pos, rot_dim, ctypes.byref(sc),
                                     _stream(None)), "qkn_rope_table")
    return out


class PreparedRopeCache:
    """qkn_rope_cache with its arguments checked and marshalled once: Q and K rows (normalised first where a
    segment has w) rotated by pos (int32 [T]) with table, Q to q.y, K to k.y where given, K and V to rows `slots`
    (int64 [T], page * page size + row; negative: not cached) of the cache (a KVCache4: quantised to 4 bits). table
    None: no rotation."""

    def __init__(self, table: Optional[torch.Tensor], pos: Optional[torch.Tensor], head_dim: int,
                 q: Optional[RopeSeg] = None, k: Optional[RopeSeg] = None, v: Optional[torch.Tensor] = None,
                 cache: Union[KVCache, KVCache4, None] = None, slots: Optional[torch.Tensor] = None,
                 interleaved: bool = False, eps: float = 1e-6):
        if q is None and k is None:
            raise ValueError("q, k or both must be given")
        T, tp, segs = None, None, []
        for name, s in (("q", q), ("k", k)):
            if s is None:
                segs.append(None)
                continue
            px, ldx, Ts, width = _rows(s.x, f"{name}.x")
            if width % head_dim:
                raise ValueError(f"{name}.x: {width} columns are not whole heads of {head_dim}")
            if T is not None and Ts != T:
                raise ValueError("q and k must have the same number of tokens")
            T = Ts
            py, ldy = None, 0
            if s.y is None and name == "q":
                s.y = torch.empty((T, width), dtype=s.x.dtype, device=s.x.device)
            if s.y is not None:
                py, ldy, Ty, wy = _rows(s.y, f"{name}.y")
                if (Ty, wy) != (T, width):
                    raise ValueError(f"{name}.y: shape must match x")
            pp = None
            if s.w is not None:
                if s.partials is None or s.partials.dim() != 2 or s.partials.shape[1] != T:
                    raise ValueError(f"{name}.partials: expected [tp, {T}]")
                if tp is not None and s.partials.shape[0] != tp:
                    raise ValueError("q and k must have statistics of the same number of ranks")
                tp = s.partials.shape[0]
                pp = _f32(s.partials, f"{name}.partials")
            segs.append(QknRopeSeg(px, ldx, _f32(s.w, f"{name}.w", width), pp, s.d_full, py, ldy, width // head_dim))
        pv, ldv = None, 0
        if v is not None:
            pv, ldv, Tv, wv = _rows(v, "v")
            if cache is None or (Tv, wv) != (T, cache.v.shape[1] * head_dim):
                raise ValueError("v: expected a cache and rows of its heads, as many as q's and k's")
        rot, n_pos, pt, pp = 0, 0, None, None
        if table is not None:
            if table.dim() != 3 or table.shape[2] != 2:
                raise ValueError("table: expected [positions, rot_dim / 2, 2]")
            n_pos, rot = table.shape[0], 2 * table.shape[1]
            pt = _f32(table, "table")
            if rot:
                if pos is None:
                    raise ValueError("pos: needed with a table")
                pp = _index(pos, "pos", torch.int32, T)
        ps = None
        if cache is not None:
            if slots is None:
                raise ValueError("slots: needed with a cache")
            ps = _index(slots, "slots", torch.int64, T)
        # as they are now: the tensors stay referenced whatever becomes of the caller's objects
        self.q, self.k, self.v, self.cache = copy.copy(q), copy.copy(k), v, copy.copy(cache)
        self._keep = (table, pos, slots)
        self._cache = cache.struct() if cache is not None else None
        self._segs = segs
        ref = [ctypes.byref(s) if s is not None else None for s in segs]
        self._args = (ref[0], ref[1], pv, ldv, T, head_dim, rot, int(interleaved), pt, n_pos, pp, ps,
                      ctypes.byref(self._cache) if cache is not None else None, tp or 1, ctypes.c_float(eps))
        self._name = "qkn_rope_cache4" if isinstance(cache, KVCache4) else "qkn_rope_cache"
        self._fn = getattr(load(), self._name)

    def __call__(self, stream=None):
        _check(self._fn(*self._args, _stream(stream)), self._name)
        return self.q.y if self.q is not None else None


def qkn_rope_cache(table, pos, head_dim, q=None, k=None, v=None, cache=None, slots=None, interleaved=False,
                   eps=1e-6, stream=None):
    """PreparedRopeCache made and called once; returns q's rotated rows."""
    with _on(stream):
        return PreparedRopeCache(table, pos, head_dim, q, k, v, cache, slots, interleaved, eps)()


def _workspace(workspace: Optional[torch.Tensor], need: int, device) -> torch.Tensor:
    if workspace is None:
        return torch.empty(max(need, 16), dtype=torch.uint8, device=device)
    if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace: expected a contiguous uint8 GPU tensor")
    return workspace


class PreparedAttn:
    """qkn_attn (qkn_attn_sinks, qkn_attn4) with its arguments and workspace prepared once (calls share the workspace: on one stream at a time):
    attention of the new tokens q (bf16 [T, heads *
    head_dim], the sequences in order) over the cache that holds their keys and values already.

    block_table int32 [batch, pages of a sequence], q_start int32 [batch + 1], kv_len int32 [batch] (new tokens
    included) are read by the kernel on the device: a replayed graph sees what they hold then. Tokens before q_start's
    first entry and behind its last are padding: out is 0 there, lse -infinity. max_q and max_kv: the
    largest numbers of new and cached tokens of a sequence (the default: T, and what block_table's rows can hold).
    lse: optional fp32 [T, heads], receives the log-sum-exp. window: keys that a token sees, its own the last (0:
    all); sinks: the sequence's first tokens, which it sees as well. cache may be a KVCache4."""

    def __init__(self, q: torch.Tensor, cache: Union[KVCache, KVCache4], block_table: torch.Tensor, q_start: torch.Tensor,
                 kv_len: torch.Tensor, max_q: Optional[int] = None, max_kv: Optional[int] = None,
                 scale: Optional[float] = None, causal: bool = True, window: int = 0,
                 out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, sinks: int = 0):
        c = cache.struct()
        pq, ldq, T, width = _rows(q, "q")
        if width % c.head_dim or (width // c.head_dim) % c.n_kv:
            raise ValueError(f"q: {width} columns are not a multiple of {c.n_kv} heads of {c.head_dim}")
        heads = width // c.head_dim
        if out is None:
            out = torch.empty((T, width), dtype=q.dtype, device=q.device)
        po, ldo, To, wo = _rows(out, "out")
        if (To, wo) != (T, width):
            raise ValueError("out: shape must match q")
        if block_table.dim() != 2:
            raise ValueError("block_table: expected [batch, pages]")
        batch, pages = block_table.shape
        if q_start.numel() != batch + 1 or kv_len.numel() != batch:
            raise ValueError(f"q_start, kv_len: expected {batch + 1} and {batch} elements")
        if lse is not None and tuple(lse.shape) != (T, heads):
            raise ValueError(f"lse: expected [{T}, {heads}]")
        limit = 2 ** 31 - 1
        if not 0 <= sinks <= limit:
            raise ValueError(f"sinks: expected 0 to {limit}, got {sinks}")
        max_q = min(T, limit) if max_q is None else max_q
        max_kv = min(pages * c.page_size, limit) if max_kv is None else max_kv
        a = QknAttnArgs(pq, ldq, po, ldo, _f32(lse, "lse"), _index(q_start, "q_start", torch.int32, batch + 1),
                        _index(kv_len, "kv_len", torch.int32, batch),
                        _index(block_table, "block_table", torch.int32, batch * pages), pages, T, batch, heads, max_q,
                        max_kv, int(causal), window, c.head_dim ** -0.5 if scale is None else scale)
        lib = load()
        name = "qkn_attn4" if isinstance(cache, KVCache4) else "qkn_attn"
        need = getattr(lib, name + "_workspace_bytes")(ctypes.byref(a), ctypes.byref(c))
        if need < 0:
            _check(int(need), name + "_workspace_bytes")
        self._name = name if name == "qkn_attn4" else "qkn_attn_sinks"
        self.workspace = _workspace(workspace, need, q.device)
        self.q, self.out, self.lse, self.cache = q, out, lse, copy.copy(cache)
        self._keep = (block_table, q_start, kv_len, a, c)
        self._args = (ctypes.byref(a), sinks, ctypes.byref(c), self.workspace.data_ptr(), self.workspace.numel())
        self._fn = getattr(lib, self._name)

    def __call__(self, stream=None) -> torch.Tensor:
        _check(self._fn(*self._args, _stream(stream)), self._name)
        return self.out


def qkn_attn(q, cache, block_table, q_start, kv_len, max_q=None, max_kv=None, scale=None, causal=True, window=0,
             out=None, lse=None, workspace=None, stream=None, sinks=0) -> torch.Tensor:
    """PreparedAttn made and called once."""
    with _on(stream):
        return PreparedAttn(q, cache, block_table, q_start, kv_len, max_q, max_kv, scale, causal, window, out, lse,
                            workspace, sinks)()


class PreparedCache4Load:
    """qkn_cache4_load with its arguments prepared once: the rows `slots` (int64 [T], page * page size + row; outside the
    cache: zeros) of a 4-bit cache as bf16 [T, kv heads * head_dim], to k and v (allocated if both are None)."""

    def __init__(self, cache: KVCache4, slots: torch.Tensor, k: Optional[torch.Tensor] = None,
                 v: Optional[torch.Tensor] = None):
        c, T = cache.struct(), slots.numel()
        width = c.n_kv * c.head_dim
        if k is None and v is None:
            k, v = (torch.empty(T, width, dtype=torch.bfloat16, device=slots.device) for _ in range(2))
        rows = []
        for name, t in (("k", k), ("v", v)):
            if t is None:
                rows += [None, 0]
                continue
            p, ld, Tt, w = _rows(t, name)
            if (Tt, w) != (T, width):
                raise ValueError(f"{name}: expected [{T}, {width}]")
            rows += [p, ld]
        self.k, self.v, self.cache = k, v, copy.copy(cache)
        self._keep = (slots, c)
        self._args = (ctypes.byref(c), _index(slots, "slots", torch.int64, T), T, *rows)
        self._fn = load().qkn_cache4_load

    def __call__(self, stream=None):
        _check(self._fn(*self._args, _stream(stream)), "qkn_cache4_load")
        return self.k, self.v


def qkn_cache4_load(cache, slots, k=None, v=None, stream=None):
    """PreparedCache4Load made and called once; returns (k, v)."""
    with _on(stream):
        return PreparedCache4Load(cache, slots, k, v)()


@dataclass
class AdapterSeg:
    """One output (Q, K or V) of the adapters: a bf16 [adapters, rank, hidden], b bf16 [adapters, d_local, rank] (any
    strides with a contiguous last dimension), base the projection's rows (None: y, in place)."""

    a: torch.Tensor
    b: torch.Tensor
    y: Optional[torch.Tensor] = None         # bf16 [T, d_local]; allocated if None and base is given
    partials: Optional[torch.Tensor] = None  # fp32 [T]; not taken if None
    base: Optional[torch.Tensor] = None      # bf16 [T, d_local]


def _matrices(t: torch.Tensor, what: str):
    """(pointer, stride of an adapter, stride of a row) of a [adapters, rows, columns] tensor."""
    if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{what}: expected a bf16 GPU tensor [adapters, rows, columns], last dimension contiguous")
    return t.data_ptr(), t.stride(0), t.stride(1) if t.shape[1] > 1 else max(t.stride(1), t.shape[2])


class PreparedAdapters:
    """qkn_adapters_add with its arguments and workspace prepared once (calls share the workspace: on one stream at a
    time): y = base + scale_i B_i A_i x for the tokens
    of each request's adapter i = ids[t] (int32 [T]; outside the adapters: none), and the Phase A statistic of the
    stored rows. x is the projection's input (bf16 [T, hidden]), scale fp32 [adapters] or None."""

    def __init__(self, x: torch.Tensor, segs, ids: torch.Tensor, scale: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None):
        px, ldx, T, hidden = _rows(x, "x")
        segs = list(segs)
        if not 1 <= len(segs) <= 3:
            raise ValueError("1 to 3 segments are expected")
        count, rank = segs[0].a.shape[:2] if segs[0].a.dim() == 3 else (0, 0)
        arr = (QknAdapterSeg * len(segs))()
        for i, s in enumerate(segs):
            a, b = _matrices(s.a, f"seg{i}.a"), _matrices(s.b, f"seg{i}.b")
            d = s.b.shape[1]
            if tuple(s.a.shape) != (count, rank, hidden) or tuple(s.b.shape) != (count, d, rank):
                raise ValueError(f"seg{i}: expected a [{count}, {rank}, {hidden}] and b [{count}, d, {rank}], got "
                                 f"{tuple(s.a.shape)}, {tuple(s.b.shape)}")
            if s.y is None:
                if s.base is None:
                    raise ValueError(f"seg{i}: base, y or both must be given")
                s.y = torch.empty((T, d), dtype=s.base.dtype, device=s.base.device)
            py, ldy, Ty, wy = _rows(s.y, f"seg{i}.y")
            pb, ldb, Tb, wb = (py, ldy, Ty, wy) if s.base is None else _rows(s.base, f"seg{i}.base")
            if (Ty, wy) != (T, d) or (Tb, wb) != (T, d):
                raise ValueError(f"seg{i}: y and base must be [{T}, {d}]")
            arr[i] = QknAdapterSeg(*a, *b, pb, ldb, py, ldy, _f32(s.partials, f"seg{i}.partials", T), d)
        lib = load()
        need = lib.qkn_adapters_workspace_bytes(T, hidden, rank, len(segs))
        if need < 0:
            _check(int(need), "qkn_adapters_workspace_bytes")
        self.workspace = _workspace(workspace, need, x.device)
        self.segs = [copy.copy(s) for s in segs]
        self._keep = (x, ids, scale)
        self._args = (px, ldx, T, hidden, arr, len(segs), rank, count, _index(ids, "ids", torch.int32, T),
                      _f32(scale, "scale", count), self.workspace.data_ptr(), self.workspace.numel())
        self._fn = lib.qkn_adapters_add

    def __call__(self, stream=None):
        _check(self._fn(*self._args, _stream(stream)), "qkn_adapters_add")
        return [(s.y, s.partials) for s in self.segs]


def qkn_adapters_add(x, segs, ids, scale=None, workspace=None, stream=None):
    """PreparedAdapters made and called once; returns the segments' (y, partials)."""
    with _on(stream):
        return PreparedAdapters(x, segs, ids, scale, workspace)()
