"""The key/value cache around the verification step (argument marshalling only).

Speculative sampling passes gamma drafted tokens and the token before them
through the target model at once and keeps accepted_len + 1 of them (Sec. 3.1).
The target model's attention therefore writes gamma + 1 cache entries a
sequence and step, reads everything cached so far, and keeps the accepted part.
This module has the cache's operators, each a call of the HIP library
(include/spec_cache.h) on the current stream:

* :meth:`PagedCache.plan` builds block tables and slot maps on the GPU from the
  sequences' lengths, the verification's ``accepted_len`` and the sequences that
  ended -- nothing of it passes through the host;
* :func:`append` (:meth:`PagedCache.append`) writes new keys and values to the
  mapped slots;
* :func:`attend` (:meth:`PagedCache.attend`) is the attention of the new tokens
  to a prefix that the whole batch shares, whose reads the sequences' tokens
  share, and to each sequence's own entries.

A step of a target model with such a cache::

    cache = PagedCache(B, num_pages=N, page_size=16, max_pages=M, max_new=gamma_max + 1, prefix_pages=X)
    k_cache, v_cache = cache.new_storage(kv_heads, head_dim, torch.bfloat16)   # for each layer
    cache.plan(gamma + 1, accepted_len=accepted_len)     # what was verified last stays
    cache.append(k, v, k_cache, v_cache)                 # k, v [B, gamma + 1, kv_heads, head_dim]
    out = cache.attend(q, k_cache, v_cache)              # q [B, gamma + 1, q_heads, head_dim]

:class:`~paper_2406_11016_amd.decode_loop.DecodeLoop` plans its cache's next
step itself when it is given one.  Tensors of a step are padded to the same
number of tokens a sequence, as the ragged verification's are.
"""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Tuple

import torch

from . import binding
from .binding import SpecVerifyError, _check, _i32, _ptr, _sz, _vp

MAX_BATCH = 4096
HEAD_DIMS = (64, 80, 96, 128, 256)
DTYPE_CODES = {torch.float16: binding.SV_F16, torch.bfloat16: binding.SV_BF16}

SYMBOLS = (
    "spec_cache_init",
    "spec_cache_plan",
    "spec_cache_append",
    "spec_cache_attend",
    "spec_cache_attend_workspace_bytes",
)

_i64x3 = ctypes.c_int64 * 3


class Tables(ctypes.Structure):
    """``sv_cache_tables_t`` (see spec_cache.h)."""
    _fields_ = [("lengths", _vp), ("counts", _vp), ("held", _vp), ("block_table", _vp), ("free_pages", _vp),
                ("free_count", _vp), ("batch", _i32), ("max_pages", _i32), ("num_pages", _i32), ("page_size", _i32)]


class AppendDesc(ctypes.Structure):
    """``sv_cache_append_desc_t``."""
    _fields_ = [("k", _vp), ("v", _vp), ("k_stride", _i64x3), ("v_stride", _i64x3), ("k_cache", _vp),
                ("v_cache", _vp), ("page_stride", ctypes.c_int64), ("slots", _vp), ("dtype", ctypes.c_int),
                ("batch", _i32), ("max_new", _i32), ("kv_heads", _i32), ("head_dim", _i32), ("num_pages", _i32),
                ("page_size", _i32)]


class AttendDesc(ctypes.Structure):
    """``sv_cache_attend_desc_t``."""
    _fields_ = [("q", _vp), ("out", _vp), ("q_stride", _i64x3), ("out_stride", _i64x3), ("k_cache", _vp),
                ("v_cache", _vp), ("page_stride", ctypes.c_int64), ("block_table", _vp), ("lengths", _vp),
                ("counts", _vp), ("prefix_table", _vp), ("prefix_len", _i32), ("dtype", ctypes.c_int),
                ("batch", _i32), ("max_new", _i32), ("q_heads", _i32), ("kv_heads", _i32), ("head_dim", _i32),
                ("max_pages", _i32), ("num_pages", _i32), ("page_size", _i32), ("scale", ctypes.c_float),
                ("workspace", _vp), ("workspace_bytes", _sz)]


# the same structures, packed in one go: filling a ctypes structure field by
# field takes as long as the launch itself
_pack_append = struct.Struct("@QQ6qQQqQ7i4x").pack
_pack_attend = struct.Struct("@QQ6qQQqQQQQ10ifQN").pack

_lib = None


def load_library() -> ctypes.CDLL:
    """The HIP library with the cache's functions declared (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    lib = binding.load_library()
    lib.spec_cache_init.argtypes = [ctypes.POINTER(Tables), _i32, _vp]
    lib.spec_cache_plan.argtypes = [ctypes.POINTER(Tables), _vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp]
    lib.spec_cache_append.argtypes = [_vp, _vp]
    lib.spec_cache_attend.argtypes = [_vp, _vp]
    for f in (lib.spec_cache_init, lib.spec_cache_plan, lib.spec_cache_append, lib.spec_cache_attend):
        f.restype = ctypes.c_int
    lib.spec_cache_attend_workspace_bytes.argtypes = [_i32] * 5
    lib.spec_cache_attend_workspace_bytes.restype = _sz
    _lib = lib
    return lib


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(index: int, f, what: str, *args) -> None:
    """f(*args, stream) on the current stream of the tensors' device."""
    if _current_device() == index:
        st = f(*args, _stream(index))
    else:
        with torch.cuda.device(index):
            st = f(*args, _stream(index))
    if st != 0:
        _check(st, what)


def _stream(index: int) -> int:
    if binding._raw_stream is not None:
        return binding._raw_stream(index)
    return torch.cuda.current_stream(index).cuda_stream


def _int32(name: str, t: torch.Tensor, shape, index: int) -> None:
    if t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous() or t.get_device() != index:
        raise SpecVerifyError(f"{name} must be a contiguous int32 {list(shape)} tensor on device {index}")


def _rows(name: str, t: torch.Tensor, shape, index: int, dtype):
    """The address and the strides of a [batch, tokens, heads, head_dim] tensor that the kernels can address."""
    if t.shape != shape or t.get_device() != index or t.dtype != dtype:
        raise SpecVerifyError(f"{name} must be a {dtype} {list(shape)} tensor on device {index}")
    at, (sb, st, sh, sd) = t.data_ptr(), t.stride()
    if sd != 1 or (sb | st | sh) & 7 or at & 15:
        raise SpecVerifyError(f"{name}: head_dim must be dense, the other strides multiples of 8 elements and the data "
                              f"aligned to 16 bytes (strides {t.stride()})")
    return at, sb, st, sh


def _caches(k_cache: torch.Tensor, v_cache: torch.Tensor):
    """A pair of caches: device, dtype, shape, addresses and the stride of their pages."""
    index, dtype, shape, strides = k_cache.get_device(), k_cache.dtype, k_cache.shape, k_cache.stride()
    if index < 0 or len(shape) != 4 or dtype not in DTYPE_CODES:
        raise SpecVerifyError("caches must be float16 or bfloat16 device tensors [num_pages, kv_heads, page_size, "
                              "head_dim]")
    if v_cache.shape != shape or v_cache.dtype != dtype or v_cache.get_device() != index or v_cache.stride() != strides:
        raise SpecVerifyError("k_cache and v_cache must be alike in shape, strides, dtype and device")
    (n, h, p, d), (sn, sh, sp, sd) = shape, strides
    if n == 1:
        sn = max(sn, h * p * d)
    k, v = k_cache.data_ptr(), v_cache.data_ptr()
    if sd != 1 or sp != d or (h > 1 and sh != p * d) or (sn | k >> 1 | v >> 1) & 7 or (k | v) & 1:
        raise SpecVerifyError("a cache's pages must be dense and aligned to 16 bytes")
    return index, dtype, shape, k, v, sn


def append(k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
           slots: torch.Tensor) -> None:
    """New keys and values ``[B, n, kv_heads, head_dim]`` into the slots that ``slots`` (int32 ``[B, n]``) names;
    tokens with a slot outside the cache (-1) are left out.  Rows may lie apart (views of a fused projection)."""
    lib = _lib if _lib is not None else load_library()
    index, dtype, (num_pages, h, p, d), k_at, v_at, page_stride = _caches(k_cache, v_cache)
    shape = k.shape
    if len(shape) != 4 or shape[2] != h or shape[3] != d:
        raise SpecVerifyError(f"k and v must be [batch, tokens, {h}, {d}] for these caches; k is {list(shape)}")
    B, n = shape[0], shape[1]
    k_from, kb, kt, kh = _rows("k", k, shape, index, dtype)
    v_from, vb, vt, vh = _rows("v", v, shape, index, dtype)
    _int32("slots", slots, (B, n), index)
    _call(index, lib.spec_cache_append, "spec_cache_append",
          _pack_append(k_from, v_from, kb, kt, kh, vb, vt, vh, k_at, v_at, page_stride, slots.data_ptr(),
                       DTYPE_CODES[dtype], B, n, h, d, num_pages, p))


def attend_workspace_bytes(batch: int, max_new: int, q_heads: int, kv_heads: int, head_dim: int) -> int:
    n = load_library().spec_cache_attend_workspace_bytes(batch, max_new, q_heads, kv_heads, head_dim)
    if n == 0:
        raise SpecVerifyError(f"invalid sizes: batch={batch} max_new={max_new} q_heads={q_heads} kv_heads={kv_heads} "
                              f"head_dim={head_dim}")
    return int(n)


def new_attend_workspace(batch: int, max_new: int, q_heads: int, kv_heads: int, head_dim: int, device) -> torch.Tensor:
    """A workspace for attend() at these sizes (reusable across ordered calls; needs no initialisation)."""
    return torch.empty(attend_workspace_bytes(batch, max_new, q_heads, kv_heads, head_dim), dtype=torch.uint8,
                       device=device)


def attend(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor,
           lengths: torch.Tensor, counts: Optional[torch.Tensor] = None, *,
           prefix_table: Optional[torch.Tensor] = None, prefix_len: int = 0, scale: Optional[float] = None,
           out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of new tokens ``q [B, n, q_heads, head_dim]`` whose keys and values are in the cache already.

    Token i of sequence b sees the shared prefix (``prefix_len`` tokens in the pages of ``prefix_table``, int32) and
    its sequence's own tokens ``0 .. lengths[b] + i`` (``block_table [B, max_pages]``, ``lengths [B]``, int32).  Rows
    behind ``counts[b]`` (int32 [B]; all n without it) are neither read nor written; a new ``out`` is zero there, for
    which all of it is filled first: pass ``out`` to go without.  ``out`` does not overlap ``q``, nor itself.  For
    inference: the result has no gradient, whatever ``q`` requires.  At head_dim 256 the batch is at most 2,048, else
    4,096.  ``scale`` (1e-30 to 1e30) defaults to ``head_dim ** -0.5``.  ``workspace`` (see new_attend_workspace) avoids
    an allocation a call.
    """
    lib = _lib if _lib is not None else load_library()
    index, dtype, (num_pages, K, P, D), k_at, v_at, page_stride = _caches(k_cache, v_cache)
    shape = q.shape
    if len(shape) != 4 or shape[3] != D:
        raise SpecVerifyError(f"q must be [batch, tokens, q_heads, {D}] for these caches; it is {list(shape)}")
    B, n, H, _ = shape
    q_at, qb, qt, qh = _rows("q", q, shape, index, dtype)
    if block_table.dim() != 2:
        raise SpecVerifyError("block_table must be [batch, max_pages]")
    M = block_table.shape[1]
    _int32("block_table", block_table, (B, M), index)
    _int32("lengths", lengths, (B,), index)
    if counts is not None:
        _int32("counts", counts, (B,), index)
    if prefix_len:
        if prefix_table is None or prefix_table.dim() != 1 or prefix_table.numel() * P < prefix_len:
            raise SpecVerifyError(f"prefix_table must name the pages of {prefix_len} tokens")
        _int32("prefix_table", prefix_table, prefix_table.shape, index)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=q.device) if counts is None else \
            torch.zeros(shape, dtype=dtype, device=q.device)
    out_at, ob, ot, oh = _rows("out", out, shape, index, dtype)
    if workspace is None:
        workspace = new_attend_workspace(B, n, H, K, D, q.device)
    elif not workspace.is_contiguous() or workspace.get_device() != index:
        raise SpecVerifyError(f"workspace must be a contiguous tensor on device {index}")
    _call(index, lib.spec_cache_attend, "spec_cache_attend",
          _pack_attend(q_at, out_at, qb, qt, qh, ob, ot, oh, k_at, v_at, page_stride, block_table.data_ptr(),
                       lengths.data_ptr(), 0 if counts is None else counts.data_ptr(),
                       prefix_table.data_ptr() if prefix_len else 0, prefix_len, DTYPE_CODES[dtype], B, n, H, K, D, M,
                       num_pages, P, D ** -0.5 if scale is None else scale, workspace.data_ptr(),
                       workspace.numel() * workspace.element_size()))
    return out


class PagedCache:
    """The tables of a batch's paged cache, on the GPU: one set for all layers of a model.

    ``num_pages`` pages of ``page_size`` tokens (a power of two from 16 to 1024) serve ``batch`` sequences of up to
    ``max_pages`` pages each and, in the first ``prefix_pages`` of them, a prefix that all sequences share
    (:meth:`set_prefix`).  The buffers are static: captured graphs may hold them.  Calls go to the current stream and
    have to be ordered, as all calls that share tables, caches or a workspace.
    """

    def __init__(self, batch: int, *, num_pages: int, page_size: int, max_pages: int, max_new: int,
                 prefix_pages: int = 0, device="cuda"):
        def new(*shape):
            return torch.empty(shape, dtype=torch.int32, device=device)

        if min(batch, num_pages, max_pages, max_new) < 1 or not 0 <= prefix_pages <= num_pages:
            raise SpecVerifyError(f"invalid sizes: batch={batch} num_pages={num_pages} max_pages={max_pages} "
                                  f"max_new={max_new} prefix_pages={prefix_pages}")
        self._adopt(new(batch), new(batch), new(batch), new(batch, max_pages), new(num_pages), new(1), page_size,
                    max_new)
        self.prefix_table = torch.arange(prefix_pages, dtype=torch.int32, device=self.device)
        self._prefix_first = True
        self.reset()

    @classmethod
    def over(cls, lengths: torch.Tensor, counts: torch.Tensor, held: torch.Tensor, block_table: torch.Tensor,
             free_pages: torch.Tensor, free_count: torch.Tensor, *, page_size: int, max_new: int,
             prefix_table: Optional[torch.Tensor] = None) -> "PagedCache":
        """Over a program's own tables (int32; see sv_cache_tables_t), as they are.  ``prefix_table`` names the pages
        of the shared prefix, any that are in no sequence's table and not free."""
        self = cls.__new__(cls)
        self._adopt(lengths, counts, held, block_table, free_pages, free_count, page_size, max_new)
        self.prefix_table = prefix_table if prefix_table is not None else lengths.new_empty(0)
        self._prefix_first = self.prefix_table.numel() == 0
        _int32("prefix_table", self.prefix_table, (self.prefix_table.numel(),), self._index)
        return self

    def _adopt(self, lengths, counts, held, block_table, free_pages, free_count, page_size, max_new) -> None:
        self._lib = load_library()
        index = lengths.get_device()
        if index < 0 or block_table.dim() != 2 or free_pages.dim() != 1:
            raise SpecVerifyError("the tables must be device tensors: lengths, counts, held [batch], block_table "
                                  "[batch, max_pages], free_pages [num_pages], free_count [1]")
        B, M = block_table.shape
        N = free_pages.numel()
        for name, t, shape in (("lengths", lengths, (B,)), ("counts", counts, (B,)), ("held", held, (B,)),
                               ("block_table", block_table, (B, M)), ("free_pages", free_pages, (N,)),
                               ("free_count", free_count, (1,))):
            _int32(name, t, shape, index)
        if not 1 <= B <= MAX_BATCH or M < 1 or N < 1 or max_new < 1 or not 16 <= page_size <= 1024 or \
                page_size & (page_size - 1) or max(N, M) * page_size >= 1 << 31 or B * max_new >= 1 << 31:
            raise SpecVerifyError(f"invalid sizes: batch={B} (1 to {MAX_BATCH}) num_pages={N} max_pages={M} "
                                  f"max_new={max_new} page_size={page_size} (a power of two from 16 to 1024)")
        self.device, self._index = lengths.device, index
        self.batch, self.max_pages, self.num_pages = B, M, N
        self.page_size, self.max_new = page_size, max_new
        self.lengths, self.counts, self.held = lengths, counts, held
        self.block_table, self.free_pages, self.free_count = block_table, free_pages, free_count
        self.prefix_len = 0
        # what the last plan wrote: the leading [B, n] of these
        self._slots = torch.full((B * max_new,), -1, dtype=torch.int32, device=self.device)
        self._positions = torch.full((B * max_new,), -1, dtype=torch.int32, device=self.device)
        self._views = {}
        self.slots, self.positions = self._view(max_new)
        self._tables = Tables(lengths.data_ptr(), counts.data_ptr(), held.data_ptr(), block_table.data_ptr(),
                              free_pages.data_ptr(), free_count.data_ptr(), B, M, N, page_size)
        self._tables_ref = ctypes.byref(self._tables)
        self._workspaces, self._workspace_of = {}, {}

    def _view(self, n: int) -> Tuple[torch.Tensor, torch.Tensor]:
        got = self._views.get(n)
        if got is None:
            if not 1 <= n <= self.max_new:
                raise SpecVerifyError(f"{n} new tokens: 1 to max_new={self.max_new}")
            size = self.batch * n
            got = (self._slots[:size].view(self.batch, n), self._positions[:size].view(self.batch, n))
            self._views[n] = got
        return got

    def reset(self) -> None:
        """No sequence holds a page, and all pages but the prefix's are free.  (With a prefix on pages of the program's
        choice not in a captured graph: sorting the pages clears memory in ways that replays do not repeat.)"""
        if not self._prefix_first and torch.cuda.is_current_stream_capturing():
            raise SpecVerifyError("reset() with a prefix on pages of the program's choice cannot be captured")
        _call(self._index, self._lib.spec_cache_init, "spec_cache_init", self._tables_ref,
              self.prefix_table.numel() if self._prefix_first else 0)
        if not self._prefix_first:
            # the prefix's pages, wherever they are, out of the stack
            page = torch.arange(self.num_pages - 1, -1, -1, dtype=torch.int32, device=self.device)
            taken = torch.isin(page, self.prefix_table)
            order = torch.argsort(taken.to(torch.int32), stable=True)
            self.free_pages.copy_(torch.where(taken[order], -1, page[order]))
            self.free_count.copy_((~taken).sum())

    def set_prefix(self, length: int) -> None:
        """All sequences begin with the ``length`` tokens in the prefix's pages (``prefix_table``: the caches' first
        ones, token i in slot i, unless the program named others).  Graphs captured before go on with the length that
        was set then."""
        if not 0 <= length <= self.prefix_table.numel() * self.page_size:
            raise SpecVerifyError(f"a prefix of {length} tokens does not fit {self.prefix_table.numel()} pages")
        self.prefix_len = length

    def new_storage(self, kv_heads: int, head_dim: int, dtype) -> Tuple[torch.Tensor, torch.Tensor]:
        """Key and value caches of one layer, ``[num_pages, kv_heads, page_size, head_dim]`` (uninitialised)."""
        if dtype not in DTYPE_CODES:
            raise SpecVerifyError(f"caches hold one of {list(DTYPE_CODES)}; got {dtype}")
        shape = (self.num_pages, kv_heads, self.page_size, head_dim)
        return tuple(torch.empty(shape, dtype=dtype, device=self.device) for _ in range(2))

    def plan(self, n: int, *, new_tokens: Optional[torch.Tensor] = None, accepted_len: Optional[torch.Tensor] = None,
             release: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Plans the next step of up to ``n`` new tokens a sequence (spec_cache_plan).

        ``release[b]`` nonzero: the sequence has ended, its pages are free and it starts anew.  Otherwise
        ``accepted_len[b] + 1`` of its last plan's tokens stay (all of them without ``accepted_len``), and
        ``new_tokens[b]`` (n without it) get slots.  All are int32 [B] on the GPU.  Returns ``(slots, positions)``,
        int32 [B, n], -1 behind a sequence's last token: views of static buffers that the next plan overwrites.
        A sequence that could not be served has ``counts[b] == -1`` and no slots.
        """
        slots, positions = self._views.get(n) or self._view(n)
        index, shape = self._index, (self.batch,)
        if accepted_len is not None:
            _int32("accepted_len", accepted_len, shape, index)
        if new_tokens is not None:
            _int32("new_tokens", new_tokens, shape, index)
        if release is not None:
            _int32("release", release, shape, index)
        _call(index, self._lib.spec_cache_plan, "spec_cache_plan", self._tables_ref, _ptr(accepted_len),
              _ptr(new_tokens), _ptr(release), n, self.prefix_len, slots.data_ptr(), positions.data_ptr())
        self.slots, self.positions = slots, positions
        return slots, positions

    def _described(self, k_cache: torch.Tensor) -> None:
        """Slots and block tables count in the tables' pages: a cache has such pages, and as many or more."""
        if k_cache.dim() != 4 or k_cache.shape[2] != self.page_size or k_cache.shape[0] < self.num_pages:
            raise SpecVerifyError(f"the tables are of {self.num_pages} pages of {self.page_size} tokens; the cache is "
                                  f"{list(k_cache.shape)}")

    def append(self, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor) -> None:
        """The planned tokens' keys and values ``[B, n, kv_heads, head_dim]`` into their slots."""
        self._described(k_cache)
        append(k, v, k_cache, v_cache, self.slots)

    def append_prefix(self, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                      start: int = 0) -> None:
        """Keys and values ``[1, n, kv_heads, head_dim]`` of the prefix's tokens from ``start`` on."""
        self._described(k_cache)
        end = start + k.shape[1]
        if start < 0 or end > self.prefix_table.numel() * self.page_size:
            raise SpecVerifyError(f"prefix tokens {start} to {end} do not fit {self.prefix_table.numel()} pages")
        pages = self.prefix_table[torch.arange(start, end, device=self.device) // self.page_size]
        at = torch.arange(start, end, device=self.device, dtype=torch.int32) % self.page_size
        append(k, v, k_cache, v_cache, (pages * self.page_size + at)[None])

    def _workspace(self, *sizes: int) -> torch.Tensor:
        """One for each power of two of bytes, and none is given up: captured graphs may hold it."""
        size = 1 << (attend_workspace_bytes(*sizes) - 1).bit_length()
        if size not in self._workspaces:
            self._workspaces[size] = torch.empty(size, dtype=torch.uint8, device=self.device)
        return self._workspaces[size]

    def attend(self, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, *, scale: Optional[float] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of the planned tokens ``q [B, n, q_heads, head_dim]`` (see attend()).  The workspaces are kept
        and shared by all layers: calls have to be ordered."""
        if q.dim() != 4:
            raise SpecVerifyError(f"q must be [batch, tokens, q_heads, head_dim]; it is {list(q.shape)}")
        self._described(k_cache)
        key = (q.shape, k_cache.shape[1])
        workspace = self._workspace_of.get(key)
        if workspace is None:
            workspace = self._workspace_of[key] = self._workspace(*q.shape[:3], k_cache.shape[1], q.shape[3])
        return attend(q, k_cache, v_cache, self.block_table, self.lengths, self.counts, prefix_table=self.prefix_table,
                      prefix_len=self.prefix_len, scale=scale, out=out, workspace=workspace)
