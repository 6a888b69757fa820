"""Thin ctypes binding of the attention-layer calls (``include/treewy_attn.h``) and one attention
layer's speculative round.

Function names and argument order follow the C header; as in ``binding``, torch tensors supply
device memory and the stream, every computation runs in the library's CUDA kernels, and outputs are
written in place.  Devices, shapes, strides and types are checked here (``ValueError``), sizes and alignment by
the library (``binding.TreewyError``).
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import binding as tw
from .binding import Tree

SEQ_BAD_PAGE, SEQ_BAD_LENGTH, SEQ_BAD_POSITION = 64, 128, 256


class KVCacheStruct(ctypes.Structure):
    """Mirror of ``treewy_kv_cache_t``."""
    _fields_ = [
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("stride_page", ctypes.c_int64), ("stride_slot", ctypes.c_int64), ("stride_head", ctypes.c_int64),
        ("page_table", ctypes.c_void_p), ("context_len", ctypes.c_void_p),
        ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
        ("H_kv", ctypes.c_int32), ("d_head", ctypes.c_int32),
    ]


class RopeStruct(ctypes.Structure):
    """Mirror of ``treewy_rope_t``."""
    _fields_ = [
        ("cos_sin", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("pair_axis", ctypes.c_void_p),
        ("n_axes", ctypes.c_int32), ("max_positions", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
    ]


_lib = None


def load_library():
    """The library with the attention calls' prototypes set; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    lib = tw.load_library()
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    cache, rope, tree = ctypes.POINTER(KVCacheStruct), ctypes.POINTER(RopeStruct), vp
    lib.treewy_rope.argtypes = [rope, vp, i64, vp, i64, i32, i32, i32, i32, ctypes.c_int, vp, vp]
    lib.treewy_rope_rows.argtypes = [rope, i32, i32, vp, vp, i64, vp, i64, i32, i32, i32, ctypes.c_int, vp, vp]
    lib.treewy_kv_append.argtypes = [cache, rope, i32, i32, vp, vp, i64, vp, i64, i32, vp, i64, vp, i64, ctypes.c_int, vp, vp]
    verify = [cache, tree, vp, i64, vp, i64, vp, i64, i32, f32, vp, i32, ctypes.c_int, vp, vp, ctypes.c_size_t, vp, vp]
    lib.treewy_attn_verify.argtypes = verify
    lib.treewy_attn_verify_generic.argtypes = verify
    lib.treewy_kv_commit.argtypes = [cache, tree, vp, i64, vp, i64, vp, ctypes.c_int, vp, vp, vp]
    for fn in (lib.treewy_rope, lib.treewy_rope_rows, lib.treewy_kv_append, lib.treewy_attn_verify, lib.treewy_attn_verify_generic,
               lib.treewy_kv_commit):
        fn.restype = ctypes.c_int
    lib.treewy_attn_workspace.argtypes = [cache, tree, i32, i32, ctypes.c_int]
    lib.treewy_attn_workspace.restype = ctypes.c_size_t
    _lib = lib
    return lib


def _require(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _int32(t: torch.Tensor | None, n: int, what: str, dev: int) -> int | None:
    """Checks an optional int32 array; returns its address."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous int32 tensor of at least {n} elements wanted")
    if t.get_device() != dev:
        raise ValueError(f"{what}: on another device")
    return t.data_ptr()


def _rows(x: torch.Tensor, T: int, H: int, d: int, dtype: torch.dtype, what: str, dev: int) -> int:
    """Checks packed rows [T, H, d] (heads contiguous, tokens at any distance); returns that distance."""
    try:
        (n, h, c), (row, head, one) = x.shape, x.stride()
    except ValueError:
        n = h = c = row = head = one = -1
    if x.dtype is not dtype or h != H or c != d or n < T:
        raise ValueError(f"{what}: {dtype} [{T}, {H}, {d}] wanted, got {x.dtype} {list(x.shape)}")
    if (one != 1 and d > 1) or (head != d and H > 1):
        raise ValueError(f"{what}: the heads of a token have to be contiguous")
    if x.get_device() != dev:
        raise ValueError(f"{what}: on another device")
    return row if n > 1 else H * d


def _on_gpu(dev: int, work: int) -> None:
    """A call that has something to do wants a GPU's memory (dev: torch's number of it, negative for the host)."""
    if dev < 0 and work > 0:
        raise ValueError("tensors in a GPU's memory wanted")


# (These calls are a few microseconds of GPU work in a decoding step, so the host side is kept short: raw addresses,
# structs built once where the object is kept, the stream's handle without a Stream object.)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, x: torch.Tensor) -> int | None:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and x.is_cuda:
        return _raw_stream(x.get_device())
    return torch.cuda.current_stream().cuda_stream


_TREE = struct.Struct("4i6P")                         # treewy_tree_t, which takes ctypes twice as long to fill
assert _TREE.size == ctypes.sizeof(tw.TreeStruct)


def _tree_struct(tree: Tree, dev: int) -> bytes:
    """The tree as the C calls take it.  Its arrays may be replaced between calls, so what is read of it is checked for each."""
    offsets, mask = tree.node_offsets, tree.anc_mask
    if offsets.dtype is not torch.int32 or offsets.numel() <= tree.B or not offsets.is_contiguous() or offsets.get_device() != dev:
        raise ValueError("tree: node_offsets: contiguous int32 [B + 1] on the cache's device wanted")
    if mask.dtype is not torch.int64 or mask.numel() < tree.T or not mask.is_contiguous() or mask.get_device() != dev:
        raise ValueError("tree: anc_mask: contiguous int64 [T] on the cache's device wanted")
    return _TREE.pack(tree.B, tree.T, tree.H_v, tree.max_nodes, offsets.data_ptr(), 0, 0, mask.data_ptr(), 0, 0)


class KVCache:
    """A paged cache (``treewy_kv_cache_t``): k, v [n_pages, page_size, H_kv, d_head] in any order of
    strides with d_head innermost (the same for both), page_table [B, max_pages] and context_len [B] int32.
    The object refers to the tensors' memory: contents may change between calls, storage may not."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, context_len: torch.Tensor):
        _require(k.dtype in tw._DTYPES and v.dtype == k.dtype, "k, v: both bfloat16 or both float32 wanted")
        _require(k.dim() == 4 and k.shape == v.shape and k.stride() == v.stride(), "k, v: same 4-d shape and strides wanted")
        _require(k.shape[3] == 1 or k.stride(3) == 1, "k, v: d_head has to be contiguous")
        _require(page_table.dim() == 2 and page_table.is_contiguous() and page_table.dtype == torch.int32,
                 "page_table: contiguous int32 [B, max_pages] wanted")
        self._dev = k.get_device()
        _int32(context_len, page_table.shape[0], "context_len", self._dev)
        _require(page_table.device == k.device == v.device == context_len.device, "cache tensors on different devices")
        self.k, self.v, self.page_table, self.context_len = k, v, page_table, context_len
        self.B, self.max_pages = (int(n) for n in page_table.shape)
        self.n_pages, self.page_size, self.H_kv, self.d_head = (int(n) for n in k.shape)
        self.dtype = k.dtype
        self._dt = tw._DTYPES[k.dtype]
        self._struct = KVCacheStruct(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2),
                                     page_table.data_ptr(), context_len.data_ptr(), self.n_pages, self.page_size,
                                     self.max_pages, self.H_kv, self.d_head)
        self._ref = ctypes.byref(self._struct)


class Rope:
    """Rotary positions (``treewy_rope_t``): cos_sin [max_positions, rot_dim] fp32 (cosines, then sines),
    positions [n_axes, T] (or [T]) int32, pair_axis [rot_dim / 2] uint8 (None: one axis)."""

    def __init__(self, cos_sin: torch.Tensor, positions: torch.Tensor, pair_axis: torch.Tensor | None = None,
                 interleaved: bool = False):
        _require(cos_sin.dtype == torch.float32 and cos_sin.dim() == 2 and cos_sin.is_contiguous(),
                 "cos_sin: contiguous float32 [max_positions, rot_dim] wanted")
        if positions.dim() == 1:
            positions = positions[None]
        _require(positions.dtype == torch.int32 and positions.dim() == 2 and positions.is_contiguous(),
                 "positions: contiguous int32 [n_axes, T] wanted")
        _require(pair_axis is None or (pair_axis.dtype == torch.uint8 and pair_axis.is_contiguous()
                                       and pair_axis.numel() == cos_sin.shape[1] // 2),
                 "pair_axis: uint8 [rot_dim / 2] wanted")
        _require(cos_sin.device == positions.device and (pair_axis is None or pair_axis.device == cos_sin.device),
                 "rotary tensors on different devices")
        self.cos_sin, self.positions, self.pair_axis = cos_sin, positions, pair_axis
        self._dev = cos_sin.get_device()
        self.T = int(positions.shape[1])
        self._struct = RopeStruct(cos_sin.data_ptr(), positions.data_ptr(),
                                  None if pair_axis is None else pair_axis.data_ptr(), int(positions.shape[0]),
                                  int(cos_sin.shape[0]), int(cos_sin.shape[1]), int(bool(interleaved)))
        self._ref = ctypes.byref(self._struct)


def treewy_rope(rope: Rope, x: torch.Tensor, y: torch.Tensor, inverse: bool = False,
                row_status: torch.Tensor | None = None, stream=None) -> None:
    """y [T, H, d] <- x rotated by its tokens' positions (inverse: the other way, which is the backward pass)."""
    T, H, d = x.shape
    dt = tw._DTYPES.get(x.dtype)
    if T != rope.T or dt is None:
        raise ValueError(f"x: bfloat16 or float32, {rope.T} tokens as rope.positions has, wanted")
    dev = rope._dev
    _on_gpu(dev, T)
    ld_x, ld_y = _rows(x, T, H, d, x.dtype, "x", dev), _rows(y, T, H, d, x.dtype, "y", dev)
    tw._call("treewy_rope", load_library().treewy_rope, rope._ref, x.data_ptr(), ld_x, y.data_ptr(), ld_y, T, H, d,
             int(inverse), dt, _int32(row_status, 1, "row_status", dev), _stream(stream, x))


def treewy_rope_rows(rope: Rope, row_offsets: torch.Tensor, x: torch.Tensor, y: torch.Tensor, inverse: bool = False,
                     seq_status: torch.Tensor | None = None, stream=None) -> None:
    """treewy_rope for the packed rows of the sequences at row_offsets [B + 1]: a position out of range flags its sequence."""
    T, H, d = x.shape
    B, dt = row_offsets.numel() - 1, tw._DTYPES.get(x.dtype)
    if T != rope.T or dt is None or B < 0:
        raise ValueError(f"x: bfloat16 or float32, {rope.T} tokens as rope.positions has, wanted; row_offsets: B + 1 of them")
    dev = rope._dev
    _on_gpu(dev, T)
    ld_x, ld_y = _rows(x, T, H, d, x.dtype, "x", dev), _rows(y, T, H, d, x.dtype, "y", dev)
    tw._call("treewy_rope_rows", load_library().treewy_rope_rows, rope._ref, B, T, _int32(row_offsets, B + 1, "row_offsets", dev),
             x.data_ptr(), ld_x, y.data_ptr(), ld_y, H, d, int(inverse), dt, _int32(seq_status, B, "seq_status", dev), _stream(stream, x))


def treewy_kv_append(cache: KVCache, row_offsets: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                     rope: Rope | None = None, q: torch.Tensor | None = None, q_out: torch.Tensor | None = None,
                     seq_status: torch.Tensor | None = None, stream=None) -> None:
    """Rows k, v [T, H_kv, d] of the sequences at row_offsets [B + 1] go behind context_len of each sequence's
    cache, k rotated on the way; q [T, H_q, d], when given, is rotated into q_out in the same pass."""
    T, H_kv, d, dtype, dev = k.shape[0], cache.H_kv, cache.d_head, cache.dtype, cache._dev
    if rope is not None and (rope.T != T or rope._dev != dev):
        raise ValueError("rope: as many positions as rows, on the cache's device, wanted")
    _on_gpu(dev, T)
    ld_k, ld_v = _rows(k, T, H_kv, d, dtype, "k", dev), _rows(v, T, H_kv, d, dtype, "v", dev)
    H_q = ld_q = ld_qo = 0
    q_at = qo_at = None
    if q is not None:
        if q_out is None:
            raise ValueError("q_out: wanted with q")
        H_q = q.shape[1]
        ld_q, ld_qo = _rows(q, T, H_q, d, dtype, "q", dev), _rows(q_out, T, H_q, d, dtype, "q_out", dev)
        q_at, qo_at = q.data_ptr(), q_out.data_ptr()
    tw._call("treewy_kv_append", load_library().treewy_kv_append, cache._ref, None if rope is None else rope._ref, cache.B, T,
             _int32(row_offsets, cache.B + 1, "row_offsets", dev), k.data_ptr(), ld_k, v.data_ptr(), ld_v, H_q, q_at, ld_q, qo_at,
             ld_qo, cache._dt, _int32(seq_status, cache.B, "seq_status", dev), _stream(stream, k))


def attn_workspace(cache: KVCache, tree: Tree, H_q: int, shared_len: int = 0) -> torch.Tensor:
    """A workspace for ``treewy_attn_verify`` calls of these sizes (one per call in flight)."""
    n = load_library().treewy_attn_workspace(cache._ref, _tree_struct(tree, cache._dev), H_q, shared_len, cache._dt)
    return torch.empty((max(int(n), 16),), dtype=torch.uint8, device=cache.k.device)


def treewy_attn_verify(cache: KVCache, tree: Tree, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float,
                       O: torch.Tensor, workspace: torch.Tensor, shared_pages: torch.Tensor | None = None,
                       shared_len: int = 0, seq_status: torch.Tensor | None = None, stream=None,
                       generic: bool = False) -> None:
    """O [T, H_q, d] <- attention of every draft node (q, k, v: packed rows) over its sequence's cached tokens
    and its ancestors."""
    lib = load_library()
    T, H_kv, d, dtype, dev = tree.T, cache.H_kv, cache.d_head, cache.dtype, cache._dev
    _on_gpu(dev, T)
    H_q = q.shape[1]
    if tree.B != cache.B:
        raise ValueError("tree: another number of sequences than the cache's page table")
    ld_q = _rows(q, T, H_q, d, dtype, "q", dev)
    ld_k, ld_v = _rows(k, T, H_kv, d, dtype, "k", dev), _rows(v, T, H_kv, d, dtype, "v", dev)
    if _rows(O, T, H_q, d, dtype, "O", dev) != H_q * d and T > 0:
        raise ValueError("O: contiguous rows wanted")
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous and on the cache's device wanted")
    fn = lib.treewy_attn_verify_generic if generic else lib.treewy_attn_verify
    tw._call("treewy_attn_verify_generic" if generic else "treewy_attn_verify", fn, cache._ref, _tree_struct(tree, dev),
             q.data_ptr(), ld_q, k.data_ptr(), ld_k, v.data_ptr(), ld_v, H_q, scale,
             _int32(shared_pages, shared_len // cache.page_size, "shared_pages", dev), shared_len, cache._dt, O.data_ptr(),
             workspace.data_ptr(), workspace.numel() * workspace.element_size(), _int32(seq_status, cache.B, "seq_status", dev),
             _stream(stream, q))


def treewy_kv_commit(cache: KVCache, tree: Tree, k: torch.Tensor, v: torch.Tensor, accepted: torch.Tensor,
                     new_context_len: torch.Tensor | None = None, seq_status: torch.Tensor | None = None,
                     stream=None) -> None:
    """The accepted path's rows of k, v [T, H_kv, d] go behind context_len; new_context_len [B] receives the
    lengths after it."""
    if tree.B != cache.B:
        raise ValueError("tree: another number of sequences than the cache's page table")
    B, T, H_kv, d, dtype, dev = cache.B, tree.T, cache.H_kv, cache.d_head, cache.dtype, cache._dev
    _on_gpu(dev, B)
    ld_k, ld_v = _rows(k, T, H_kv, d, dtype, "k", dev), _rows(v, T, H_kv, d, dtype, "v", dev)
    tw._call("treewy_kv_commit", load_library().treewy_kv_commit, cache._ref, _tree_struct(tree, dev), k.data_ptr(), ld_k, v.data_ptr(),
             ld_v, _int32(accepted, B, "accepted", dev), cache._dt, _int32(new_context_len, B, "new_context_len", dev),
             _int32(seq_status, B, "seq_status", dev), _stream(stream, k))


class AttentionLayer:
    """One attention layer's side of a speculative round, on the current stream: the paged cache, the rotary table and
    a workspace stay with the layer; each call takes the round's packed rows.  The cache's ``context_len`` is
    advanced by ``commit`` and ``append_and_attend``.  Layers of one model that share a context_len array leave that to the
    last of them, since all of a round write at the same place: the others pass advance=False.

    seq_status [B], zeroed by the caller ahead of a round and passed to all of its calls, receives their flags; without it
    the layer keeps its own.  A sequence that is flagged in it, by whichever layer, keeps its length, and its rows of the
    outputs mean nothing."""

    def __init__(self, cache: KVCache, H_q: int, cos_sin: torch.Tensor, pair_axis: torch.Tensor | None = None,
                 interleaved: bool = False, scale: float | None = None):
        if H_q < 1 or H_q % cache.H_kv != 0:
            raise ValueError("H_q: a multiple of the cache's heads wanted")
        self.cache, self.H_q = cache, H_q
        self.cos_sin, self.pair_axis, self.interleaved = cos_sin, pair_axis, interleaved
        self.scale = cache.d_head ** -0.5 if scale is None else scale
        self._len = cache.context_len.view(-1)[:cache.B]
        self._new_len = torch.empty_like(self._len)
        self._own = torch.zeros_like(self._len)    # status words of a round whose caller has none
        self._round = None                         # those of the round that verify began
        # the cache with the token that append_and_attend has just written
        self._ahead = KVCache(cache.k, cache.v, cache.page_table, self._new_len)
        self._unseen = None                        # ancestor masks of nodes that see no draft row
        self._ws, self._ws_for = None, None

    def _workspace(self, tree: Tree, shared_len: int) -> torch.Tensor:
        sizes = (tree.B, tree.T, tree.max_nodes, shared_len)
        if self._ws_for != sizes:
            ws = attn_workspace(self.cache, tree, self.H_q, shared_len)
            if self._ws is None or ws.numel() > self._ws.numel():
                self._ws = ws
            self._ws_for = sizes
        return self._ws

    def _out(self, q: torch.Tensor) -> torch.Tensor:
        return torch.empty((q.shape[0], self.H_q, self.cache.d_head), dtype=q.dtype, device=q.device)

    def _rope(self, positions: torch.Tensor) -> Rope:
        return Rope(self.cos_sin, positions, self.pair_axis, self.interleaved)

    def _begin(self, tree: Tree, seq_status: torch.Tensor | None) -> torch.Tensor:
        """The status words of a round that begins."""
        if tree.B != self.cache.B:
            raise ValueError("tree: another number of sequences than the cache's page table")
        _int32(seq_status, self.cache.B, "seq_status", self.cache._dev)
        self._round = self._own.zero_() if seq_status is None else seq_status.view(-1)[:self.cache.B]
        return self._round

    def verify(self, tree: Tree, positions: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
               seq_status: torch.Tensor | None = None, shared_pages: torch.Tensor | None = None,
               shared_len: int = 0) -> torch.Tensor:
        """Rotates q and k in place (keep k and v until commit) and returns the attention's output for every node."""
        status = self._begin(tree, seq_status)
        rope = self._rope(positions)
        offsets = tree.node_offsets[:tree.B + 1]
        treewy_rope_rows(rope, offsets, q, q, seq_status=status)
        treewy_rope_rows(rope, offsets, k, k, seq_status=status)
        O = self._out(q)
        treewy_attn_verify(self.cache, tree, q, k, v, self.scale, O, self._workspace(tree, shared_len), shared_pages,
                           shared_len, status)
        return O

    def commit(self, tree: Tree, k: torch.Tensor, v: torch.Tensor, accepted: torch.Tensor,
               seq_status: torch.Tensor | None = None, advance: bool = True) -> None:
        """The accepted path's keys and values enter the cache.  Sequences that verify or this call has flagged keep their
        length (what is written behind it does not count)."""
        begun = self._round
        status = self._begin(tree, seq_status) if begun is None or seq_status is not None else begun
        if begun is not None and begun.data_ptr() != status.data_ptr():
            status |= begun
        self._round = None
        treewy_kv_commit(self.cache, tree, k, v, accepted, self._new_len, status)
        if advance:
            torch.where(status == 0, self._new_len, self._len, out=self._len)

    def append_and_attend(self, tree: Tree, positions: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                          seq_status: torch.Tensor | None = None, advance: bool = True,
                          shared_pages: torch.Tensor | None = None, shared_len: int = 0) -> torch.Tensor:
        """Ordinary decoding: one token a sequence, written to the cache (rotated on the way) and attended from there."""
        if tree.T != tree.B:
            raise ValueError("tree: one node a sequence wanted")
        status = self._begin(tree, seq_status)
        self._round = None
        q_out, O = self._out(q), self._out(q)
        treewy_kv_append(self.cache, tree.node_offsets, k, v, self._rope(positions), q, q_out, status)
        # The token is in the cache already: it is seen there and not as a draft row.  One node at most, so that a sequence with
        # none or with several is flagged.
        if shared_len > 0:                         # (with the token the attention would take one that is a token short)
            status |= (self._len < shared_len) * SEQ_BAD_LENGTH
        torch.add(self._len, 1, out=self._new_len)
        if self._unseen is None or self._unseen.numel() < tree.T:
            self._unseen = torch.zeros((tree.T,), dtype=torch.int64, device=q.device)
        alone = Tree(**{**vars(tree), "anc_mask": self._unseen, "max_nodes": 1})
        treewy_attn_verify(self._ahead, alone, q_out, k, v, self.scale, O, self._workspace(alone, shared_len), shared_pages,
                           shared_len, status)
        if advance:
            self._len.add_(status == 0)
        return O
