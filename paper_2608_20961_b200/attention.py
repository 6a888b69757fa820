"""Thin ctypes binding of the attention-layer calls (``include/treewy_attn.h``, ``include/treewy_prompt.h``) and one
attention layer's steps: a speculative round, a prompt or a piece of one, single tokens.

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

SEQ_BAD_PAGE, SEQ_BAD_LENGTH, SEQ_BAD_POSITION, SEQ_NO_PAGES = 64, 128, 256, 512


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


class HeadNormStruct(ctypes.Structure):
    """Mirror of ``treewy_head_norm_t``."""
    _fields_ = [("weight", ctypes.c_void_p), ("weight_dtype", ctypes.c_int), ("eps", ctypes.c_float), ("plus_one", ctypes.c_int32)]


class PagePoolStruct(ctypes.Structure):
    """Mirror of ``treewy_page_pool_t``."""
    _fields_ = [("page_table", ctypes.c_void_p), ("free_pages", ctypes.c_void_p), ("free_count", ctypes.c_void_p),
                ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32)]


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
    norm, pool, size, dt = ctypes.POINTER(HeadNormStruct), ctypes.POINTER(PagePoolStruct), ctypes.c_size_t, ctypes.c_int
    lib.treewy_norm_rope.argtypes = [norm, rope, i32, i32, vp, vp, i64, vp, i64, i32, i32, dt, vp, vp]
    lib.treewy_norm_rope_backward.argtypes = [norm, rope, vp, i64, vp, i64, vp, i64, vp, i32, i32, i32, dt, vp, size, vp, vp]
    lib.treewy_kv_append_norm.argtypes = [cache, rope, norm, norm, i32, i32, vp, vp, i64, vp, i64, i32, vp, i64, vp, i64, dt, vp, vp]
    chunk = [cache, i32, i32, vp, vp, i64, i32, f32, i32, i32, dt, vp, vp, size, vp, vp]
    lib.treewy_attn_chunk.argtypes = chunk
    lib.treewy_attn_chunk_generic.argtypes = chunk
    lib.treewy_pages_reserve.argtypes = [pool, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.treewy_pages_release.argtypes = [pool, i32, vp, vp, vp, vp]
    for fn in (lib.treewy_norm_rope, lib.treewy_norm_rope_backward, lib.treewy_kv_append_norm, lib.treewy_attn_chunk,
               lib.treewy_attn_chunk_generic, lib.treewy_pages_reserve, lib.treewy_pages_release):
        fn.restype = ctypes.c_int
    lib.treewy_norm_rope_workspace.argtypes = [i32, i32, i32, dt]
    lib.treewy_attn_chunk_workspace.argtypes = [cache, i32, i32, i32, i32, i32, dt]
    lib.treewy_norm_rope_workspace.restype = lib.treewy_attn_chunk_workspace.restype = size
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
    return row if n > 1 else -(-H * d * x.element_size() // 16) * 16 // x.element_size()  # (one row's does not count, but has to be a legal one)


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
    _on_gpu(dev, T if seq_status is None else cache.B)
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


class HeadNorm:
    """Root-mean-square norm of each head (``treewy_head_norm_t``): weight [d_head] bfloat16 or float32, the same for all heads;
    plus_one: 1 + weight is meant.  The object refers to the weight's memory."""

    def __init__(self, weight: torch.Tensor, eps: float = 1e-6, plus_one: bool = False):
        _require(weight.dtype in tw._DTYPES and weight.dim() == 1 and weight.is_contiguous(),
                 "weight: contiguous bfloat16 or float32 [d_head] wanted")
        self.weight, self.eps, self.plus_one, self.d = weight, eps, plus_one, int(weight.numel())
        self._dev = weight.get_device()
        self._struct = HeadNormStruct(weight.data_ptr(), tw._DTYPES[weight.dtype], eps, int(bool(plus_one)))
        self._ref = ctypes.byref(self._struct)


def _norm(norm: HeadNorm | None, d: int, what: str, dev: int):
    if norm is None:
        return None
    if norm.d != d or norm._dev != dev:
        raise ValueError(f"{what}: a weight of {d} elements on the rows' device wanted")
    return norm._ref


def _norm_rows(norm: HeadNorm, rope: Rope | None, x: torch.Tensor):
    """What the norm's calls check of x [T, H, d]."""
    if x.dim() != 3 or x.dtype not in tw._DTYPES:
        raise ValueError("x: bfloat16 or float32 [T, H, d] wanted")
    T, H, d = x.shape
    dev = x.get_device()
    if rope is not None and (rope.T != T or rope._dev != dev):
        raise ValueError("rope: as many positions as rows, on their device, wanted")
    return T, H, d, dev, _norm(norm, d, "norm", dev)


def treewy_norm_rope(norm: HeadNorm, rope: Rope | None, x: torch.Tensor, y: torch.Tensor, row_offsets: torch.Tensor | None = None,
                     seq_status: torch.Tensor | None = None, stream=None) -> None:
    """y [T, H, d] <- x, each head normalised and then rotated (rope None: normalised only).  With row_offsets [B + 1] a
    position out of range flags its sequence, else the one word of seq_status."""
    T, H, d, dev, ref = _norm_rows(norm, rope, x)
    B = 0 if row_offsets is None else row_offsets.numel() - 1
    if B < 0:
        raise ValueError("row_offsets: B + 1 of them wanted")
    _on_gpu(dev, T)
    ld_x, ld_y = _rows(x, T, H, d, x.dtype, "x", dev), _rows(y, T, H, d, x.dtype, "y", dev)
    tw._call("treewy_norm_rope", load_library().treewy_norm_rope, ref, None if rope is None else rope._ref, B, T,
             _int32(row_offsets, B + 1, "row_offsets", dev), x.data_ptr(), ld_x, y.data_ptr(), ld_y, H, d, tw._DTYPES[x.dtype],
             _int32(seq_status, B or 1, "seq_status", dev), _stream(stream, x))


def norm_rope_workspace(x: torch.Tensor) -> torch.Tensor:
    """A workspace for ``treewy_norm_rope_backward`` calls on rows like x [T, H, d] (one per call in flight)."""
    T, H, d = x.shape
    n = load_library().treewy_norm_rope_workspace(T, H, d, tw._DTYPES[x.dtype])
    return torch.empty((max(int(n), 16),), dtype=torch.uint8, device=x.device)


def treewy_norm_rope_backward(norm: HeadNorm, rope: Rope | None, x: torch.Tensor, dy: torch.Tensor, dx: torch.Tensor,
                              dweight: torch.Tensor, workspace: torch.Tensor, row_status: torch.Tensor | None = None,
                              stream=None) -> None:
    """dx [T, H, d] and dweight [d] (float32) <- the gradients of treewy_norm_rope's input and weight, given that of its
    output.  dx may be x or dy."""
    T, H, d, dev, ref = _norm_rows(norm, rope, x)
    _on_gpu(dev, 1)
    ld_x, ld_dy, ld_dx = (_rows(r, T, H, d, x.dtype, what, dev) for r, what in ((x, "x"), (dy, "dy"), (dx, "dx")))
    if dweight.dtype is not torch.float32 or dweight.numel() != d or not dweight.is_contiguous() or dweight.get_device() != dev:
        raise ValueError(f"dweight: contiguous float32 [{d}] on the rows' device wanted")
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous and on the rows' device wanted")
    tw._call("treewy_norm_rope_backward", load_library().treewy_norm_rope_backward, ref, None if rope is None else rope._ref,
             x.data_ptr(), ld_x, dy.data_ptr(), ld_dy, dx.data_ptr(), ld_dx, dweight.data_ptr(), T, H, d, tw._DTYPES[x.dtype],
             workspace.data_ptr(), workspace.numel() * workspace.element_size(), _int32(row_status, 1, "row_status", dev),
             _stream(stream, x))


def treewy_kv_append_norm(cache: KVCache, row_offsets: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_norm: HeadNorm | None,
                          rope: Rope | None = None, q: torch.Tensor | None = None, q_out: torch.Tensor | None = None,
                          q_norm: HeadNorm | None = None, seq_status: torch.Tensor | None = None, stream=None) -> None:
    """treewy_kv_append with the keys' (and queries') heads normalised ahead of the rotation."""
    T, H_kv, d, dtype, dev = k.shape[0], cache.H_kv, cache.d_head, cache.dtype, cache._dev
    if rope is not None and (rope.T != T or rope._dev != dev):
        raise ValueError("rope: as many positions as rows, on the cache's device, wanted")
    _on_gpu(dev, T if seq_status is None else cache.B)
    ld_k, ld_v = _rows(k, T, H_kv, d, dtype, "k", dev), _rows(v, T, H_kv, d, dtype, "v", dev)
    H_q = ld_q = ld_qo = 0
    q_at = qo_at = None
    if q is not None:
        if q_out is None:
            raise ValueError("q_out: wanted with q")
        H_q = q.shape[1]
        ld_q, ld_qo = _rows(q, T, H_q, d, dtype, "q", dev), _rows(q_out, T, H_q, d, dtype, "q_out", dev)
        q_at, qo_at = q.data_ptr(), q_out.data_ptr()
    tw._call("treewy_kv_append_norm", load_library().treewy_kv_append_norm, cache._ref, None if rope is None else rope._ref,
             _norm(q_norm, d, "q_norm", dev), _norm(k_norm, d, "k_norm", dev), cache.B, T,
             _int32(row_offsets, cache.B + 1, "row_offsets", dev), k.data_ptr(), ld_k, v.data_ptr(), ld_v, H_q, q_at, ld_q, qo_at,
             ld_qo, cache._dt, _int32(seq_status, cache.B, "seq_status", dev), _stream(stream, k))


def _window(window: int, sinks: int) -> None:
    """(ctypes would cut them to 32 bits without a word; the library refuses negative ones.)"""
    if not (-1 << 31 <= window < 1 << 31 and -1 << 31 <= sinks < 1 << 31):
        raise ValueError("window, sinks: 32 bits wanted")


def attn_chunk_workspace(cache: KVCache, T: int, H_q: int, window: int = 0, sinks: int = 0) -> torch.Tensor:
    """A workspace for ``treewy_attn_chunk`` calls of up to T rows with this window (one per call in flight)."""
    _window(window, sinks)
    n = load_library().treewy_attn_chunk_workspace(cache._ref, cache.B, T, H_q, window, sinks, cache._dt)
    return torch.empty((max(int(n), 16),), dtype=torch.uint8, device=cache.k.device)


def treewy_attn_chunk(cache: KVCache, row_offsets: torch.Tensor, q: torch.Tensor, scale: float, O: torch.Tensor,
                      workspace: torch.Tensor, window: int = 0, sinks: int = 0, seq_status: torch.Tensor | None = None, stream=None,
                      generic: bool = False) -> None:
    """O [T, H_q, d] <- attention of every new row (q: packed rows of the sequences at row_offsets [B + 1]; their keys and
    values are in the cache behind context_len) over the cached tokens up to its own: all of them, or (window > 0) the last
    `window` and the first `sinks`."""
    lib = load_library()
    if q.dim() != 3:
        raise ValueError("q: [T, H_q, d] wanted")
    (T, H_q, d), dtype, dev = q.shape, cache.dtype, cache._dev
    if d != cache.d_head:
        raise ValueError("q: the cache's d_head wanted")
    _window(window, sinks)
    _on_gpu(dev, T if seq_status is None else cache.B)
    ld_q = _rows(q, T, H_q, d, dtype, "q", dev)
    if _rows(O, T, H_q, d, dtype, "O", dev) != H_q * d and T > 0:
        raise ValueError("O: contiguous rows wanted")
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace: contiguous and on the cache's device wanted")
    tw._call("treewy_attn_chunk_generic" if generic else "treewy_attn_chunk", lib.treewy_attn_chunk_generic if generic else lib.treewy_attn_chunk,
             cache._ref, cache.B, T, _int32(row_offsets, cache.B + 1, "row_offsets", dev), q.data_ptr(), ld_q, H_q, scale, window, sinks,
             cache._dt, O.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
             _int32(seq_status, cache.B, "seq_status", dev), _stream(stream, q))


class PagePool:
    """A page table kept on the GPU and the stack of pages that nobody holds (``treewy_page_pool_t``): page_table [B, max_pages]
    (negative: no page), free_pages [n_pages], free_count [1], all int32.  The object refers to the tensors' memory.
    Who holds a page is not counted: one in the tables of several sequences (a shared prompt) is released for the last of them
    only, with `first` behind it for the others."""

    def __init__(self, page_table: torch.Tensor, page_size: int, n_pages: int, free_pages: torch.Tensor, free_count: torch.Tensor):
        _require(page_table.dim() == 2 and page_table.is_contiguous() and page_table.dtype == torch.int32,
                 "page_table: contiguous int32 [B, max_pages] wanted")
        self._dev = page_table.get_device()
        _int32(free_pages, n_pages, "free_pages", self._dev)
        _int32(free_count, 1, "free_count", self._dev)
        self.page_table, self.free_pages, self.free_count = page_table, free_pages, free_count
        self.page_size, self.n_pages = page_size, n_pages
        self.B, self.max_pages = (int(n) for n in page_table.shape)
        self._struct = PagePoolStruct(page_table.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(), n_pages, page_size, self.max_pages)
        self._ref = ctypes.byref(self._struct)

    @classmethod
    def empty(cls, B: int, max_pages: int, page_size: int, n_pages: int, device) -> "PagePool":
        """No sequence holds a page; page 0 is taken first."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.full((B, max_pages), -1, **i32), page_size, n_pages, torch.arange(n_pages - 1, -1, -1, **i32),
                   torch.full((1,), n_pages, **i32))


def treewy_pages_reserve(pool: PagePool, context_len: torch.Tensor, row_offsets: torch.Tensor, T: int,
                         positions: torch.Tensor | None = None, slots: torch.Tensor | None = None,
                         seq_status: torch.Tensor | None = None, stream=None) -> None:
    """Pages for the rows at row_offsets [B + 1] (T in all) behind context_len [B]; positions [T] int32 receives each row's token
    number and slots [T] int64 its place in the cache."""
    B, dev = pool.B, pool._dev
    _on_gpu(dev, B)
    if slots is not None and (slots.dtype is not torch.int64 or slots.numel() < T or not slots.is_contiguous() or slots.get_device() != dev):
        raise ValueError(f"slots: contiguous int64 [{T}] on the pool's device wanted")
    tw._call("treewy_pages_reserve", load_library().treewy_pages_reserve, pool._ref, B, T, _int32(context_len, B, "context_len", dev),
             _int32(row_offsets, B + 1, "row_offsets", dev), _int32(positions, T, "positions", dev),
             None if slots is None else slots.data_ptr(), _int32(seq_status, B, "seq_status", dev), _stream(stream, pool.page_table))


def treewy_pages_release(pool: PagePool, first: torch.Tensor, end: torch.Tensor, seq_status: torch.Tensor | None = None,
                         stream=None) -> None:
    """The pages whose tokens all lie in first[b] .. end[b] - 1 go back to the pool (each once: see PagePool on shared ones)."""
    B, dev = pool.B, pool._dev
    _on_gpu(dev, B)
    tw._call("treewy_pages_release", load_library().treewy_pages_release, pool._ref, B, _int32(first, B, "first", dev),
             _int32(end, B, "end", dev), _int32(seq_status, B, "seq_status", dev), _stream(stream, pool.page_table))


def _capturing(x: torch.Tensor) -> bool:
    """Whether the call that x goes into is being captured into a graph."""
    return x.is_cuda and torch.cuda.is_current_stream_capturing()


def _let_go(ws: torch.Tensor | None) -> None:
    """A workspace that a larger one replaces: calls on other streams than the one it was allocated on may still be at work in it.  All
    of them are ahead of the current call, as the cache is theirs too, so its memory is free when the current stream has come here."""
    if ws is not None and ws.is_cuda:
        ws.record_stream(torch.cuda.current_stream(ws.device))


class AttentionLayer:
    """One attention layer's side of a step -- a prompt or a piece of one, single tokens, a speculative round -- on the current
    stream: the paged cache, the rotary table, the norms and workspaces stay with the layer; each call takes the step's packed
    rows.  Calls of one layer, replays of captured ones among them, share these: on several streams the caller orders them.  The cache's ``context_len`` is advanced by ``prefill``, ``commit`` and ``append_and_attend``.  Layers of one model that share
    a context_len array leave that to the last of them, since all of a step write at the same place: the others pass
    advance=False.

    q_norm, k_norm: norms of the queries' and keys' heads ahead of the rotation.  window: a token sees the last `window` tokens,
    its own among them, and the first `sinks` (0: all); pages that no later token sees may go back to a pool.  Draft trees see
    everything, so a layer with a window has no ``verify``.

    seq_status [B], zeroed by the caller ahead of a round and passed to all of its calls, receives their flags; without it
    the layer keeps its own.  A sequence that is flagged in it, by whichever layer, keeps its length, and its rows of the
    outputs mean nothing."""

    def __init__(self, cache: KVCache, H_q: int, cos_sin: torch.Tensor, pair_axis: torch.Tensor | None = None,
                 interleaved: bool = False, scale: float | None = None, q_norm: HeadNorm | None = None,
                 k_norm: HeadNorm | None = None, window: int = 0, sinks: int = 0):
        if H_q < 1 or H_q % cache.H_kv != 0:
            raise ValueError("H_q: a multiple of the cache's heads wanted")
        _window(window, sinks)
        if window < 0 or sinks < 0:
            raise ValueError("window, sinks: not negative")
        _norm(q_norm, cache.d_head, "q_norm", cache._dev), _norm(k_norm, cache.d_head, "k_norm", cache._dev)
        self.q_norm, self.k_norm, self.window, self.sinks = q_norm, k_norm, window, sinks
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
        self._rows_ws, self._rows_for = None, 0    # workspace of prefill, and the rows it is for
        self._captured = []                        # workspaces that graphs refer to

    def _workspace(self, tree: Tree, shared_len: int) -> torch.Tensor:
        sizes = (tree.B, tree.T, tree.max_nodes, shared_len)
        if self._ws_for != sizes:
            ws = attn_workspace(self.cache, tree, self.H_q, shared_len)
            if self._ws is None or ws.numel() > self._ws.numel():
                _let_go(self._ws)
                self._ws = ws
            self._ws_for = sizes
        return self._in_use(self._ws)

    def _in_use(self, ws: torch.Tensor) -> torch.Tensor:
        """A workspace that a call being captured takes stays, whatever later calls take: the graph writes to it at each replay."""
        if _capturing(ws) and not any(w is ws for w in self._captured):
            self._captured.append(ws)
        return ws

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
        """Normalises and rotates q and k in place (keep k and v until commit) and returns the attention's output for every
        node."""
        if self.window > 0:
            raise ValueError("a layer with a window verifies no trees")
        status = self._begin(tree, seq_status)
        rope = self._rope(positions)
        offsets = tree.node_offsets[:tree.B + 1]
        for x, norm in ((q, self.q_norm), (k, self.k_norm)):
            if norm is None:
                treewy_rope_rows(rope, offsets, x, x, seq_status=status)
            else:
                treewy_norm_rope(norm, rope, x, x, offsets, status)
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
        if self.window > 0:
            if shared_len > 0:
                raise ValueError("shared_len: not beside a window")
            return self._rows(tree.node_offsets, positions, q, k, v, self._begin(tree, seq_status), advance, one=True)
        status = self._begin(tree, seq_status)
        self._round = None
        q_out, O = self._out(q), self._out(q)
        self._append(tree.node_offsets, positions, q, k, v, q_out, status)
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

    def _append(self, offsets: torch.Tensor, positions: torch.Tensor, q, k, v, q_out, status) -> None:
        rope = self._rope(positions)
        if self.q_norm is None and self.k_norm is None:
            treewy_kv_append(self.cache, offsets, k, v, rope, q, q_out, status)
        else:
            treewy_kv_append_norm(self.cache, offsets, k, v, self.k_norm, rope, q, q_out, self.q_norm, status)

    def _rows(self, offsets: torch.Tensor, positions: torch.Tensor, q, k, v, status: torch.Tensor, advance: bool, one: bool) -> torch.Tensor:
        """New rows enter the cache and attend to it.  one: a sequence with no row or with several is flagged."""
        self._round = None
        T, B = q.shape[0], self.cache.B
        q_out, O = self._out(q), self._out(q)
        counts = offsets[1:B + 1] - offsets[:B]
        if one:
            status |= (counts != 1) * tw.SEQ_TOO_MANY_NODES
        self._append(offsets, positions, q, k, v, q_out, status)
        if self._rows_ws is None or self._rows_for < T:
            _let_go(self._rows_ws)
            self._rows_ws, self._rows_for = attn_chunk_workspace(self.cache, T, self.H_q, self.window, self.sinks), T
        treewy_attn_chunk(self.cache, offsets, q_out, self.scale, O, self._in_use(self._rows_ws), self.window, self.sinks, status)
        if advance:
            self._len.add_(counts * (status == 0))
        return O

    def prefill(self, row_offsets: torch.Tensor, positions: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                seq_status: torch.Tensor | None = None, advance: bool = True) -> torch.Tensor:
        """New tokens -- a prompt, a piece of one, or one each; any number a sequence, none among them -- at row_offsets [B + 1]:
        normalised, rotated, written to the cache, and attended from there, each up to its own."""
        _int32(row_offsets, self.cache.B + 1, "row_offsets", self.cache._dev)
        _int32(seq_status, self.cache.B, "seq_status", self.cache._dev)
        status = self._own.zero_() if seq_status is None else seq_status.view(-1)[:self.cache.B]
        return self._rows(row_offsets.view(-1), positions, q, k, v, status, advance, one=False)
