"""Attention-layer calls without a GPU: exported symbols, struct mirrors, and refusals of misuse before any
launch."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "treewy_attn.h")
A = 0x1000  # any 16-byte aligned address, never dereferenced: every call below fails its checks first
vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def at():
    from paper_2608_20961_b200 import attention, build
    build.build()
    attention.load_library()
    return attention


def _text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_declared_symbols_are_exported(at):
    names = sorted(set(re.findall(r"\b(treewy_[a-z_]+)\s*\(", _text())))
    assert {"treewy_rope", "treewy_kv_append", "treewy_attn_verify", "treewy_kv_commit"} <= set(names)
    for name in names:
        assert hasattr(at.load_library(), name), name


def test_structs_and_status_bits_mirror_the_header(at):
    text = _text()
    for ctype, mirror in (("treewy_kv_cache_t", at.KVCacheStruct), ("treewy_rope_t", at.RopeStruct)):
        body = text[:text.index(f"}} {ctype};")]
        body = body[body.rindex("typedef struct {"):]
        names = re.findall(r"\*?(\w+)\s*[,;]", body)
        assert names == [f[0] for f in mirror._fields_]
    bits = dict(re.findall(r"TREEWY_SEQ_(\w+) = (\d+)", text))
    assert {k: int(v) for k, v in bits.items()} == {"BAD_PAGE": at.SEQ_BAD_PAGE, "BAD_LENGTH": at.SEQ_BAD_LENGTH,
                                                    "BAD_POSITION": at.SEQ_BAD_POSITION}


def _cache(at, **kw):
    base = dict(k=A, v=A, stride_page=1024, stride_slot=128, stride_head=64, page_table=A, context_len=A + 16, n_pages=4,
                page_size=8, max_pages=64, H_kv=2, d_head=64)
    base.update(kw)
    return at.KVCacheStruct(**base)


def _rope(at, **kw):
    base = dict(cos_sin=A, positions=A, pair_axis=None, n_axes=1, max_positions=16, rot_dim=64, interleaved=0)
    base.update(kw)
    return at.RopeStruct(**base)


def _tree(at, **kw):
    base = dict(B=2, T=8, H_v=1, max_nodes=0, node_offsets=A, parent=A, depth=A, anc_mask=A, cum_log_gate=A, level_order=A)
    base.update(kw)
    return at.tw.TreeStruct(**base)


INVALID, UNSUPPORTED, OK, BF16 = 1, 2, 0, 1


def _rope_call(at, rope=None, x=A, ld_x=256, y=A, ld_y=256, T=3, H=4, d=64, io=BF16, status=None):
    rope = _rope(at) if rope is None else rope
    return at.load_library().treewy_rope(ctypes.byref(rope), vp(x), ld_x, vp(y), ld_y, T, H, d, 0, io, vp(status), None)


def _append(at, cache=None, rope=None, B=2, T=8, off=A, k=A, ld_k=128, v=A, ld_v=128, H_q=4, q=A, ld_q=256, qo=A, ld_qo=256,
            io=BF16, status=None):
    cache = _cache(at) if cache is None else cache
    return at.load_library().treewy_kv_append(ctypes.byref(cache), None if rope is None else ctypes.byref(rope), B, T, vp(off),
                                              vp(k), ld_k, vp(v), ld_v, H_q, vp(q), ld_q, vp(qo), ld_qo, io, vp(status), None)


def _verify(at, cache=None, tree=None, q=A, ld_q=256, k=A, ld_k=128, v=A, ld_v=128, H_q=4, pages=None, shared=0, io=BF16,
            O=A, ws=A, ws_bytes=1 << 40, status=None, generic=False, scale=0.125):
    cache, tree = _cache(at) if cache is None else cache, _tree(at) if tree is None else tree
    lib = at.load_library()
    fn = lib.treewy_attn_verify_generic if generic else lib.treewy_attn_verify
    return fn(ctypes.byref(cache), ctypes.byref(tree), vp(q), ld_q, vp(k), ld_k, vp(v), ld_v, H_q, scale, vp(pages), shared, io,
              vp(O), vp(ws), ws_bytes, vp(status), None)


def _commit(at, cache=None, tree=None, k=A, ld_k=128, v=A, ld_v=128, acc=A, io=BF16, new=None, status=None):
    cache, tree = _cache(at) if cache is None else cache, _tree(at) if tree is None else tree
    return at.load_library().treewy_kv_commit(ctypes.byref(cache), ctypes.byref(tree), vp(k), ld_k, vp(v), ld_v, vp(acc), io,
                                              vp(new), vp(status), None)


def test_rope_refusals(at):
    for bad in (dict(x=None), dict(x=A + 2), dict(y=None), dict(ld_x=255), dict(ld_x=252), dict(T=-1), dict(H=0), dict(d=0),
                dict(status=A + 4)):
        assert _rope_call(at, **bad) == INVALID, bad
    for bad in (dict(io=7), dict(d=63)):
        assert _rope_call(at, **bad) == UNSUPPORTED, bad
    for bad in (dict(cos_sin=None), dict(positions=None), dict(n_axes=0), dict(max_positions=0), dict(rot_dim=0)):
        assert _rope_call(at, rope=_rope(at, **bad)) == INVALID, bad
    for bad in (dict(rot_dim=63), dict(rot_dim=66), dict(n_axes=33)):
        assert _rope_call(at, rope=_rope(at, **bad)) == UNSUPPORTED, bad
    assert _rope_call(at, T=0, x=None, y=None) == OK


BAD_CACHES = [(dict(n_pages=-1), INVALID), (dict(page_size=0), INVALID), (dict(max_pages=-1), INVALID), (dict(H_kv=0), INVALID),
              (dict(d_head=0), INVALID), (dict(d_head=60), UNSUPPORTED), (dict(d_head=264), UNSUPPORTED), (dict(k=None), INVALID),
              (dict(v=A + 8), INVALID), (dict(page_table=None), INVALID), (dict(context_len=None), INVALID),
              (dict(stride_slot=132), INVALID), (dict(stride_page=-1024), INVALID), (dict(stride_head=65), INVALID),
              (dict(page_size=1 << 20, max_pages=1 << 20), UNSUPPORTED)]


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_cache_refusals(at, bad, code):
    cache = _cache(at, **bad)
    assert _append(at, cache=cache) == code
    assert _verify(at, cache=cache) == code
    assert _commit(at, cache=cache) == code


def test_append_refusals(at):
    for bad in (dict(B=-1), dict(T=-1), dict(H_q=-1), dict(off=None), dict(k=None), dict(v=A + 2), dict(ld_k=120), dict(ld_v=129),
                dict(q=None), dict(qo=None), dict(ld_q=248), dict(ld_qo=257), dict(status=A + 4)):
        assert _append(at, **bad) == INVALID, bad
    assert _append(at, io=5) == UNSUPPORTED
    assert _append(at, rope=_rope(at, rot_dim=128)) == UNSUPPORTED
    assert _append(at, B=0, T=0, k=None, v=None, q=None) == OK


def test_verify_and_commit_refusals(at):
    for generic in (False, True):
        for bad in (dict(q=None), dict(k=A + 2), dict(v=None), dict(O=None), dict(ld_q=128), dict(ld_k=132), dict(H_q=3), dict(H_q=0),
                    dict(shared=8), dict(shared=12, pages=A), dict(shared=-8, pages=A), dict(status=A + 4), dict(ws_bytes=0),
                    dict(ws=None), dict(scale=0.0), dict(scale=-0.5), dict(scale=float("inf")), dict(scale=float("nan"))):
            assert _verify(at, generic=generic, **bad) == INVALID, bad
        assert _verify(at, io=3, generic=generic) == UNSUPPORTED
        for bad, code in ((dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(max_nodes=-1), INVALID), (dict(max_nodes=65), UNSUPPORTED),
                          (dict(node_offsets=None), INVALID), (dict(anc_mask=None), INVALID)):
            assert _verify(at, tree=_tree(at, **bad), generic=generic) == code, bad
            assert _commit(at, tree=_tree(at, **bad)) == code, bad
        assert _verify(at, tree=_tree(at, B=0, T=0), q=None, generic=generic) == OK
    for bad in (dict(k=None), dict(v=A + 2), dict(acc=None), dict(ld_k=120), dict(new=A + 16), dict(new=A + 4), dict(status=A + 4)):
        assert _commit(at, **bad) == INVALID, bad
    assert _commit(at, tree=_tree(at, B=0, T=0), k=None) == OK


def test_binding_checks_shapes_types_and_strides(at):
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    k, v = z(4, 8, 2, 64), z(4, 8, 2, 64)
    cache = at.KVCache(k, v, i32(2, 2), i32(2))
    for bad in ((z(4, 8, 2, 64, dt=torch.float16), v, i32(2, 2), i32(2)), (k, z(4, 8, 2, 32), i32(2, 2), i32(2)),
                (k, v.transpose(1, 2).contiguous().transpose(1, 2), i32(2, 2), i32(2)), (k, v, i32(2, 4)[:, ::2], i32(2)),
                (k, v, i32(2, 2).long(), i32(2)), (k, v, i32(2, 2), i32(1))):
        with pytest.raises(ValueError):
            at.KVCache(*bad)
    rope = at.Rope(z(16, 64, dt=torch.float32), i32(6))
    with pytest.raises(ValueError):
        at.Rope(z(16, 64), i32(6))
    with pytest.raises(ValueError):
        at.Rope(z(16, 64, dt=torch.float32), i32(1, 6), torch.zeros(31, dtype=torch.uint8))
    x = z(6, 4, 64)
    for bad in (z(5, 4, 64), z(6, 4, 128)[..., ::2], z(4, 6, 64).transpose(0, 1)):
        with pytest.raises(ValueError):
            at.treewy_rope(rope, x, bad)
    with pytest.raises(ValueError):
        at.treewy_rope(rope, z(5, 4, 64), z(5, 4, 64))
    with pytest.raises(ValueError):
        at.treewy_kv_append(cache, i32(2), z(6, 2, 64), z(6, 2, 64))
    with pytest.raises(ValueError):
        at.treewy_kv_append(cache, i32(3), z(6, 2, 64), z(6, 2, 64), q=x)
    tree = at.tw.Tree.empty(torch.tensor([0, 3, 6], dtype=torch.int32), i32(6), 1)
    ws = z(64, dt=torch.uint8)
    with pytest.raises(ValueError):
        at.treewy_attn_verify(cache, tree, x, z(6, 1, 64), z(6, 2, 64), 1.0, z(6, 4, 64), ws)
    with pytest.raises(ValueError):
        at.treewy_attn_verify(cache, tree, x, z(6, 2, 64), z(6, 2, 64), 1.0, z(6, 4, 128)[..., :64], ws)
    with pytest.raises(ValueError):
        at.treewy_kv_commit(cache, tree, z(6, 2, 64), z(6, 2, 64), torch.zeros(2, dtype=torch.int64))


def test_empty_calls_need_no_gpu(at):
    class FakeStream:
        cuda_stream = 0
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    cache = at.KVCache(z(4, 8, 2, 64), z(4, 8, 2, 64), i32(0, 2), i32(0))
    tree = at.tw.Tree.empty(i32(1), i32(0), 1)
    call = at.tw.prebound(at.treewy_attn_verify, cache, tree, z(0, 4, 64), z(0, 2, 64), z(0, 2, 64), 1.0, z(0, 4, 64),
                          torch.zeros(16, dtype=torch.uint8), stream=FakeStream())
    call()
    at.treewy_kv_commit(cache, tree, z(0, 2, 64), z(0, 2, 64), i32(0), stream=FakeStream())
    at.treewy_kv_append(cache, i32(1), z(0, 2, 64), z(0, 2, 64), stream=FakeStream())
