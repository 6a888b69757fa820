"""The calls that take new rows through an attention layer, without a GPU: exported symbols, struct mirrors, and refusals of
misuse before any launch."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "treewy_prompt.h")
A = 0x1000  # any 16-byte aligned address, never dereferenced: every call below fails its checks first
OK, INVALID, UNSUPPORTED = 0, 1, 2
F32, BF16 = 0, 1
ref = ctypes.byref


@pytest.fixture(scope="module")
def at():
    from paper_2608_20961_b200 import attention, build
    build.build()
    attention.load_library()
    global F32, BF16
    F32, BF16 = attention.tw._DTYPES[torch.float32], attention.tw._DTYPES[torch.bfloat16]
    return attention


def _text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_declared_symbols_are_exported(at):
    names = sorted(set(re.findall(r"\b(treewy_[a-z_]+)\s*\(", _text())))
    assert {"treewy_norm_rope", "treewy_norm_rope_backward", "treewy_kv_append_norm", "treewy_attn_chunk",
            "treewy_pages_reserve", "treewy_pages_release"} <= set(names)
    for name in names:
        assert hasattr(at.load_library(), name), name


def test_structs_and_status_bits_mirror_the_header(at):
    text = _text()
    for ctype, mirror in (("treewy_head_norm_t", at.HeadNormStruct), ("treewy_page_pool_t", at.PagePoolStruct)):
        body = text[:text.index(f"}} {ctype};")]
        body = body[body.rindex("typedef struct {"):]
        assert re.findall(r"\*?(\w+)\s*[,;]", body) == [f[0] for f in mirror._fields_]
    assert dict(re.findall(r"TREEWY_SEQ_(\w+) = (\d+)", text)) == {"NO_PAGES": str(at.SEQ_NO_PAGES)}


def _cache(at, **kw):
    base = dict(k=A, v=A, stride_page=1024, stride_slot=128, stride_head=64, page_table=A, context_len=A + 16, n_pages=4,
                page_size=8, max_pages=64, H_kv=2, d_head=64)
    base.update(kw)
    return at.KVCacheStruct(**base)


def _rope(at, **kw):
    base = dict(cos_sin=A, positions=A, pair_axis=None, n_axes=1, max_positions=16, rot_dim=64, interleaved=0)
    base.update(kw)
    return at.RopeStruct(**base)


def _norm(at, **kw):
    base = dict(weight=A, weight_dtype=BF16, eps=1e-6, plus_one=0)
    base.update(kw)
    return at.HeadNormStruct(**base)


def _chunk(at, generic=False, cache=None, B=2, T=6, off=A, q=A, ld_q=256, H_q=4, scale=0.5, window=0, sinks=0, io=None, O=A, ws=A,
           ws_bytes=1 << 40, status=None):
    lib = at.load_library()
    fn = lib.treewy_attn_chunk_generic if generic else lib.treewy_attn_chunk
    return fn(ref(cache or _cache(at)), B, T, off, q, ld_q, H_q, scale, window, sinks, BF16 if io is None else io, O, ws, ws_bytes, status, None)


@pytest.mark.parametrize("generic", [False, True])
def test_chunk_refusals(at, generic):
    for bad in (dict(B=-1), dict(T=-1), dict(off=None), dict(q=None), dict(q=A + 2), dict(O=None), dict(O=A + 8), dict(ld_q=128), dict(ld_q=260),
                dict(H_q=0), dict(H_q=3), dict(window=-1), dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(status=A + 4), dict(ws=None), dict(ws_bytes=0), dict(ws=A + 4)):
        assert _chunk(at, generic, **bad) == INVALID, bad
    assert _chunk(at, generic, io=7) == UNSUPPORTED
    for bad, code in ((dict(d_head=60), UNSUPPORTED), (dict(d_head=264), UNSUPPORTED), (dict(page_size=0), INVALID), (dict(k=None), INVALID),
                      (dict(page_table=None), INVALID), (dict(context_len=A + 4), INVALID), (dict(stride_slot=4), INVALID),
                      (dict(max_pages=1 << 29), UNSUPPORTED)):
        assert _chunk(at, generic, cache=_cache(at, **bad)) == code, bad
    assert _chunk(at, generic, B=0, T=0, q=None, O=None, off=None) == OK
    assert _chunk(at, generic, T=0, q=None, O=None, off=None) == OK
    assert at.load_library().treewy_attn_chunk_generic(None, 2, 6, A, A, 256, 4, 0.5, 0, 0, BF16, A, A, 1 << 40, None, None) == INVALID


def test_norm_refusals(at):
    lib = at.load_library()

    def call(norm=None, rope=None, B=0, T=3, off=None, x=A, ld_x=128, y=A, ld_y=128, H=2, d=64, io=None, status=None):
        return lib.treewy_norm_rope(ref(norm or _norm(at)), ref(rope or _rope(at)), B, T, off, x, ld_x, y, ld_y, H, d, BF16 if io is None else io,
                                    status, None)

    def back(norm=None, rope=None, x=A, ld_x=128, dy=A, ld_dy=128, dx=A, ld_dx=128, dw=A, T=3, H=2, d=64, io=None, ws=A, n=1 << 30, status=None):
        return lib.treewy_norm_rope_backward(ref(norm or _norm(at)), ref(rope or _rope(at)), x, ld_x, dy, ld_dy, dx, ld_dx, dw, T, H, d,
                                             BF16 if io is None else io, ws, n, status, None)

    for bad in (dict(T=-1), dict(H=0), dict(d=0), dict(x=None), dict(ld_x=120), dict(ld_x=132), dict(x=A + 2), dict(status=A + 4),
                dict(norm=_norm(at, weight=None)), dict(norm=_norm(at, weight=A + 2)), dict(norm=_norm(at, eps=0.0)),
                dict(norm=_norm(at, eps=float("nan"))), dict(norm=_norm(at, eps=float("inf"))), dict(rope=_rope(at, positions=None)),
                dict(rope=_rope(at, n_axes=0))):
        assert call(**bad) == INVALID, bad
        assert back(**bad) == INVALID, bad
    for bad in (dict(d=63), dict(d=258, ld_x=600), dict(io=9), dict(norm=_norm(at, weight_dtype=9)), dict(rope=_rope(at, rot_dim=66)),
                dict(H=1 << 26, ld_x=1 << 33)):
        assert call(**bad) == UNSUPPORTED, bad
        assert back(**bad) == UNSUPPORTED, bad
    for bad in (dict(y=None), dict(ld_y=64), dict(B=-1), dict(B=2), dict(B=2, off=A + 4)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(dy=None), dict(dx=A + 8), dict(dw=None), dict(dw=A + 4), dict(ws=None), dict(n=100), dict(ld_dy=4), dict(ld_dx=12)):
        assert back(**bad) == INVALID, bad
    assert lib.treewy_norm_rope(None, None, 0, 3, None, A, 128, A, 128, 2, 64, BF16, None, None) == INVALID
    assert call(T=0, x=None, y=None) == OK


def test_append_norm_refusals(at):
    lib = at.load_library()

    def call(cache=None, rope=None, qn=None, kn=None, B=2, T=6, off=A, k=A, ld_k=128, v=A, ld_v=128, H_q=4, q=A, ld_q=256, qo=A, ld_qo=256, io=None,
             status=None):
        return lib.treewy_kv_append_norm(ref(cache or _cache(at)), ref(rope or _rope(at)), ref(qn or _norm(at)), ref(kn or _norm(at)), B, T, off, k,
                                         ld_k, v, ld_v, H_q, q, ld_q, qo, ld_qo, BF16 if io is None else io, status, None)

    for bad in (dict(B=-1), dict(T=-1), dict(H_q=-1), dict(off=None), dict(k=None), dict(v=A + 2), dict(ld_k=120), dict(ld_v=129),
                dict(q=None), dict(qo=None), dict(ld_q=248), dict(ld_qo=257), dict(status=A + 4), dict(qn=_norm(at, eps=-1.0)),
                dict(kn=_norm(at, weight=None))):
        assert call(**bad) == INVALID, bad
    assert call(io=5) == UNSUPPORTED
    assert call(kn=_norm(at, weight_dtype=3)) == UNSUPPORTED
    assert call(B=0, T=0, k=None, v=None, q=None) == OK


def test_pages_refusals(at):
    lib = at.load_library()
    pool = lambda **kw: at.PagePoolStruct(**{**dict(page_table=A, free_pages=A, free_count=A, n_pages=4, page_size=8, max_pages=3), **kw})
    reserve = lambda p=None, B=2, T=3, n=A, off=A, pos=None, slots=None, status=None: lib.treewy_pages_reserve(
        ref(p or pool()), B, T, n, off, pos, slots, status, None)
    release = lambda p=None, B=2, first=A, end=A, status=None: lib.treewy_pages_release(ref(p or pool()), B, first, end, status, None)
    for bad in (dict(n_pages=-1), dict(page_size=0), dict(max_pages=-1), dict(page_table=None), dict(free_pages=None), dict(free_count=None),
                dict(free_count=A + 4)):
        assert reserve(pool(**bad)) == INVALID and release(pool(**bad)) == INVALID, bad
    for bad in (dict(max_pages=1 << 30), dict(page_size=1 << 30)):
        assert reserve(pool(**bad)) == UNSUPPORTED and release(pool(**bad)) == UNSUPPORTED, bad
    for bad in (dict(B=-1), dict(T=-1), dict(n=None), dict(off=A + 4), dict(pos=A + 4), dict(slots=A + 8), dict(status=A + 4)):
        assert reserve(**bad) == INVALID, bad
    for bad in (dict(B=-1), dict(first=None), dict(end=A + 4), dict(status=A + 4)):
        assert release(**bad) == INVALID, bad
    assert lib.treewy_pages_reserve(None, 2, 3, A, A, None, None, None, None) == INVALID
    assert reserve(B=0, n=None) == OK and release(B=0, first=None) == OK


def test_binding_checks_shapes_types_and_strides(at):
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    cache = at.KVCache(z(4, 8, 2, 64), z(4, 8, 2, 64), i32(2, 2), i32(2))
    ws = z(64, dt=torch.uint8)
    x, off = z(6, 4, 64), i32(3)
    for bad in ((off, z(6, 4, 32), x), (off, z(6, 4, 64, dt=torch.float32), x), (off, x, z(5, 4, 64)), (off, x, z(6, 4, 128)[..., :64]),
                (i32(2), x, z(6, 4, 64)), (off.long(), x, z(6, 4, 64)), (off, z(6, 256), x), (off, x, z(6, 4, 64))):    # (the last: no GPU)
        with pytest.raises(ValueError):
            at.treewy_attn_chunk(cache, bad[0], bad[1], 1.0, bad[2], ws)
    for bad in (z(64, dt=torch.float16), z(2, 64), z(128)[::2]):
        with pytest.raises(ValueError):
            at.HeadNorm(bad)
    norm, rope = at.HeadNorm(z(64)), at.Rope(z(16, 64, dt=torch.float32), i32(6))
    for bad in ((at.HeadNorm(z(32)), rope, x, x), (norm, at.Rope(z(16, 64, dt=torch.float32), i32(5)), x, x), (norm, rope, x, z(6, 4, 32)),
                (norm, rope, z(6, 4, 64, dt=torch.float16), x), (norm, rope, x, x)):
        with pytest.raises(ValueError):
            at.treewy_norm_rope(*bad)
    for bad in ((x, x, z(64)), (z(6, 4, 32), x, z(64, dt=torch.float32)), (x, z(5, 4, 64), z(64, dt=torch.float32)), (x, x, z(60, dt=torch.float32))):
        with pytest.raises(ValueError):
            at.treewy_norm_rope_backward(norm, rope, x, bad[0], bad[1], bad[2], ws)
    with pytest.raises(ValueError):
        at.treewy_kv_append_norm(cache, off, z(6, 2, 64), z(6, 2, 64), at.HeadNorm(z(32)))
    with pytest.raises(ValueError):
        at.treewy_kv_append_norm(cache, off, z(6, 2, 64), z(6, 2, 64), norm, rope, x)
    for bad in ((i32(2, 4)[:, ::2], 8, 4, i32(4), i32(1)), (i32(2, 4), 8, 4, i32(3), i32(1)), (i32(2, 4), 8, 4, i32(4).long(), i32(1)),
                (i32(2, 4), 8, 4, i32(4), i32(0))):
        with pytest.raises(ValueError):
            at.PagePool(*bad)
    pool = at.PagePool(i32(2, 4), 8, 4, i32(4), i32(1))
    for bad in (dict(context_len=i32(1)), dict(row_offsets=i32(2)), dict(positions=i32(5)), dict(slots=i32(6)), {}):     # (the last: no GPU)
        with pytest.raises(ValueError):
            at.treewy_pages_reserve(**{**dict(pool=pool, context_len=i32(2), row_offsets=off, T=6), **bad})
    with pytest.raises(ValueError):
        at.treewy_pages_release(pool, i32(2), i32(1))


def test_empty_calls_need_no_gpu(at):
    class FakeStream:
        cuda_stream = 0
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    cache = at.KVCache(z(4, 8, 2, 64), z(4, 8, 2, 64), i32(0, 2), i32(0))
    call = at.tw.prebound(at.treewy_attn_chunk, cache, i32(1), z(0, 4, 64), 1.0, z(0, 4, 64), torch.zeros(16, dtype=torch.uint8),
                          stream=FakeStream())
    call()
    at.treewy_norm_rope(at.HeadNorm(z(64)), None, z(0, 2, 64), z(0, 2, 64), stream=FakeStream())
    at.treewy_kv_append_norm(cache, i32(1), z(0, 2, 64), z(0, 2, 64), at.HeadNorm(z(64)), stream=FakeStream())
    pool = at.PagePool(i32(0, 4), 8, 4, i32(4), i32(1))
    at.treewy_pages_reserve(pool, i32(0), i32(1), 0, stream=FakeStream())
    at.treewy_pages_release(pool, i32(0), i32(0), stream=FakeStream())


def test_the_norms_gradient_against_differences():
    """The formulas that the kernels are tested against, against differences of the forward formula in 64 bits."""
    from tests import attn_util as au, prompt_util as pu
    gen = torch.Generator().manual_seed(1)
    x, w, dy = torch.randn(3, 2, 12, generator=gen, dtype=torch.float64), torch.rand(12, generator=gen, dtype=torch.float64) + 0.5, None
    dy = torch.randn(3, 2, 12, generator=gen, dtype=torch.float64)
    rope = (au.rope_table(8, 50), torch.randint(50, (2, 3), generator=gen, dtype=torch.int32), torch.tensor([0, 1, 1, 0], dtype=torch.uint8), False)
    for plus_one in (False, True):
        f = lambda x, w: float((pu.norm_reference(x, w, 0.01, rope, plus_one) * dy).sum())
        dx, dw = pu.norm_backward_reference(x, w, 0.01, dy, rope, plus_one)
        h = 1e-5
        for t, grad in ((x, dx), (w, dw)):
            for i in range(t.numel()):
                d = torch.zeros_like(t)
                d.view(-1)[i] = h
                args = lambda s: (x + s * d, w) if t is x else (x, w + s * d)
                diff = (f(*args(1)) - f(*args(-1))) / (2 * h)
                assert abs(diff - float(grad.view(-1)[i])) < 1e-7


def test_layer_refusals(at):
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    cache = at.KVCache(z(4, 8, 2, 64), z(4, 8, 2, 64), i32(2, 2), i32(2))
    table = z(16, 64, dt=torch.float32)
    for bad in (dict(window=-1), dict(sinks=-2), dict(q_norm=at.HeadNorm(z(32))), dict(k_norm=at.HeadNorm(z(32)))):
        with pytest.raises(ValueError):
            at.AttentionLayer(cache, 4, table, **bad)
    layer = at.AttentionLayer(cache, 4, table, window=8, sinks=1)
    tree = at.tw.Tree.empty(torch.tensor([0, 1, 2], dtype=torch.int32), i32(2), 1)
    rows = (z(2, 4, 64), z(2, 2, 64), z(2, 2, 64))
    with pytest.raises(ValueError):
        layer.verify(tree, i32(2), *rows)
    with pytest.raises(ValueError):
        layer.append_and_attend(tree, i32(2), *rows, shared_pages=i32(1), shared_len=8)
    with pytest.raises(ValueError):
        layer.prefill(i32(2), i32(2), *rows)
