"""Refusals of the attention calls and of AttentionLayer, without a GPU."""
import ctypes

import pytest
import torch

A = 0x1000  # any 16-byte aligned address, never dereferenced: every call below fails its checks first
vp = ctypes.c_void_p
INVALID, UNSUPPORTED, OK, BF16 = 1, 2, 0, 1


@pytest.fixture(scope="module")
def at():
    from paper_2608_20961_b200 import attention, build
    build.build()
    attention.load_library()
    return attention


def z(*s, dt=torch.bfloat16):
    return torch.zeros(s, dtype=dt)


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


def test_rope_rows_refusals(at):
    rope = at.RopeStruct(cos_sin=A, positions=A, pair_axis=None, n_axes=1, max_positions=16, rot_dim=64, interleaved=0)

    def call(B=2, T=3, off=A, x=A, ld_x=256, y=A, ld_y=256, H=4, d=64, io=BF16, status=None):
        return at.load_library().treewy_rope_rows(ctypes.byref(rope), B, T, vp(off), vp(x), ld_x, vp(y), ld_y, H, d, 0, io, vp(status), None)
    for bad in (dict(B=-1), dict(T=-1), dict(off=None), dict(off=A + 4), dict(x=None), dict(y=A + 2), dict(ld_x=255), dict(H=0),
                dict(status=A + 4)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(io=7), dict(d=63)):
        assert call(**bad) == UNSUPPORTED, bad
    assert call(T=0, off=None, x=None, y=None) == OK and call(B=0, off=None) == OK
    handle = at.Rope(z(16, 64, dt=torch.float32), i32(6))
    for off, x in ((i32(3), z(5, 4, 64)), (i32(3).long(), z(6, 4, 64)), (i32(0), z(6, 4, 64)), (i32(3), z(6, 4, 64, dt=torch.float16))):
        with pytest.raises(ValueError):
            at.treewy_rope_rows(handle, off, x, x)


def calls(at, dev="cpu"):
    """Every call of the binding as (function, keyword arguments), with something to do."""
    t = lambda x: x.to(dev)
    cache = at.KVCache(t(z(4, 8, 2, 64)), t(z(4, 8, 2, 64)), t(i32(2, 2)), t(i32(2)))
    tree = at.tw.Tree.empty(t(torch.tensor([0, 3, 6], dtype=torch.int32)), t(i32(6)), 1)
    rope = at.Rope(t(z(16, 64, dt=torch.float32)), t(i32(6)))
    rows = lambda h: t(z(6, h, 64))
    return cache, tree, rope, [
        (at.treewy_rope, dict(rope=rope, x=rows(4), y=rows(4), row_status=t(i32(1)))),
        (at.treewy_rope_rows, dict(rope=rope, row_offsets=t(torch.tensor([0, 3, 6], dtype=torch.int32)), x=rows(4), y=rows(4), seq_status=t(i32(2)))),
        (at.treewy_kv_append, dict(cache=cache, row_offsets=t(torch.tensor([0, 3, 6], dtype=torch.int32)), k=rows(2), v=rows(2), rope=rope, q=rows(4),
                                   q_out=rows(4), seq_status=t(i32(2)))),
        (at.treewy_attn_verify, dict(cache=cache, tree=tree, q=rows(4), k=rows(2), v=rows(2), scale=1.0, O=rows(4), workspace=t(z(1 << 24, dt=torch.uint8)),
                                     shared_pages=t(i32(1)), shared_len=8, seq_status=t(i32(2)))),
        (at.treewy_kv_commit, dict(cache=cache, tree=tree, k=rows(2), v=rows(2), accepted=t(i32(2)), new_context_len=t(i32(2)), seq_status=t(i32(2))))]


class Stream:
    cuda_stream = 0


def test_host_tensors_are_refused(at):
    for fn, kw in calls(at)[3]:
        with pytest.raises(ValueError):
            fn(**kw, stream=Stream())


@pytest.mark.gpu
def test_tensors_of_two_devices_are_refused(at):
    """One argument at a time on the host: refused before a kernel could meet its address."""
    cache, tree, rope, all_calls = calls(at, "cuda:0")
    for fn, kw in all_calls:
        for name, x in kw.items():
            if isinstance(x, torch.Tensor):
                with pytest.raises(ValueError):
                    fn(**{**kw, name: x.cpu()})
        if "tree" in kw:
            for name in ("node_offsets", "anc_mask"):
                with pytest.raises(ValueError):
                    fn(**{**kw, "tree": at.tw.Tree(**{**vars(tree), name: getattr(tree, name).cpu()})})
    cpu = calls(at)
    with pytest.raises(ValueError):
        at.treewy_kv_append(**{**all_calls[2][1], "rope": cpu[2]})
    for bad in (dict(positions=rope.positions.cpu()), dict(cos_sin=rope.cos_sin.cpu()), dict(pair_axis=torch.zeros(32, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            at.Rope(**{**dict(cos_sin=rope.cos_sin, positions=rope.positions), **bad})


@pytest.mark.parametrize("bad", [dict(node_offsets=i32(2)), dict(node_offsets=i32(3).long()), dict(node_offsets=i32(6)[::2]),
                                 dict(anc_mask=torch.zeros(5, dtype=torch.int64)), dict(anc_mask=i32(6)),
                                 dict(anc_mask=torch.zeros(12, dtype=torch.int64)[::2])])
def test_arrays_of_a_tree_are_checked(at, bad):
    cache, tree, _, _ = calls(at)
    with pytest.raises(ValueError):
        at.attn_workspace(cache, at.tw.Tree(**{**vars(tree), **bad}), 4)


def test_rows_past_32_bits_are_refused(at):
    """Offsets within a token's row are 32-bit in the kernels."""
    lib, H = at.load_library(), 1 << 24                # x 128 = 2^31 elements, 4 GB of bf16
    cache = lambda H_kv: at.KVCacheStruct(k=A, v=A, stride_page=1 << 40, stride_slot=1 << 34, stride_head=128, page_table=A, context_len=A + 16,
                                          n_pages=4, page_size=8, max_pages=64, H_kv=H_kv, d_head=128)
    rope = at.RopeStruct(cos_sin=A, positions=A, pair_axis=None, n_axes=1, max_positions=16, rot_dim=64, interleaved=0)
    tree = at.tw.TreeStruct(B=1, T=1, H_v=1, max_nodes=1, node_offsets=A, parent=None, depth=None, anc_mask=A, cum_log_gate=None, level_order=None)
    ref, ld = ctypes.byref, 1 << 34
    assert lib.treewy_rope(ref(rope), vp(A), ld, vp(A), ld, 1, H, 128, 0, BF16, None, None) == UNSUPPORTED
    for hk, hq in ((1, H), (H, 0)):
        assert lib.treewy_kv_append(ref(cache(hk)), ref(rope), 1, 1, vp(A), vp(A), ld, vp(A), ld, hq, vp(A), ld, vp(A), ld, BF16, None, None) == UNSUPPORTED
    for fn in (lib.treewy_attn_verify, lib.treewy_attn_verify_generic):
        for hk in (1, H):
            assert fn(ref(cache(hk)), ref(tree), vp(A), ld, vp(A), ld, vp(A), ld, H, 0.1, None, 0, BF16, vp(A), vp(A), 1 << 60, None, None) == UNSUPPORTED
    assert lib.treewy_kv_commit(ref(cache(H)), ref(tree), vp(A), ld, vp(A), ld, vp(A), BF16, None, None, None) == UNSUPPORTED
