"""The workspaces that an AttentionLayer keeps: those that graphs refer to stay when a call wants a larger one."""
import gc
import weakref

import pytest
import torch

BF16, I32 = torch.bfloat16, torch.int32


@pytest.fixture(scope="module")
def at():
    from paper_2608_20961_b200 import attention, build
    build.build()
    attention.load_library()
    return attention


def _layer(at, dev="cpu", B=2, max_pages=40):
    kv = lambda: torch.zeros((B * max_pages, 16, 2, 64), dtype=BF16, device=dev)
    table = torch.arange(B * max_pages, dtype=I32, device=dev).view(B, max_pages)
    cache = at.KVCache(kv(), kv(), table, torch.zeros(B, dtype=I32, device=dev))
    return at.AttentionLayer(cache, 8, torch.ones(1024, 64, device=dev))


def _tree(at, n, dev="cpu", B=2):
    """Chains of n nodes."""
    off = torch.arange(0, (B + 1) * n, n, dtype=I32, device=dev)
    tree = at.tw.Tree.empty(off, torch.arange(-1, n - 1, dtype=I32, device=dev).repeat(B), 1, n)
    tree.anc_mask.copy_(((1 << torch.arange(1, n + 1, dtype=torch.int64, device=dev)) - 1).repeat(B))
    return tree


@pytest.mark.parametrize("captured", [False, True])
def test_a_captured_workspace_stays(at, monkeypatch, captured):
    """No GPU: which workspaces the layer still holds once it has taken a larger one."""
    monkeypatch.setattr(at, "_capturing", lambda x: captured, raising=False)
    layer = _layer(at)
    first = weakref.ref(layer._workspace(_tree(at, 1), 0))
    size = first().numel()
    monkeypatch.setattr(at, "_capturing", lambda x: False, raising=False)
    assert layer._workspace(_tree(at, 40), 0).numel() > size
    gc.collect()
    assert (first() is not None) == captured


@pytest.mark.gpu
@pytest.mark.parametrize("step", ["verify", "token"])
def test_a_captured_round_keeps_its_workspace(at, step):
    """A larger tree makes the layer take a larger workspace; a graph that was captured ahead of that still has its own."""
    dev, gen = "cuda:0", torch.Generator().manual_seed(1)
    layer = _layer(at, dev)
    layer.cache.k.normal_(), layer.cache.v.normal_()
    layer.cache.context_len.fill_(600)
    rows = lambda n: [torch.randn(2 * n, h, 64, generator=gen).to(BF16).to(dev) for h in (8, 2, 2)]
    run = lambda tree, pos, x: (layer.verify(tree, pos, *x) if step == "verify" else layer.append_and_attend(tree, pos, *x, advance=False))
    pos = lambda n: (600 + torch.arange(n, dtype=I32)).repeat(2).to(dev)
    small, x = _tree(at, 1, dev), rows(1)
    pos1 = torch.zeros(2, dtype=I32, device=dev)                       # (table of ones: a rotation, the same each time)
    layer.cos_sin[:, :32], layer.cos_sin[:, 32:] = 1.0, 0.0
    want = run(small, pos1, x).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(small, pos1, x)
    size = layer._ws.numel()
    layer.verify(_tree(at, 60, dev), pos(60), *rows(60))
    assert layer._ws.numel() > size
    held = [torch.full((size,), 0x5a, dtype=torch.uint8, device=dev) for _ in range(4)]     # whoever is given freed memory
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(bool((h == 0x5a).all()) for h in held)


@pytest.mark.gpu
@pytest.mark.parametrize("step", ["prefill", "verify"])
def test_a_workspace_that_another_stream_is_at_is_not_handed_out(at, step):
    """Allocated on one stream, used on another, replaced there: the first stream's next allocation must not be that memory while the other
    has not come so far.  (Addresses alone are looked at.)"""
    dev = "cuda:0"
    layer, other = _layer(at, dev), _layer(at, dev)
    i32, rows = (lambda *x: torch.tensor(x, dtype=I32, device=dev)), (lambda T: [torch.zeros(T, h, 64, dtype=BF16, device=dev) for h in (8, 2, 2)])

    def run(n, x, layer=layer):
        if step == "verify":
            layer.verify(trees[n], pos[2 * n], *x)
        else:
            layer.prefill(i32_of[n], pos[2 * n], *x, advance=False)
    trees, i32_of = {n: _tree(at, n, dev) for n in (2, 40)}, {n: i32(0, n, 2 * n) for n in (2, 40)}
    pos, data = {2 * n: torch.zeros(2 * n, dtype=I32, device=dev) for n in (2, 40)}, {n: rows(2 * n) for n in (2, 40)}
    space = lambda: layer._ws if step == "verify" else layer._rows_ws
    run(40, data[40], other)                 # (what a first call loads is loaded here)
    run(2, data[2])
    where, size, side = space().data_ptr(), space().numel(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(600_000_000)       # (about a third of a second)
        run(2, data[2])
        run(40, data[40])
    assert space().numel() > size
    held = [torch.empty(size, dtype=torch.uint8, device=dev) for _ in range(8)]
    assert not side.query(), "the other stream has finished too early to show anything"
    assert where not in [h.data_ptr() for h in held]
    torch.cuda.synchronize()
