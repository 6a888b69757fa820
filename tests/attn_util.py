"""Test-side glue of the attention-layer calls: random cases, and the operators in 64 bits on the CPU, node by
node from their definitions."""
from __future__ import annotations

import math
from dataclasses import dataclass, field

import numpy as np
import torch


@dataclass
class Case:
    """Sequences with paged caches and draft trees, on the CPU."""
    dtype: torch.dtype
    L: list
    N: list
    Hq: int
    Hkv: int
    D: int
    page: int
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    kc: torch.Tensor            # [n_pages, page, Hkv, D]
    vc: torch.Tensor
    table: torch.Tensor         # [B, max_pages] int32
    offsets: torch.Tensor
    parent: torch.Tensor
    mask: torch.Tensor          # int64 view of the uint64 masks
    shared: int = 0
    shared_pages: torch.Tensor | None = None
    scale: float = 0.0
    extra: dict = field(default_factory=dict)

    @property
    def B(self):
        return len(self.L)

    @property
    def T(self):
        return int(self.offsets[-1])


def random_tree(n, rng, chain=False, max_depth=8, forest=False):
    parent, depth = [-1], [0]
    for i in range(1, n):
        p = i - 1 if chain else int(rng.integers(-1 if forest else 0, i))
        while not chain and p >= 0 and depth[p] + 1 >= max_depth:
            p = int(rng.integers(-1 if forest else 0, i))
        parent.append(p)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    mask = []
    for i, p in enumerate(parent):
        mask.append((mask[p] if p >= 0 else 0) | (1 << i))
    return parent, mask


def make_case(L, N, Hq=4, Hkv=2, D=64, page=16, dtype=torch.bfloat16, seed=0, shared=0, chain=False, forest=False,
              poison=True, room=0, max_depth=8, q_scale=1.0):
    """poison: every cache slot that no sequence may read holds NaN.  room: pages beyond what L needs."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator().manual_seed(seed)
    B, T = len(L), sum(N)
    randn = lambda *s: torch.randn(s, generator=gen).to(dtype)
    need = [-(-l // page) + room for l in L]
    sp = shared // page
    n_pages = sp + sum(n - sp for n in need) + 2
    order = rng.permutation(n_pages)
    table = np.full((B, max(max(need), 1)), -7, np.int32)   # entries that are not needed are not valid pages
    at = sp
    for b, n in enumerate(need):
        table[b, sp:n] = order[at:at + n - sp]
        at += n - sp
    kc, vc = randn(n_pages, page, Hkv, D), randn(n_pages, page, Hkv, D)
    if poison:
        keep = torch.zeros(n_pages, page, dtype=torch.bool)
        keep[order[:sp].tolist()] = True
        for b, l in enumerate(L):
            for j in range(shared, l):
                keep[int(table[b, j // page]), j % page] = True
        kc[~keep], vc[~keep] = math.nan, math.nan
    parent, mask = [], []
    for n in N:
        p, m = random_tree(n, rng, chain, max_depth, forest)
        parent += p
        mask += m
    return Case(dtype=dtype, L=list(L), N=list(N), Hq=Hq, Hkv=Hkv, D=D, page=page, q=(randn(T, Hq, D) * q_scale).to(dtype),
                k=randn(T, Hkv, D), v=randn(T, Hkv, D), kc=kc, vc=vc, table=torch.from_numpy(table),
                offsets=torch.tensor(np.concatenate([[0], np.cumsum(N)]), dtype=torch.int32),
                parent=torch.tensor(parent, dtype=torch.int32),
                mask=torch.from_numpy(np.array(mask, np.uint64).view(np.int64)), shared=shared,
                shared_pages=torch.tensor(order[:sp], dtype=torch.int32) if sp else None, scale=1.0 / math.sqrt(D))


def attn_reference(c: Case):
    """o = sum_j softmax_j(scale q.k_j) v_j in 64 bits; a node that sees nothing gets 0.  What a node may not
    see is left out of the sums, never multiplied.  Returns o and sum_j w_j |v_j|, the scale that errors of the
    weights w have in o."""
    f = lambda x: x.to(torch.float64)
    out = torch.zeros(c.T, c.Hq, c.D, dtype=torch.float64)
    size = torch.zeros_like(out)
    off, G = c.offsets.tolist(), c.Hq // c.Hkv
    masks = c.mask.numpy().view(np.uint64)
    for b in range(c.B):
        page = lambda j: int(c.shared_pages[j // c.page]) if j < c.shared else int(c.table[b, j // c.page])
        pages, slots = [page(j) for j in range(c.L[b])], [j % c.page for j in range(c.L[b])]
        past_k, past_v = f(c.kc[pages, slots]), f(c.vc[pages, slots])              # [L, Hkv, D]
        for i in range(c.N[b]):
            t = off[b] + i
            see = [off[b] + j for j in range(c.N[b]) if (int(masks[t]) >> j) & 1]
            k, v = torch.cat([past_k, f(c.k[see])]), torch.cat([past_v, f(c.v[see])])
            if k.shape[0] == 0:
                continue
            for h in range(c.Hq):
                s = (k[:, h // G] @ f(c.q[t, h])) * c.scale
                w = torch.exp(s - s.max())
                out[t, h] = (w @ v[:, h // G]) / w.sum()
                size[t, h] = (w @ v[:, h // G].abs()) / w.sum()
    return out, size


# Error bounds, per element, on o against 64 bits.  Both kernels: scores, statistics and sums in fp32; a score is
# a dot product of at most 256 terms whose absolute terms sum to about 10 here, so it is off by some
# sqrt(256) * 2^-24 * 10 = 1e-5 at most, and a weight by as much of itself: 2^-15 (3e-5) of sum w |v|.  The store rounds
# once: 2^-8 of |o| in bf16.  The tensor-core kernel rounds each weight to bf16: another 2^-8 of sum w |v|.
FP32_PART = 2.0 ** -15
BF16_HALF_ULP = 2.0 ** -8         # bf16 keeps 8 significant bits


def attn_bound(c: Case, ref, size, tensor_cores):
    tol = FP32_PART * size + 1e-30
    if c.dtype == torch.bfloat16:
        tol = tol + BF16_HALF_ULP * (ref.abs() + tol)
        if tensor_cores:
            tol = tol + BF16_HALF_ULP * (1 + BF16_HALF_ULP) * size
    return tol


def assert_attn(c: Case, O, ref, size, tensor_cores, rows=None):
    err = (O.to(torch.float64) - ref).abs()
    over = err - attn_bound(c, ref, size, tensor_cores)
    if rows is not None:
        over = over[rows]
    assert not torch.isnan(over).any(), "NaN in the output"
    assert float(over.max()) <= 0, (float(over.max()), float(err.max()))


def rope_reference(x, table, positions, pair_axis, interleaved=False, inverse=False):
    """Pair by pair in 64 bits."""
    y = x.to(torch.float64).clone()
    half = table.shape[1] // 2
    for p in range(half):
        axis = int(pair_axis[p]) if pair_axis is not None else 0
        row = table[positions[axis].long()].to(torch.float64)
        c, s = row[:, p, None], row[:, half + p, None] * (-1 if inverse else 1)
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + half)
        a, b = x[..., i].to(torch.float64), x[..., j].to(torch.float64)
        y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    return y


def rope_table(rot, top, base=10000.0):
    freq = base ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))
    angle = torch.arange(top, dtype=torch.float64)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def on_gpu(c: Case, max_nodes=0, layout="slots"):
    """The case's tensors on the device, as the library's handles.  layout: "slots" keeps [page, slot, head, d],
    "heads" stores [page, head, slot, d]."""
    from paper_2608_20961_b200 import attention as at, binding as tw
    dev = torch.device("cuda:0")
    d = lambda t: t.to(dev)
    kc, vc = d(c.kc), d(c.vc)
    if layout == "heads":
        kc, vc = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kc, vc))
    # q, k, v as column ranges of one projection's output
    T = c.T
    qkv = torch.cat([x.reshape(T, -1) for x in (c.q, c.k, c.v)], 1).to(dev)
    nq, nk = c.Hq * c.D, c.Hkv * c.D
    g = dict(q=qkv[:, :nq].view(T, c.Hq, c.D), k=qkv[:, nq:nq + nk].view(T, c.Hkv, c.D),
             v=qkv[:, nq + nk:].view(T, c.Hkv, c.D))
    g["cache"] = at.KVCache(kc, vc, d(c.table), d(torch.tensor(c.L, dtype=torch.int32)))
    tree = tw.Tree.empty(d(c.offsets), d(c.parent), 1, max_nodes)
    tree.anc_mask = d(c.mask)
    g["tree"] = tree
    g["shared_pages"] = None if c.shared_pages is None else d(c.shared_pages)
    return g


def run_attn(c: Case, generic=False, max_nodes=0, layout="slots", status=None, canary=7.25):
    """O and the status words of one treewy_attn_verify call, on the CPU."""
    from paper_2608_20961_b200 import attention as at
    g = on_gpu(c, max_nodes, layout)
    O = torch.full((c.T, c.Hq, c.D), canary, dtype=c.dtype, device="cuda:0")
    status = torch.zeros(c.B, dtype=torch.int32, device="cuda:0")
    ws = at.attn_workspace(g["cache"], g["tree"], c.Hq, c.shared)
    ws.fill_(0xff)                                    # whatever it holds must not matter (all NaN here)
    at.treewy_attn_verify(g["cache"], g["tree"], g["q"], g["k"], g["v"], c.scale, O, ws, g["shared_pages"], c.shared,
                          status, generic=generic)
    torch.cuda.synchronize()
    return O.cpu(), status.cpu().tolist()
