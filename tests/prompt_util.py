"""Test-side glue of the calls that take new rows through an attention layer: random cases, and the operators in 64 bits from
their definitions."""
from __future__ import annotations

import math
from dataclasses import dataclass

import numpy as np
import torch

from tests import attn_util as au

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
HALF_STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}   # of a rounding, relative to the value


@dataclass
class Case:
    """New rows behind paged contexts; the rows' own keys and values are in the cache.  On the CPU."""
    dtype: torch.dtype
    L: list
    N: list
    Hq: int
    Hkv: int
    D: int
    page: int
    window: int
    sinks: int
    q: torch.Tensor
    kc: torch.Tensor            # [n_pages, page, Hkv, D]
    vc: torch.Tensor
    table: torch.Tensor
    offsets: torch.Tensor
    scale: float
    T: int

    @property
    def B(self):
        return len(self.L)

    def seen(self, p):
        """Tokens that the row at position p sees."""
        first = max(0, p - self.window + 1) if self.window else 0
        return list(range(min(self.sinks, first))) + list(range(first, p + 1))


def make_case(L, N, Hq=4, Hkv=2, D=64, page=16, window=0, sinks=0, dtype=BF16, seed=0, poison=True, q_scale=1.0, gaps=None):
    """poison: every slot that no row sees holds NaN, and table entries without a token that is seen are no pages.  gaps: packed
    rows of no sequence ahead of each sequence."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator().manual_seed(seed)
    B = len(L)
    gaps = gaps or [0] * (B + 1)
    randn = lambda *s: torch.randn(s, generator=gen).to(dtype)
    assert sum(gaps) == 0 or B == 1, "offsets leave no room between sequences"
    offsets = np.concatenate([[0], np.cumsum(N)]) + gaps[0]
    T = int(offsets[-1]) + (gaps[-1] if sum(gaps) else 0)
    need = [-(-(l + n) // page) for l, n in zip(L, N)]
    n_pages = sum(need) + 2
    order = rng.permutation(n_pages)
    table = np.full((B, max(max(need), 1)), -7, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    c = Case(dtype, list(L), list(N), Hq, Hkv, D, page, window, sinks, (randn(T, Hq, D) * q_scale).to(dtype),
             randn(n_pages, page, Hkv, D), randn(n_pages, page, Hkv, D), torch.from_numpy(table),
             torch.tensor(offsets, dtype=torch.int32), 1.0 / math.sqrt(D), T)
    if poison:
        keep = torch.zeros(n_pages, page, dtype=torch.bool)
        for b in range(B):
            used = {x for p in (L[b], L[b] + N[b] - 1) for x in c.seen(p)} | set(range(L[b], L[b] + N[b])) if N[b] else set()
            if N[b] and window:
                used |= {x for p in range(L[b], L[b] + N[b]) for x in c.seen(p)}
            for x in used:
                keep[int(table[b, x // page]), x % page] = True
            for e in range(need[b]):
                if not any(e * page <= x < (e + 1) * page for x in used):
                    c.table[b, e] = -7
        c.kc[~keep], c.vc[~keep] = math.nan, math.nan
    return c


def chunk_reference(c: Case):
    """o = sum_x softmax_x(scale q.k_x) v_x over the tokens a row sees, in 64 bits; what it does not see is left out of
    the sums.  Returns o and sum_x w_x |v_x|, the scale that errors of the weights w have in o."""
    out = torch.zeros(c.T, c.Hq, c.D, dtype=F64)
    size, G = torch.zeros_like(out), c.Hq // c.Hkv
    for b in range(c.B):
        row = c.table[b].long()
        for i in range(c.N[b]):
            x = torch.tensor(c.seen(c.L[b] + i))
            t = int(c.offsets[b]) + i
            k, v = (s[row[x // c.page], x % c.page].to(F64).repeat_interleave(G, 1) for s in (c.kc, c.vc))
            s = torch.einsum("xhd,hd->xh", k, c.q[t].to(F64)) * c.scale
            w = torch.exp(s - s.amax(0))
            out[t], size[t] = (torch.einsum("xh,xhd->hd", w, y) / w.sum(0)[:, None] for y in (v, v.abs()))
    return out, size


def chunk_reference_gpu(c: Case):
    """The same for larger cases without NaN, whole rows at a time on the GPU."""
    out = torch.zeros(c.T, c.Hq, c.D, dtype=F64)
    size, G = torch.zeros_like(out), c.Hq // c.Hkv
    kc, vc, q = c.kc.cuda(), c.vc.cuda(), c.q.cuda()
    for b in range(c.B):
        if c.N[b] == 0:
            continue
        lo, L, n = int(c.offsets[b]), c.L[b], c.N[b]
        pages = c.table[b, :-(-(L + n) // c.page)].long().clamp(min=0).cuda()
        p, x = torch.arange(L, L + n, device="cuda")[:, None], torch.arange(L + n, device="cuda")
        hidden = x > p
        if c.window:
            hidden |= (p - x >= c.window) & (x >= c.sinks)
        for h in range(c.Hq):
            k, v = (s[pages, :, h // G].reshape(-1, c.D)[:L + n].to(F64) for s in (kc, vc))
            v = torch.where(hidden.all(0)[:, None], 0.0, v)
            s = ((q[lo:lo + n, h].to(F64) @ k.T) * c.scale).masked_fill_(hidden, -math.inf)
            w = torch.exp(s - s.amax(1, keepdim=True))
            total = w.sum(1, keepdim=True)
            out[lo:lo + n, h], size[lo:lo + n, h] = ((w @ y / total).cpu() for y in (v, v.abs()))
    return out, size


def assert_chunk(c: Case, O, ref, size, tensor_cores, rows=None):
    """The bounds of tests/attn_util.py: the same arithmetic."""
    au.assert_attn(c, O, ref, size, tensor_cores, rows)


def on_gpu(c: Case, layout="slots"):
    from paper_2608_20961_b200 import attention as at
    d = lambda t: t.to("cuda:0")
    kc, vc = d(c.kc), d(c.vc)
    if layout == "heads":
        kc, vc = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kc, vc))
    wide = torch.cat([d(c.q).reshape(c.T, -1), torch.full((c.T, 64), 3.0, dtype=c.dtype, device="cuda:0")], 1)
    return dict(cache=at.KVCache(kc, vc, d(c.table), d(torch.tensor(c.L, dtype=torch.int32))), offsets=d(c.offsets),
                q=wide[:, :c.Hq * c.D].view(c.T, c.Hq, c.D))


def run_chunk(c: Case, generic=False, layout="slots", canary=7.25):
    """O and the status words of one call, on the CPU."""
    from paper_2608_20961_b200 import attention as at
    g = on_gpu(c, layout)
    O = torch.full((c.T, c.Hq, c.D), canary, dtype=c.dtype, device="cuda:0")
    status = torch.zeros(c.B, dtype=torch.int32, device="cuda:0")
    ws = at.attn_chunk_workspace(g["cache"], c.T, c.Hq, c.window, c.sinks)
    ws.fill_(0xff)                                    # whatever it holds must not matter (all NaN here)
    at.treewy_attn_chunk(g["cache"], g["offsets"], g["q"], c.scale, O, ws, c.window, c.sinks, status, generic=generic)
    torch.cuda.synchronize()
    return O.cpu(), status.cpu().tolist()


# ------------------------------------------------------------------------------------------ norms

def rotate(x, rope, inverse=False):
    return x if rope is None else au.rope_reference(x, *rope, inverse=inverse)


def norm_reference(x, w, eps, rope=None, plus_one=False):
    """rope: table, positions, pair_axis, interleaved.  64 bits."""
    x, w = x.to(F64), w.to(F64) + (1 if plus_one else 0)
    return rotate(w * x / (x.square().mean(-1, keepdim=True) + eps).sqrt(), rope)


def norm_backward_reference(x, w, eps, dy, rope=None, plus_one=False):
    x, w, g = x.to(F64), w.to(F64) + (1 if plus_one else 0), rotate(dy.to(F64), rope, inverse=True)
    r = (x.square().mean(-1, keepdim=True) + eps) ** -0.5
    n = x * r
    return r * (w * g - n * (w * g * n).mean(-1, keepdim=True)), (g * n).sum((0, 1))


def pair_size(x, rope):
    """|a| + |b| of each element's pair: what errors of a rotated pair are relative to."""
    y = x.abs().clone()
    if rope is not None:
        half = rope[0].shape[1] // 2
        for p in range(half):
            i, j = (2 * p, 2 * p + 1) if rope[3] else (p, p + half)
            y[..., i] = y[..., j] = x[..., i].abs() + x[..., j].abs()
    return y


# ------------------------------------------------------------------------------------------ pages

class Pages:
    """The page table's upkeep with a list for a stack, one page at a time."""

    def __init__(self, table, free, count, page, n_pages):
        self.table, self.free, self.count, self.page, self.n_pages = [list(r) for r in table], list(free), count, page, n_pages

    def release(self, first, end):
        back, status = [], [0] * len(first)
        for b, row in enumerate(self.table):
            for e in range(len(row)):
                if max(first[b], 0) <= e * self.page and (e + 1) * self.page <= end[b] and row[e] >= 0:
                    back.append((b, row[e]))
                    row[e] = -1
        for b, p in reversed(back):
            if p >= self.n_pages or self.count >= self.n_pages:
                status[b] |= 64
            else:
                self.free[self.count] = p
                self.count += 1
        return status

    def reserve(self, L, off, T):
        """Status words, positions and slots (None: left)."""
        status, position, slot = [0] * len(L), [None] * T, [None] * T
        start, wanted = self.count, 0
        for b, row in enumerate(self.table):
            lo, n, ln = off[b], off[b + 1] - off[b], L[b]
            if lo < 0 or n < 0 or lo + n > T:
                status[b] |= 32
                continue
            if ln < 0 or ln + n > len(row) * self.page:
                status[b] |= 128
                continue
            es = range(ln // self.page, (ln + n - 1) // self.page + 1) if n else []
            if n and ln % self.page and not 0 <= row[es[0]] < self.n_pages:
                status[b] |= 64
                es = []
            if any(row[e] >= self.n_pages for e in es):
                status[b] |= 64
            want = [e for e in es if row[e] < 0]
            wanted += len(want)
            if want and wanted > start:
                status[b] |= 512
            else:
                for e in want:
                    self.count -= 1
                    p = self.free[self.count]
                    if 0 <= p < self.n_pages:
                        row[e] = p
                    else:
                        status[b] |= 64
            for j in range(n):
                x = ln + j
                p = row[x // self.page]
                position[lo + j] = x
                slot[lo + j] = p * self.page + x % self.page if 0 <= p < self.n_pages else -1
        return status, position, slot
