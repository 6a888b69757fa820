"""What is measured of the operators that take a prompt through an attention layer: attention of new rows over a paged
cache (whole, or a sliding window beside a few first tokens), norms of queries and keys with the rotation in the same
pass (written to the cache, or backward), and the page table's upkeep.

``own = False`` computes each operator in its plain form (elementary torch operations in 32 bits);
``own = True`` calls the library.  Both work on what ``prepare`` makes.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # a long prompt in one go
        dict(name="chunk prompt 8k", op="attn", dtype="bf16", B=1, new=8192, mix=0, ctx=0, window=0, sinks=0,
             Hq=32, Hkv=8, D=128, page=16),
        # a serving step with wide heads: some prompts' pieces among sequences that decode
        dict(name="chunk mixed batch", op="attn", dtype="bf16", B=37, new=777, mix=1, ctx=8192, window=0, sinks=0,
             Hq=16, Hkv=2, D=256, page=32),
        # a question of some hundred tokens behind a long document
        dict(name="chunk behind 64k", op="attn", dtype="bf16", B=1, new=301, mix=0, ctx=65537, window=0, sinks=0,
             Hq=32, Hkv=8, D=128, page=64),
        # a layer with a window: a batch of prompts
        dict(name="window prompt", op="attn", dtype="bf16", B=3, new=4999, mix=0, ctx=1000, window=1024, sinks=4,
             Hq=32, Hkv=8, D=64, page=16),
        # the same layer kind decoding: one token each, long contexts of which a window is left
        dict(name="window decode", op="attn", dtype="bf16", B=64, new=1, mix=0, ctx=12001, window=4096, sinks=4,
             Hq=32, Hkv=8, D=128, page=16),
        # 32-bit inputs, three heads to a group, small pages: what a numerics check of a layer runs
        dict(name="window f32 odd", op="attn", dtype="f32", B=4, new=77, mix=0, ctx=333, window=100, sinks=3,
             Hq=6, Hkv=2, D=80, page=8),
        # one new token for each sequence of a batch, normalised, rotated and written
        dict(name="norm append decode", op="append", dtype="bf16", B=64, new=1, ctx=1001, Hq=32, Hkv=8, D=128, rot=128,
             axes=1, page=16),
        # prompts of up to 4k tokens, a quarter of each wide head rotated
        dict(name="norm append prompt", op="append", dtype="bf16", B=5, new=4097, ctx=130, Hq=16, Hkv=2, D=256, rot=64,
             axes=3, page=32),
        # training: gradients of the queries of a batch of rows
        dict(name="norm backward", op="backward", dtype="bf16", T=8199, H=32, D=128, rot=128, axes=1, interleaved=0),
        # 32 bits, few rows, odd heads, pairs side by side, part of the head rotated
        dict(name="norm backward f32", op="backward", dtype="f32", T=61, H=5, D=80, rot=48, axes=1, interleaved=1),
        # between two rounds of a decoding batch: pages of rejected drafts go back, the next round's are taken
        dict(name="pages decode", op="pages", B=64, new=9, ctx=4000, page=16),
        # prompts join a large batch
        dict(name="pages prompts", op="pages", B=509, new=1023, ctx=300, page=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "attn", "norm", "append", "backward", "pages"])
    if op == "pages":
        return dict(op=op, B=_log(rng, 1, 600), new=_log(rng, 1, 1000), ctx=_log(rng, 1, 5000),
                    page=rng.choice([8, 16, 24, 64]))
    if op in ("norm", "backward"):
        D = rng.choice([64, 80, 96, 128, 256])
        return dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), T=_log(rng, 1, 8000), H=rng.randint(1, 24), D=D,
                    rot=rng.choice([D, D // 2, 32]), axes=rng.choice([1, 2, 3]), interleaved=rng.randint(0, 1))
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8])
    D, page = rng.choice([64, 128, 256]), rng.choice([8, 16, 32, 64, 128])
    if op == "append":
        return dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), B=rng.randint(1, 32), new=_log(rng, 1, 300),
                    ctx=_log(rng, 1, 2000), Hq=Hkv * G, Hkv=Hkv, D=D, rot=rng.choice([D, D // 4]),
                    axes=rng.choice([1, 3]), page=page)
    windowed = rng.random() < 0.5
    mix = rng.randint(0, 1)
    if rng.random() < 0.2:      # 32-bit inputs run at the sizes of a check
        return dict(op=op, dtype="f32", B=rng.randint(1, 6), new=_log(rng, 1, 200), mix=mix, ctx=_log(rng, 1, 1000),
                    window=_log(rng, 1, 500) if windowed else 0, sinks=rng.choice([0, 1, 4, 70]) if windowed else 0,
                    Hq=Hkv * G, Hkv=Hkv, D=D, page=page)
    ctx, new = _log(rng, 1, 30000), _log(rng, 1, 6000)
    while (ctx + new) * new * Hkv * G > 1_500_000_000:      # the scores of a sequence stay below the largest listed one's
        new = max(1, new // 2)
    room = min(600_000_000 // ((ctx + new) * Hkv * D), 1_500_000_000 // ((ctx + new) * new * Hkv * G))
    return dict(op=op, dtype="bf16", B=_log(rng, 1, max(1, min(48, room))), new=new, mix=mix, ctx=ctx,
                window=_log(rng, 1, 5000) if windowed else 0, sinks=rng.choice([0, 1, 4, 4, 130]) if windowed else 0,
                Hq=Hkv * G, Hkv=Hkv, D=D, page=page)


# ------------------------------------------------------------------------------------------ inputs

def _sizes(case, seed):
    """Context lengths and new rows of each sequence, as lists; the latter are the case's own, so that outputs have the
    same shape whatever the seed."""
    r, own_r = np.random.RandomState(seed % (1 << 31)), np.random.RandomState(7)
    B, ctx, most = case["B"], case["ctx"], case["new"]
    L = r.randint(ctx // 4, ctx + 1, B)
    L[r.randint(B)] = ctx
    N = own_r.randint((most + 1) // 2, most + 1, B)
    if case.get("mix"):         # most of the batch decodes
        N = np.where(own_r.rand(B) < 0.8, 1, N)
    N[own_r.randint(B)] = most
    return L.tolist(), N.tolist(), r


def _rotary(case, T, top, gen):
    """Table of cosines and sines, positions on each axis, and the axis of each pair."""
    rot, axes = case["rot"], case["axes"]
    freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) / (rot // 2))
    angle = torch.arange(top, dtype=torch.float64, device=DEV)[:, None] * freq
    table = torch.cat([angle.cos(), angle.sin()], 1).float()
    positions = torch.randint(top, (axes, T), generator=gen, device=DEV, dtype=torch.int32)
    pair_axis = (torch.arange(rot // 2, device=DEV) * axes // (rot // 2)).to(torch.uint8)
    return table, positions, pair_axis


def _int(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _table(r, room, page, max_pages, n_pages):
    """Pages dealt out in random order for `room` slots of each sequence; -1 behind them.  Also the pages left over."""
    free = r.permutation(n_pages).astype(np.int32)
    need = -(-np.asarray(room) // page)
    table, at = np.full((len(room), max_pages), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = free[at:at + n]
        at += n
    return table, free[at:]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    if op == "pages":
        return _prepare_pages(case, seed)
    dtype, D = DTYPES[case["dtype"]], case["D"]
    rand = lambda *s: torch.randn(s, generator=gen, device=DEV, dtype=dtype)
    weight = lambda: 1.0 + 0.2 * torch.randn(D, generator=gen, device=DEV)
    s = dict(case=case, scale=1.0 / math.sqrt(D), eps=1e-6)
    if op in ("norm", "backward"):
        T, H = case["T"], case["H"]
        s["x"], s["w"] = rand(T, H, D), weight().to(dtype)
        if op == "backward":
            s["dy"] = rand(T, H, D)
        s["table"], s["positions"], s["pair_axis"] = _rotary(case, T, 4096, gen)
    else:
        L, N, r = _sizes(case, seed)
        B, T, Hq, Hkv, page = case["B"], sum(N), case["Hq"], case["Hkv"], case["page"]
        s.update(T=T, B=B, N=N, context_len=_int(L), L=L, offsets=_int(np.concatenate([[0], np.cumsum(N)])))
        # queries, keys and values of the packed rows come out of one projection, side by side
        qkv = rand(T, (Hq + 2 * Hkv) * D)
        s["q"] = qkv[:, :Hq * D].view(T, Hq, D)
        s["k"] = qkv[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D)
        s["v"] = qkv[:, (Hq + Hkv) * D:].view(T, Hkv, D)
        room = [a + b for a, b in zip(L, N)]
        most = -(-(case["ctx"] + case["new"]) // page)
        n_pages = sum(-(-(case["ctx"] + n) // page) for n in N) + 3
        table, _ = _table(r, room, page, most, n_pages)
        s["page_table"] = torch.from_numpy(table).to(DEV)
        s["kc"], s["vc"] = (rand(n_pages, page, Hkv, D) for _ in range(2))
        if op == "append":
            s["seq"] = torch.from_numpy(np.repeat(np.arange(B), N)).to(DEV)
            s["local"] = torch.from_numpy(np.concatenate([np.arange(n) for n in N])).to(DEV)
            s["table"], s["positions"], s["pair_axis"] = _rotary(case, T, case["ctx"] + case["new"], gen)
            s["wq"], s["wk"] = weight().to(dtype), weight().to(dtype)
    if own:
        _handles(s)
    return s


def _prepare_pages(case, seed):
    L, N, r = _sizes(case, seed)
    B, page = case["B"], case["page"]
    most = -(-(case["ctx"] + case["new"] + case["new"]) // page)
    n_pages = B * most + 5
    # the drafts of the round before had reserved more than was kept of them
    ahead = [a + int(r.randint(0, case["new"] + 1)) for a in L]
    table, left = _table(r, ahead, page, most, n_pages)
    free = np.zeros(n_pages, np.int32)
    free[:len(left)] = left
    s = dict(case=case, T=sum(N), B=B, L=L, N=N, context_len=_int(L), n_pages=n_pages,
             offsets=_int(np.concatenate([[0], np.cumsum(N)])), page_table=torch.from_numpy(table).to(DEV),
             free=torch.from_numpy(free).to(DEV), count=_int([len(left)]), end=_int([most * page] * B))
    if own:
        from paper_2608_20961_b200 import attention as at
        s["pool"] = at.PagePool(s["page_table"], page, n_pages, s["free"], s["count"])
    return s


def _handles(s):
    """What a program that uses the library keeps beside its tensors."""
    from paper_2608_20961_b200 import attention as at
    case = s["case"]
    if "table" in s:
        s["rope"] = at.Rope(s["table"], s["positions"], s["pair_axis"], interleaved=bool(case.get("interleaved", 0)))
    for name in ("w", "wq", "wk"):
        if name in s:
            s["norm_" + name] = at.HeadNorm(s[name], s["eps"])
    if "kc" in s:
        s["cache"] = at.KVCache(s["kc"], s["vc"], s["page_table"], s["context_len"])
    if case["op"] == "attn":
        s["workspace"] = at.attn_chunk_workspace(s["cache"], s["T"], case["Hq"], case["window"], case["sinks"])
    if case["op"] == "backward":
        s["workspace"] = at.norm_rope_workspace(s["x"])


# -------------------------------------------------------------------------------------- plain forms

def _rotate(x, s, interleaved, inverse):
    """x [T, H, D] in 32 bits, its first rot elements rotated in pairs."""
    table, half = s["table"], s["table"].shape[1] // 2
    at = s["positions"].long()[s["pair_axis"].long()].T            # [T, half]: each pair's position
    pair = torch.arange(half, device=x.device)
    cos, sin = table[at, pair][:, None], table[at, pair + half][:, None]
    if inverse:
        sin = -sin
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def _normed(x, eps):
    """x in 32 bits over its root mean square, and one over that."""
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    return x * r, r


def _plain_norm(s):
    x, _ = _normed(s["x"].float(), s["eps"])
    return _rotate(x * s["w"].float(), s, s["case"]["interleaved"], False).to(s["x"].dtype)


def _plain_backward(s):
    g = _rotate(s["dy"].float(), s, s["case"]["interleaved"], True)
    xn, r = _normed(s["x"].float(), s["eps"])
    dw = (g * xn).sum((0, 1))
    g = g * s["w"].float()
    dx = r * (g - xn * (g * xn).mean(-1, keepdim=True))
    return dx.to(s["x"].dtype), dw


def _plain_append(s):
    page = s["case"]["page"]
    turn = lambda x, w: _rotate(_normed(x.float(), s["eps"])[0] * w.float(), s, 0, False).to(x.dtype)
    slot = s["context_len"].long()[s["seq"]] + s["local"]
    at = s["page_table"].long()[s["seq"], slot // page]
    s["kc"][at, slot % page] = turn(s["k"], s["wk"])
    s["vc"][at, slot % page] = s["v"]
    return turn(s["q"], s["wq"]), s["kc"], s["vc"]


def _plain_attn(s):
    c = s["case"]
    Hq, Hkv, D, page = c["Hq"], c["Hkv"], c["D"], c["page"]
    G, W = Hq // Hkv, c["window"] or (1 << 30)
    out, lo = torch.empty((s["T"], Hq, D), dtype=s["q"].dtype, device=DEV), 0
    for b, (L, n) in enumerate(zip(s["L"], s["N"])):
        # cached tokens that some row sees, and the rows' own positions
        first = max(0, L - W + 1)
        x = torch.cat([torch.arange(min(c["sinks"], first), device=DEV), torch.arange(first, L + n, device=DEV)])
        at = s["page_table"][b].long()[x // page]
        keys, values = (t[at, x % page].float().transpose(0, 1) for t in (s["kc"], s["vc"]))    # [Hkv, X, D]
        for i in range(0, n, 2048):
            m = min(2048, n - i)
            p = L + i + torch.arange(m, device=DEV)
            sees = (x <= p[:, None]) & ((x > p[:, None] - W) | (x < c["sinks"]))                # [m, X]
            q = s["q"][lo + i:lo + i + m].float().view(m, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, m * G, D)
            score = ((q @ keys.transpose(1, 2)) * s["scale"]).view(Hkv, m, G, -1)
            score = score.masked_fill_(~sees[:, None], -math.inf)
            w = (score - score.amax(-1, keepdim=True)).exp_()
            o = (w.view(Hkv, m * G, -1) @ values).view(Hkv, m, G, D) / w.sum(-1, keepdim=True)
            out[lo + i:lo + i + m] = o.permute(1, 0, 2, 3).reshape(m, Hq, D).to(out.dtype)
        lo += n
    return out


def _plain_pages(s):
    page, table, free, count = s["case"]["page"], s["page_table"], s["free"], s["count"]
    e = torch.arange(table.shape[1], device=DEV)
    L, off = s["context_len"].long(), s["offsets"].long()
    n = off[1:] - off[:-1]
    # pages behind what is kept go back: in the order in which they would be taken again
    gone = (e >= ((L + page - 1) // page)[:, None]) & (table >= 0)
    pages = table[gone]
    top = count.long() + pages.numel()
    free[(top - 1 - torch.arange(pages.numel(), device=DEV)).long()] = pages
    table[gone] = -1
    # pages for the new rows
    want = (e >= (L // page)[:, None]) & (e <= ((L + n - 1) // page)[:, None]) & (table < 0) & (n > 0)[:, None]
    rank = want.flatten().cumsum(0).view(want.shape) - 1
    table[want] = free[(top - 1 - rank[want]).long()]
    count.copy_(top - want.sum())
    row = torch.arange(s["T"], device=DEV)
    b = torch.searchsorted(off, row, right=True) - 1
    position = L[b] + row - off[b]
    return table, free, count, position.to(torch.int32), table.long()[b, position // page] * page + position % page


# ------------------------------------------------------------------------------------------- passes

def _own(s):
    from paper_2608_20961_b200 import attention as at
    c = s["case"]
    if c["op"] == "norm":
        y = torch.empty_like(s["x"])
        at.treewy_norm_rope(s["norm_w"], s["rope"], s["x"], y)
        return y
    if c["op"] == "backward":
        dx, dw = torch.empty_like(s["x"]), torch.empty(c["D"], device=DEV)
        at.treewy_norm_rope_backward(s["norm_w"], s["rope"], s["x"], s["dy"], dx, dw, s["workspace"])
        return dx, dw
    if c["op"] == "append":
        q_out = torch.empty((s["T"], c["Hq"], c["D"]), dtype=s["q"].dtype, device=DEV)
        at.treewy_kv_append_norm(s["cache"], s["offsets"], s["k"], s["v"], s["norm_wk"], s["rope"], s["q"], q_out,
                                 s["norm_wq"])
        return q_out, s["kc"], s["vc"]
    if c["op"] == "pages":
        position = torch.empty(s["T"], dtype=torch.int32, device=DEV)
        slots = torch.empty(s["T"], dtype=torch.int64, device=DEV)
        at.treewy_pages_release(s["pool"], s["context_len"], s["end"])
        at.treewy_pages_reserve(s["pool"], s["context_len"], s["offsets"], s["T"], position, slots)
        return s["page_table"], s["free"], s["count"], position, slots
    O = torch.empty((s["T"], c["Hq"], c["D"]), dtype=s["q"].dtype, device=DEV)
    at.treewy_attn_chunk(s["cache"], s["offsets"], s["q"], s["scale"], O, s["workspace"], c["window"], c["sinks"])
    return O


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "backward": _plain_backward, "append": _plain_append, "attn": _plain_attn,
            "pages": _plain_pages}[state["case"]["op"]](state)


# -------------------------------------------------------------------------------- work and 64 bits

def work(case):
    op = case["op"]
    if op == "pages":
        L, N, _ = _sizes(case, 1)
        taken = sum(-(-(a + n) // case["page"]) + -(-a // case["page"]) * -1 for a, n in zip(L, N))
        return {"bytes": 12 * sum(N) + 16 * taken + 16 * case["B"], "flops": 0}
    e, D = DTYPES[case["dtype"]].itemsize, case["D"]
    if op in ("norm", "backward"):
        rows, moved = case["T"] * case["H"], 2 if op == "norm" else 3
        return {"bytes": moved * rows * D * e + case["axes"] * case["T"] * 4, "flops": (6 if op == "norm" else 14) * rows * D}
    L, N, _ = _sizes(case, 1)
    T, Hq, Hkv = sum(N), case["Hq"], case["Hkv"]
    if op == "append":
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * D * e + case["axes"] * T * 4, "flops": 6 * T * (Hq + Hkv) * D}
    W, sinks = case["window"] or (1 << 30), case["sinks"]
    keys = seen = 0
    for a, n in zip(L, N):
        first = max(0, a - W + 1)
        keys += a + n - first + min(sinks, first)
        p = np.arange(a, a + n, dtype=np.int64)
        lo = np.maximum(0, p - W + 1)
        seen += int((p + 1 - lo + np.minimum(lo, sinks)).sum())
    return {"bytes": 2 * keys * Hkv * D * e + 2 * T * Hq * D * e, "flops": 4 * D * Hq * seen}


def exact(case, seed):
    """Sequence by sequence, head by head and pair by pair in 64 bits, from the definitions."""
    s = prepare(case, seed)
    if case["op"] == "pages":
        return _exact_pages(case, s)
    f64 = lambda x: x.to(torch.float64)
    if case["op"] == "attn":
        out, lo, G = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV), 0, case["Hq"] // case["Hkv"]
        for b, (L, n) in enumerate(zip(s["L"], s["N"])):
            pages = s["page_table"][b, :-(-(L + n) // case["page"])].long()
            i, x = torch.arange(L, L + n, device=DEV)[:, None], torch.arange(L + n, device=DEV)
            hidden = x > i
            if case["window"]:
                hidden |= (i - x >= case["window"]) & (x >= case["sinks"])
            for h in range(case["Hq"]):
                past = lambda c: f64(c[pages, :, h // G].reshape(-1, case["D"])[:L + n])
                e = torch.exp((f64(s["q"][lo:lo + n, h]) @ past(s["kc"]).T * s["scale"]).clamp_(max=600.0))
                e[hidden] = 0.0
                out[lo:lo + n, h] = (e @ past(s["vc"])) / e.sum(1)[:, None]
            lo += n
        return out
    half, wave = case["rot"] // 2, f64(s["table"])

    def turn(x, sign, side_by_side):
        y = x.clone()
        for p in range(half):
            i, j = (2 * p, 2 * p + 1) if side_by_side else (p, p + half)
            row = wave[s["positions"][int(s["pair_axis"][p])].long()]
            z = torch.complex(x[..., i].contiguous(), x[..., j].contiguous()) * torch.complex(row[:, p], sign * row[:, p + half])[:, None]
            y[..., i], y[..., j] = z.real, z.imag
        return y

    size = lambda x: (f64(x).square().sum(-1, keepdim=True) / case["D"] + s["eps"]).sqrt()
    if case["op"] == "norm":
        return turn(f64(s["x"]) / size(s["x"]) * f64(s["w"]), 1.0, case["interleaved"])
    if case["op"] == "backward":
        g, x, m = turn(f64(s["dy"]), -1.0, case["interleaved"]), f64(s["x"]), size(s["x"])
        dw = torch.einsum("thd,thd->d", g, x / m)
        g = g * f64(s["w"])
        return g / m - x * (g * x).sum(-1, keepdim=True) / (case["D"] * m ** 3), dw
    kc, vc = f64(s["kc"]), f64(s["vc"])
    q = turn(f64(s["q"]) / size(s["q"]) * f64(s["wq"]), 1.0, 0)
    k = turn(f64(s["k"]) / size(s["k"]) * f64(s["wk"]), 1.0, 0)
    table, page, lo = s["page_table"].tolist(), case["page"], 0
    for b, (L, n) in enumerate(zip(s["L"], s["N"])):
        slots = range(L, L + n)
        pages, places = [table[b][x // page] for x in slots], [x % page for x in slots]
        kc[pages, places], vc[pages, places] = k[lo:lo + n], f64(s["v"][lo:lo + n])
        lo += n
    return q, kc, vc


def _exact_pages(case, s):
    """The same upkeep with a list for a stack, one page at a time."""
    page, table, free = case["page"], s["page_table"].tolist(), s["free"].tolist()
    top, back, position, slots = int(s["count"]), [], [], []
    for b, L in enumerate(s["L"]):
        for e in range(-(-L // page), len(table[b])):
            if table[b][e] >= 0:
                back.append(table[b][e])
                table[b][e] = -1
    for p in reversed(back):
        free[top] = p
        top += 1
    for b, (L, n) in enumerate(zip(s["L"], s["N"])):
        for x in range(L, L + n):
            if table[b][x // page] < 0:
                top -= 1
                table[b][x // page] = free[top]
            position.append(x)
            slots.append(table[b][x // page] * page + x % page)
    return _int(table), _int(free), _int([top]), _int(position), torch.tensor(slots, device=DEV)
