"""What is measured of the attention-layer operators: rotary positions, writes to a paged key/value
cache, draft-tree attention over that cache, and the commit of an accepted path.

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
        # one user, one token at a time: the latency of a decoding step's attention
        dict(name="attn decode one", op="attn", dtype="bf16", B=1, nodes=1, chain=1, ctx=1023, ragged=0, shared=0,
             Hq=32, Hkv=8, D=128, page=16),
        # a full decoding batch with contexts of every length up to 8k
        dict(name="attn decode batch", op="attn", dtype="bf16", B=64, nodes=1, chain=1, ctx=8192, ragged=1, shared=0,
             Hq=32, Hkv=8, D=128, page=16),
        # draft trees of up to 32 nodes verified through a layer with wide heads
        dict(name="attn tree 32", op="attn", dtype="bf16", B=32, nodes=32, chain=0, ctx=8192, ragged=1, shared=0,
             Hq=16, Hkv=2, D=256, page=16),
        # two long documents with a chain of drafts: few rows, a long axis to split
        dict(name="attn long chain", op="attn", dtype="bf16", B=2, nodes=5, chain=1, ctx=65537, ragged=0, shared=0,
             Hq=32, Hkv=8, D=128, page=64),
        # many requests under one system prompt, each with a short context and a small tree of its own
        dict(name="attn shared prompt", op="attn", dtype="bf16", B=64, nodes=8, chain=0, ctx=4609, ragged=1,
             shared=4096, Hq=32, Hkv=8, D=128, page=16),
        # 32-bit inputs, three heads to a group, small pages: what a numerics check of a layer runs
        dict(name="attn f32 odd", op="attn", dtype="f32", B=5, nodes=3, chain=0, ctx=777, ragged=1, shared=0,
             Hq=6, Hkv=2, D=64, page=8),
        # queries and keys of an image or video prompt: time, height and width
        dict(name="rope three axes", op="rope", dtype="bf16", T=8199, H=24, D=128, rot=128, axes=3, inverse=0,
             interleaved=0),
        # gradients of a short prompt on the way back, pairs side by side, part of the head rotated
        dict(name="rope backward f32", op="rope", dtype="f32", T=61, H=5, D=80, rot=48, axes=1, inverse=1,
             interleaved=1),
        # one new token for each sequence of a batch
        dict(name="append decode", op="append", dtype="bf16", B=64, new=1, ctx=1001, Hq=32, Hkv=8, D=128, rot=128,
             axes=1, page=16),
        # prompts of up to 4k tokens written in one go, a quarter of each head rotated
        dict(name="append prompt", op="append", dtype="bf16", B=5, new=4097, ctx=130, Hq=16, Hkv=2, D=256, rot=64,
             axes=3, page=32),
        # accepted paths of trees of 32 nodes
        dict(name="commit tree 32", op="commit", dtype="bf16", B=64, nodes=32, chain=0, ctx=900, Hkv=2, D=256,
             page=16),
        # accepted drafts of chains in a large batch
        dict(name="commit chain 8", op="commit", dtype="bf16", B=509, nodes=8, chain=1, ctx=333, Hkv=8, D=128,
             page=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "rope", "append", "commit"])
    if op == "rope":
        D = rng.choice([64, 80, 96, 128, 256])
        return dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), T=_log(rng, 1, 8000), H=rng.randint(1, 24), D=D,
                    rot=rng.choice([D, D // 2, 32]), axes=rng.choice([1, 2, 3]), inverse=rng.randint(0, 1),
                    interleaved=rng.randint(0, 1))
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8])
    D, page = rng.choice([64, 128, 256]), rng.choice([8, 16, 32, 64, 128])
    if op == "append":
        return dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), B=rng.randint(1, 32), new=_log(rng, 1, 300),
                    ctx=_log(rng, 1, 2000), Hq=Hkv * G, Hkv=Hkv, D=D, rot=rng.choice([D, D // 4]),
                    axes=rng.choice([1, 3]), page=page)
    nodes = _log(rng, 1, 64)
    chain = int(nodes <= 8 and rng.random() < 0.5)
    if op == "commit":
        return dict(op=op, dtype="bf16", B=_log(rng, 1, 400), nodes=nodes, chain=chain, ctx=_log(rng, 1, 400),
                    Hkv=Hkv, D=D, page=page)
    if rng.random() < 0.2:      # 32-bit inputs run at the sizes of a check
        return dict(op=op, dtype="f32", B=rng.randint(1, 8), nodes=min(nodes, 8), chain=chain,
                    ctx=_log(rng, 1, 1000), ragged=1, shared=0, Hq=Hkv * G, Hkv=Hkv, D=D, page=page)
    ctx = _log(rng, 16, 16000)
    # the key/value elements and the scores of a case stay below those of the largest listed ones
    room = min(120_000_000 // (ctx * Hkv * D), 100_000_000 // (ctx * nodes * Hkv * G))
    B = _log(rng, 1, max(1, min(64, room)))
    shared = 0
    if B > 1 and rng.random() < 0.3:
        shared = int(ctx * rng.uniform(0.2, 0.9)) // page * page
    return dict(op=op, dtype="bf16", B=B, nodes=nodes, chain=chain, ctx=ctx, ragged=int(rng.random() < 0.7),
                shared=shared, Hq=Hkv * G, Hkv=Hkv, D=D, page=page)


# ------------------------------------------------------------------------------------------ inputs

def _sizes(case, seed):
    """Context lengths and nodes (or new tokens) of each sequence, as lists; the latter are the case's own, so
    that outputs have the same shape whatever the seed."""
    r, own_r = np.random.RandomState(seed % (1 << 31)), np.random.RandomState(7)
    B, ctx = case["B"], case["ctx"]
    if case["op"] == "attn" and not case["ragged"]:
        L = np.full(B, ctx)
    else:
        L = r.randint(case.get("shared", 0), ctx + 1, B)
        L[r.randint(B)] = ctx
    most = case["new"] if case["op"] == "append" else case["nodes"]
    if case.get("chain"):
        N = np.full(B, most)
    else:
        N = own_r.randint((most + 1) // 2, most + 1, B)
        N[own_r.randint(B)] = most
    return L.tolist(), N.tolist(), r


def _trees(N, chain, r):
    """Parents and ancestor-or-self masks of one tree for each sequence: chains, or trees of depth below 8."""
    parent, mask = [], []
    for n in N:
        depth, m = [0], [1]
        parent.append(-1)
        for i in range(1, n):
            p = i - 1 if chain else int(r.randint(i))
            while not chain and depth[p] >= 7:
                p = int(r.randint(i))
            parent.append(p)
            depth.append(depth[p] + 1)
            m.append(m[p] | (1 << i))
        mask += m
    return np.array(parent, np.int32), np.array(mask, np.uint64).view(np.int64)


def _cache(case, L, room, r, gen, dtype):
    """A cache whose pages are dealt out in random order; room: slots of each sequence in all."""
    page, shared = case["page"], case.get("shared", 0) // case["page"]
    need = [max(1, -(-n // page)) for n in room]
    n_pages = shared + sum(n - shared for n in need) + 3
    if case["op"] != "attn":            # the cache is an output there: as large as the longest contexts need
        n_pages = len(L) * -(-(case["ctx"] + case.get("new", case.get("nodes", 0))) // page) + 3
    free = r.permutation(n_pages)
    table = np.zeros((len(L), max(need)), np.int32)
    table[:, :shared] = free[:shared]
    at = shared
    for b, n in enumerate(need):
        table[b, shared:n] = free[at:at + n - shared]
        at += n - shared
    shape = (n_pages, page, case["Hkv"], case["D"])
    k, v = (torch.randn(shape, generator=gen, device=DEV, dtype=dtype) for _ in range(2))
    return k, v, torch.from_numpy(table).to(DEV)


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
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dtype, D, op = DTYPES[case["dtype"]], case["D"], case["op"]
    rand = lambda *s: torch.randn(s, generator=gen, device=DEV, dtype=dtype)
    s = dict(case=case, scale=1.0 / math.sqrt(D))
    if op == "rope":
        T, H = case["T"], case["H"]
        s["x"] = rand(T, H, D)
        s["table"], s["positions"], s["pair_axis"] = _rotary(case, T, 4096, gen)
    else:
        L, N, r = _sizes(case, seed)
        B, T, Hkv = case["B"], sum(N), case["Hkv"]
        Hq = case.get("Hq", 0)
        s.update(T=T, B=B, context_len=_int(L), offsets=_int(np.concatenate([[0], np.cumsum(N)])))
        # queries, keys and values of the packed rows come out of one projection, side by side
        qkv = rand(T, (Hq + 2 * Hkv) * D)
        s["q"] = qkv[:, :Hq * D].view(T, Hq, D)
        s["k"] = qkv[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D)
        s["v"] = qkv[:, (Hq + Hkv) * D:].view(T, Hkv, D)
        # which sequence a row belongs to, and where it stands in it
        seq = np.repeat(np.arange(B), N)
        local = np.concatenate([np.arange(n) for n in N])
        s["seq"], s["local"] = torch.from_numpy(seq).to(DEV), torch.from_numpy(local).to(DEV)
        room = L if op == "attn" else [a + b for a, b in zip(L, N)]
        s["kc"], s["vc"], s["page_table"] = _cache(case, L, room, r, gen, dtype)
        if op == "append":
            s["table"], s["positions"], s["pair_axis"] = _rotary(case, T, case["ctx"] + case["new"], gen)
        else:
            parent, mask = _trees(N, case["chain"], r)
            s["parent"], s["mask"] = torch.from_numpy(parent).to(DEV), torch.from_numpy(mask).to(DEV)
        if op == "commit":
            s["accepted"] = _int([int(r.randint(-1, n)) for n in N])
            s["nodes"] = torch.arange(case["nodes"], device=DEV)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that uses the library keeps beside its tensors."""
    from paper_2608_20961_b200 import attention as at, binding as tw
    case = s["case"]
    if "table" in s:
        s["rope"] = at.Rope(s["table"], s["positions"], s["pair_axis"], interleaved=bool(case.get("interleaved", 0)))
    if "kc" in s:
        s["cache"] = at.KVCache(s["kc"], s["vc"], s["page_table"], s["context_len"])
    if "mask" in s:
        s["tree"] = tw.Tree.empty(s["offsets"], s["parent"], 1, case["nodes"])
        s["tree"].anc_mask = s["mask"]
    if case["op"] == "attn":
        s["shared_pages"] = s["page_table"][0, :case["shared"] // case["page"]].contiguous() if case["shared"] else None
        s["workspace"] = at.attn_workspace(s["cache"], s["tree"], case["Hq"], case["shared"])


# -------------------------------------------------------------------------------------- plain forms

def _rotate(x, table, positions, pair_axis, interleaved, inverse):
    """x [T, H, D] in 32 bits, its first rot elements rotated in pairs."""
    half = table.shape[1] // 2
    at = positions.long()[pair_axis.long()].T                      # [T, half]: each pair's position
    pair = torch.arange(half, device=x.device)
    cos, sin = table[at, pair][:, None], table[at, pair + half][:, None]
    if inverse:
        sin = -sin
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def _plain_rope(s):
    c = s["case"]
    return _rotate(s["x"].float(), s["table"], s["positions"], s["pair_axis"], c["interleaved"],
                   c["inverse"]).to(s["x"].dtype)


def _plain_append(s):
    page = s["case"]["page"]
    turn = lambda x: _rotate(x.float(), s["table"], s["positions"], s["pair_axis"], 0, 0).to(x.dtype)
    slot = s["context_len"].long()[s["seq"]] + s["local"]
    at = s["page_table"].long()[s["seq"], slot // page]
    s["kc"][at, slot % page] = turn(s["k"])
    s["vc"][at, slot % page] = s["v"]
    return turn(s["q"]), s["kc"], s["vc"]


def _plain_commit(s):
    page, off, acc = s["case"]["page"], s["offsets"].long()[:-1], s["accepted"].long()
    path = torch.where(acc >= 0, s["mask"][off + acc.clamp(min=0)], 0)
    on = (path[:, None] >> s["nodes"]) & 1                          # [B, nodes]: on the accepted path
    slot = s["context_len"].long()[:, None] + on.cumsum(1) - 1
    b, node = on.nonzero(as_tuple=True)
    slot = slot[b, node]
    at = s["page_table"].long()[b, slot // page]
    s["kc"][at, slot % page] = s["k"][off[b] + node]
    s["vc"][at, slot % page] = s["v"][off[b] + node]
    return s["kc"], s["vc"], s["context_len"] + on.sum(1).to(torch.int32)


def _plain_attn(s):
    c = s["case"]
    B, n, S, Hkv, D, page = s["B"], c["nodes"], c["ctx"], c["Hkv"], c["D"], c["page"]
    G = c["Hq"] // Hkv
    pad = lambda x: x.new_zeros((B, n) + x.shape[1:]).index_put((s["seq"], s["local"]), x)   # packed rows, padded
    q = pad(s["q"].float()).view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    slot = torch.arange(S, device=DEV)
    at = s["page_table"].long()[:, slot // page]                    # [B, S]
    seen = slot < s["context_len"][:, None]                         # [B, S]

    def keys(cache, rows):
        past = torch.where(seen[..., None, None], cache[at, slot % page].float(), 0.0)
        return torch.cat([past, pad(rows.float())], 1).transpose(1, 2)          # [B, Hkv, S + n, D]

    tree = (pad(s["mask"])[..., None] >> torch.arange(n, device=DEV)) & 1       # [B, n, n]
    visible = torch.cat([seen[:, None].expand(B, n, S), tree.bool()], 2)
    score = (q @ keys(s["kc"], s["k"]).transpose(2, 3)) * s["scale"]
    score = score.view(B, Hkv, n, G, S + n).masked_fill_(~visible[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = (score - torch.where(top.isfinite(), top, 0.0)).exp_()      # (rows of padding see nothing)
    total = p.sum(-1, keepdim=True).clamp(min=1e-30)
    out = (p.view(B, Hkv, n * G, S + n) @ keys(s["vc"], s["v"])).view(B, Hkv, n, G, D) / total
    return out.permute(0, 2, 1, 3, 4)[s["seq"], s["local"]].reshape(s["T"], c["Hq"], D).to(s["q"].dtype)


# ------------------------------------------------------------------------------------------- passes

def _own(s):
    from paper_2608_20961_b200 import attention as at
    c = s["case"]
    if c["op"] == "rope":
        y = torch.empty_like(s["x"])
        at.treewy_rope(s["rope"], s["x"], y, inverse=bool(c["inverse"]))
        return y
    if c["op"] == "append":
        q_out = torch.empty((s["T"], c["Hq"], c["D"]), dtype=s["q"].dtype, device=DEV)
        at.treewy_kv_append(s["cache"], s["offsets"], s["k"], s["v"], s["rope"], s["q"], q_out)
        return q_out, s["kc"], s["vc"]
    if c["op"] == "commit":
        new_len = torch.empty_like(s["context_len"])
        at.treewy_kv_commit(s["cache"], s["tree"], s["k"], s["v"], s["accepted"], new_len)
        return s["kc"], s["vc"], new_len
    O = torch.empty((s["T"], c["Hq"], c["D"]), dtype=s["q"].dtype, device=DEV)
    at.treewy_attn_verify(s["cache"], s["tree"], s["q"], s["k"], s["v"], s["scale"], O, s["workspace"],
                          shared_pages=s["shared_pages"], shared_len=c["shared"])
    return O


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "append": _plain_append, "commit": _plain_commit,
            "attn": _plain_attn}[state["case"]["op"]](state)


# -------------------------------------------------------------------------------- work and 64 bits

def work(case):
    e, D = DTYPES[case["dtype"]].itemsize, case["D"]
    if case["op"] == "rope":
        return {"bytes": 2 * case["T"] * case["H"] * D * e + case["axes"] * case["T"] * 4,
                "flops": 3 * case["T"] * case["H"] * case["rot"]}
    L, N, r = _sizes(case, 1)
    T, Hkv = sum(N), case["Hkv"]
    if case["op"] == "append":
        heads = case["Hq"] + Hkv
        return {"bytes": 2 * T * (heads + Hkv) * D * e + case["axes"] * T * 4, "flops": 3 * T * heads * case["rot"]}
    if case["op"] == "commit":          # half of the nodes' depth is a fair path; its rows, in and out, k and v
        rows = sum(min(n, 8) / 2 for n in N)
        return {"bytes": 4 * rows * Hkv * D * e + T * 8, "flops": 0}
    shared = case["shared"]
    keys = shared + sum(n - shared for n in L)
    seen = sum(l * n + n for l, n in zip(L, N))
    return {"bytes": 2 * keys * Hkv * D * e + T * (2 * case["Hq"] + 2 * Hkv) * D * e + T * 8,
            "flops": 4 * D * case["Hq"] * seen}


def exact(case, seed):
    """Sequence by sequence and pair by pair in 64 bits, from the definitions."""
    s = prepare(case, seed)
    f64 = lambda x: x.to(torch.float64)
    if case["op"] in ("rope", "append"):
        half = case["rot"] // 2
        wave = f64(s["table"])

        def turn(x, sign, step):
            y = f64(x).clone()
            for p in range(half):
                i, j = (2 * p, 2 * p + 1) if step else (p, p + half)
                row = wave[s["positions"][int(s["pair_axis"][p])].long()]
                z = torch.complex(f64(x[..., i]), f64(x[..., j])) * torch.complex(row[:, p], sign * row[:, p + half])[:, None]
                y[..., i], y[..., j] = z.real, z.imag
            return y
        if case["op"] == "rope":
            return turn(s["x"], -1.0 if case["inverse"] else 1.0, case["interleaved"])
    off, L = s["offsets"].tolist(), s["context_len"].tolist()
    table, page = s["page_table"].tolist(), case["page"]
    if case["op"] in ("append", "commit"):
        kc, vc = f64(s["kc"]), f64(s["vc"])
        k = turn(s["k"], 1.0, 0) if case["op"] == "append" else f64(s["k"])
        v, lens = f64(s["v"]), list(L)
        for b in range(case["B"]):
            rows = range(off[b], off[b + 1])
            if case["op"] == "commit":
                a, rows = int(s["accepted"][b]), []
                while a >= 0:
                    rows.insert(0, off[b] + a)
                    a = int(s["parent"][off[b] + a])
            n, at = len(rows), L[b]
            lens[b] += n
            slots = range(at, at + n)
            pages, places = [table[b][x // page] for x in slots], [x % page for x in slots]
            kc[pages, places], vc[pages, places] = k[list(rows)], v[list(rows)]
        return (turn(s["q"], 1.0, 0), kc, vc) if case["op"] == "append" else (kc, vc, lens_tensor(lens))
    G, out = case["Hq"] // case["Hkv"], torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    parent = s["parent"].tolist()
    for b in range(case["B"]):
        lo, n = off[b], off[b + 1] - off[b]
        sees = torch.eye(n, dtype=torch.bool, device=DEV)
        for i in range(n):
            if parent[lo + i] >= 0:
                sees[i] |= sees[parent[lo + i]]
        pages = torch.tensor(table[b][:-(-L[b] // page)], device=DEV, dtype=torch.long)
        for h in range(case["Hq"]):
            g = h // G
            past = lambda c: f64(c[pages, :, g].reshape(-1, case["D"])[:L[b]])
            q, keys, values = f64(s["q"][lo:lo + n, h]), f64(s["k"][lo:lo + n, g]), f64(s["v"][lo:lo + n, g])
            new = torch.exp((q @ keys.T * s["scale"]).clamp(max=600.0)) * sees
            old = torch.exp((q @ past(s["kc"]).T * s["scale"]).clamp(max=600.0))
            out[lo:lo + n, h] = (old @ past(s["vc"]) + new @ values) / (old.sum(1) + new.sum(1))[:, None]
    return out


def lens_tensor(lens):
    return torch.tensor(lens, dtype=torch.int32, device=DEV)
