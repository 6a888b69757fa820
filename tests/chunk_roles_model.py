"""A model of the roles of the tensor-core kernel of treewy_attn_chunk and of what they hand to each other: every role is the
list of its waits, arrivals and accesses.

Accesses name a region and the version (item or tile) that they mean; a write must not meet a reader that is still at it, a
reader must find its version.  A wait names a phase by its parity, as the hardware does, and the model knows which one is meant.
Everything a role does is fixed, so an order that goes wrong is one in which some role stands still while others run: each
role is held at each of its steps in turn, and the others run as far as they come, in several orders of preference."""
from __future__ import annotations

import random
from dataclasses import dataclass

ITEMS = 8
WARPS = 2                      # of a stream (the kernel has four; two are enough to be at odds)
# heads of d: streams, S buffers of a stream, K stages, V stages
CONFIG = {64: (2, 2, 10, 10), 128: (2, 2, 5, 5), 256: (1, 4, 3, 2)}


@dataclass
class Rule:
    """The hand-over of outputs.  arrivals: of a warp of stream s on o_free[which] at the end of an item, used: whether the item has
    used that output; needed: what completes a phase; by_use: a phase is a use of an output (else an item, and a stream without a
    tile waits for the barriers of `waits`)."""
    arrivals: object           # (pair, s, which, used) -> number
    needed: int
    by_use: bool = True
    waits: tuple = ()


def programs(d, items, rule, masked=True, rescale=False, flags=None):
    """Role -> list of steps, a step being a list of operations that nobody sees the middle of.  items: (pair, tiles of each stream).
    masked: values are cleaned in every tile; rescale: every tile moves the reference (outputs at rest are read and written); flags:
    what cleaning has met is read "early", ahead of the wait for the other stream's outputs, or "late", behind it."""
    STREAMS, NB, NK, NV = CONFIG[d]
    ends = len(items)
    tiles = [max((t[-1] for t in it[1] if t), default=-1) + 1 if it[0] else sum(len(t) for t in it[1]) for it in items]
    first = [sum(tiles[:i]) for i in range(ends + 1)]
    wait = lambda name, i, phase: ("wait", (name, i), phase)
    arrive = lambda name, i: ("arrive", (name, i))
    ring = lambda name, g, n: wait(name, g % n, g // n)
    item_full = lambda i: wait("item_full", i % ITEMS, i // ITEMS)

    def softmax(s, w):
        out, count, singles = [], 0, 0
        for i, (pair, on) in enumerate(items):
            out += [[item_full(i)], [("begin", ("items", i % ITEMS), i)]]
            both = STREAMS == 2 and not pair
            before = count
            for j in on[s]:
                buf, g = s * NB + count % NB, first[i] + j
                out += [[wait("s_full", buf, count // NB)], [("begin", ("s", buf), (s, count))]]
                if rescale and count > before:
                    out += [[wait("pv_done", s * NB + (count - 1) % NB, (count - 1) // NB)], [("begin", ("o", s), i)], [("end", ("o", s), i)]]
                if masked:
                    if NV < NB and count >= NV:
                        out.append([wait("pv_done", s * NB + (count - NV) % NB, (count - NV) // NB)])
                    out += [[ring("v_full", g, NV)], [("begin", ("v", g % NV), g)], [("mark", ("met", i, s, w)), ("end", ("v", g % NV), g)]]
                out.append([("end", ("s", buf), (s, count)), arrive("p_full", buf)])
                count += 1
            if count > before:
                out.append([wait("pv_done", s * NB + (count - 1) % NB, (count - 1) // NB)])
            elif i > 0:
                out += [[wait("o_free", b, i - 1)] for b in rule.waits]
            writes = STREAMS == 1 or pair or s == 0
            met = [("have", ("met", i, t, x)) for t in range(STREAMS) for x in range(WARPS) if masked and on[t] and (not pair or t == s)]
            if writes and flags == "early":
                out.append(met)
            if both and (on[1] or not rule.by_use):
                if s == 1:
                    out.append([("write", ("ml", w), i), arrive("ml_full", w)])
                else:
                    out.append([wait("ml_full", w, singles)])
                    if on[1]:
                        out += [[("begin", ("ml", w), i)], [("end", ("ml", w), i)]]
                singles += 1
            if writes:
                if flags == "late":
                    out.append(met)
                for t in range(STREAMS):
                    if on[t] and (t == s or both):
                        out += [[("begin", ("o", t), i)], [("end", ("o", t), i)]]
            out.append([arrive("o_free", b) for b in range(STREAMS) for _ in range(rule.arrivals(pair or STREAMS == 1, s, b, bool(on[b])))])
            out.append([("end", ("items", i % ITEMS), i), arrive("item_empty", i % ITEMS)])
        return out + [[item_full(ends)]]

    def mma(me):
        """The thread's steps and, in another role, the completions of what it has issued, in order."""
        strm = me if STREAMS == 2 else 0
        out, late, k, v, made, used, uses = [], [], 0, 0, 0, 0, 0

        def issue(ops, done):
            out.extend([ops] if ops else [])
            late.append([("after", len(out))] + done)
        for i, (pair, on) in enumerate(items):
            pair = STREAMS == 2 and pair
            n, ahead = tiles[i], NB if pair or STREAMS == 1 else 2 * NB
            does_qk, does_pv = STREAMS == 2 or me == 0, STREAMS == 2 or me == 1
            out += [[item_full(i)], [("begin", ("items", i % ITEMS), i)], [("end", ("items", i % ITEMS), i), arrive("item_empty", i % ITEMS)]]
            if does_qk:
                out.append([wait("q_full", 0, i)])
            onto, asked = False, False
            for t in range(n + ahead):
                j = t - ahead
                if does_pv and j == 0 and i > 0 and not rule.by_use:
                    out.append([wait("o_free", strm, i - 1)])
                if does_pv and j >= 0:
                    if rule.by_use and j in on[strm] and not onto:
                        out += [[wait("o_free", strm, uses - 1)]] if uses else []
                        uses += 1
                    out.append([ring("v_full", v, NV)])
                    if j in on[strm]:
                        buf = strm * NB + used % NB
                        out.append([wait("p_full", buf, used // NB)])
                        issue([("begin", ("v", v % NV), v)] + ([] if onto else [("write", ("o", strm), i)]) + [("begin", ("p", buf), used)],
                              [("end", ("v", v % NV), v), ("end", ("p", buf), used), arrive("pv_done", buf), arrive("v_free", v % NV)])
                        used, onto = used + 1, True
                    else:
                        out.append([arrive("v_free", v % NV)])
                    v += 1
                if does_qk and t < n:
                    if t in on[strm]:
                        buf = strm * NB + made % NB
                        if STREAMS == 1 and made >= NB:
                            out.append([wait("pv_done", buf, made // NB - 1)])
                        out.append([ring("k_full", k, NK)])
                        # (the S buffer: its last product is done, or in this same thread's queue ahead of this)
                        issue([("begin", ("k", k % NK), k), ("queued" if STREAMS == 2 else "write", ("s", buf), (strm, made))] +
                              ([] if asked else [("begin", ("q", 0), i)]),
                              [("end", ("k", k % NK), k), arrive("s_full", buf), arrive("k_free", k % NK)])
                        made, asked = made + 1, True
                    else:
                        out.append([ring("k_full", k, NK), arrive("k_free", k % NK)])
                    k += 1
                    if t + 1 == n:
                        issue([], ([("end", ("q", 0), i)] if asked else []) + [arrive("q_free", 0)])
        return [out + [[item_full(ends)]], late]

    def producer(is_v):
        ns, name, out, late = (NV, "v", [], []) if is_v else (NK, "k", [], [])

        def issue(ops, done):
            out.append(ops)
            late.append([("after", len(out))] + done)

        def find(i):
            if i >= ITEMS:
                out.append([wait("item_empty", i % ITEMS, i // ITEMS - 1)])
            out.append([("write", ("items", i % ITEMS), i), arrive("item_full", i % ITEMS)])
        if is_v:
            find(0)
        for i in range(ends):
            if is_v:
                find(i + 1)
            else:
                out += [[item_full(i)], [("begin", ("items", i % ITEMS), i)], [("end", ("items", i % ITEMS), i), arrive("item_empty", i % ITEMS)]]
                if i > 0:
                    out.append([wait("q_free", 0, i - 1)])
                issue([("write", ("q", 0), i)], [arrive("q_full", 0)])
            for g in range(first[i], first[i + 1]):
                if g >= ns:
                    out.append([wait(name + "_free", g % ns, g // ns - 1)])
                issue([("write", (name, g % ns), g)], [arrive(name + "_full", g % ns)])
        return [out if is_v else out + [[item_full(ends)]], late]

    progs = [softmax(s, w) for s in range(STREAMS) for w in range(WARPS)]
    owners = list(range(len(progs)))
    for pair_of in (mma(0), mma(1), producer(False), producer(True)):
        at = len(progs)
        progs += pair_of
        owners += [at, at]
    count = {"k_free": STREAMS, "v_free": STREAMS, "q_free": STREAMS if STREAMS == 2 else 1, "p_full": WARPS, "o_free": rule.needed,
             "item_empty": WARPS * STREAMS + 3}
    return [[s for s in p if s] for p in progs], owners, count


class Walk:
    def __init__(self, progs, owners, count):
        self.progs, self.owners, self.count = progs, owners, count
        self.pc, self.arrived, self.marks = [0] * len(progs), {}, set()
        self.version, self.inside = {}, {}

    def runs(self, r):
        """Whether role r can take its next step; an error's text if a wait is misled."""
        if self.pc[r] == len(self.progs[r]):
            return False
        for op in self.progs[r][self.pc[r]]:
            if op[0] == "after" and self.pc[self.owners[r]] < op[1]:
                return False
            if op[0] == "wait":
                done = self.arrived.get(op[1], 0) // self.count.get(op[1][0], 1)
                if done > op[2] + 1:
                    return f"phase {op[2]} of {op[1]} has been overtaken"
                if (done & 1) == (op[2] & 1):          # (the phase of that parity is not complete, as far as the hardware tells)
                    return False
                if done <= op[2]:
                    return f"the wait for phase {op[2]} of {op[1]} passes after {done}"
        return True

    def step(self, r):
        ops = self.progs[r][self.pc[r]]
        self.pc[r] += 1
        for op in ops:
            kind, what = op[0], op[1]
            if kind == "arrive":
                self.arrived[what] = self.arrived.get(what, 0) + 1
            elif kind == "mark":
                self.marks.add(what)
            elif kind == "have" and what not in self.marks:
                return f"{what} is looked for before it is known"
            elif kind in ("write", "queued"):
                if self.inside.get(what) and kind == "write":
                    return f"{what} is overwritten for {op[2]} while {self.inside[what]} is read"
                self.version[what] = op[2]
            elif kind == "begin" and what[0] != "p":
                if self.version.get(what) != op[2]:
                    return f"{what} holds {self.version.get(what)}, not {op[2]}"
                self.inside.setdefault(what, []).append(op[2])
            elif kind == "end" and what[0] != "p":
                self.inside[what].remove(op[2])
        return None

    def run(self, order, hold=None):
        """Until nothing moves but what is held.  order: of preference (a function of the roles that can move)."""
        can, look = set(), range(len(self.progs))
        while True:
            for r in look:                           # (whose next step may have become one, or none, by the last one)
                ok = not (hold and r == hold[0] and self.pc[r] >= hold[1]) and self.runs(r)
                if isinstance(ok, str):
                    return f"role {r}: {ok}"
                (can.add if ok else can.discard)(r)
            if not can:
                return None
            moved = order(sorted(can))
            step = self.progs[moved][self.pc[moved]]
            wrong = self.step(moved)
            if wrong:
                return f"role {moved}: {wrong}"
            told = {op[1] for op in step if op[0] == "arrive"}
            look = [r for r, p in enumerate(self.progs) if r == moved or self.owners[r] == moved or
                    (self.pc[r] < len(p) and any(op[0] == "wait" and op[1] in told for op in p[self.pc[r]]))]

    def stuck(self):
        """The steps that the roles which have not come to their end stand at."""
        return [(r, s[p]) for r, (p, s) in enumerate(zip(self.pc, self.progs)) if p < len(s)]


def find(d, items, rule, orders=40, seed=0, **kw):
    """What goes wrong in some order, or None.  (Of long runs of items not every step is held: they repeat.)"""
    progs, owners, count = programs(d, items, rule, **kw)
    rng = random.Random(seed)
    holds = [(r, k) for r in range(len(progs)) for k in range(len(progs[r]))]
    holds = rng.sample(holds, min(len(holds), 150))
    for hold in [None] + holds:
        walk = Walk(progs, owners, count)
        wrong = walk.run(lambda can: can[0], hold)
        if wrong:
            return wrong
        if hold:                                     # and on, when the one that was held goes again
            wrong = walk.run(lambda can: can[-1])
            if wrong:
                return wrong
        if walk.stuck():
            return f"stuck at {walk.stuck()}"
    for _ in range(orders):                          # any order, the roles at uneven speeds
        speed = [rng.random() ** 3 + 1e-3 for _ in progs]
        walk = Walk(progs, owners, count)
        wrong = walk.run(lambda can: rng.choices(can, [speed[r] for r in can])[0])
        if wrong or walk.stuck():
            return wrong or f"stuck at {walk.stuck()}"
    return None


def pair(*tiles):
    """An item of two row tiles; tiles: which key tiles each stream takes."""
    return (True, [list(t) for t in tiles])


def single(d, n):
    """An item of one row tile: the streams take its key tiles in turn."""
    return (False, [list(range(n))]) if CONFIG[d][0] == 1 else (False, [list(range(0, n, 2)), list(range(1, n, 2))])
