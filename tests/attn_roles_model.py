"""A model of the roles of the tensor-core attention kernel and of the barriers between them: every role is the list of
its waits and arrivals, and every order in which they can run is walked.

A wait names a phase by its parity, as the hardware does, and the model also knows which phase is meant.  It reports a
wait that can pass before that phase is complete and one that can meet the phase after it (where the parity reads
"not yet" for good)."""
from __future__ import annotations

ITEMS = 8
# heads of d: K stages, V stages, S buffers, weights through shared memory
CONFIG = {64: (8, 8, 4, False), 128: (8, 4, 4, False), 256: (3, 2, 2, True)}


def programs(d, items, q_phase, q_buffers, rescale):
    """Role -> list of steps; ("wait", barrier, phase, parity), ("arrive", barrier), ("tag", tile), ("say", tile), and
    ("done", barrier): a copy or a product that arrives some time after it was issued, in the order of issue.
    items: key tiles of each item.  rescale: every tile moves the running maximum (a wait more), or none does."""
    NK, NV, NSB, P_SMEM = CONFIG[d]
    wait = lambda name, i, n: ("wait", (name, i % n), i // n, (i // n) & 1)
    arrive = lambda name, i, n: ("arrive", (name, i % n))
    done = lambda name, i, n: ("done", (name, i % n))

    def q(kind, item):
        barrier, parity = q_phase(item, q_buffers)
        return ("wait", ("q", barrier), item // q_buffers, parity) if kind == "wait" else ("arrive", ("q", barrier))

    def softmax(w):
        out = []

        def take(i):
            out.append(wait("item_full", i, ITEMS))
            if i < len(items):
                out.append(q("arrive", i))
        take(0)
        tile = 0
        for i, n in enumerate(items):
            last, j, taken = tile + n - 1, 0 if (tile & 1) == w else 1, False
            while True:
                g = tile + j
                if j >= n and (last & 1) != w:
                    out.append(("tag", last))
                if not taken and (j >= n or (q_tm[d] == 2 and j + 2 >= n)):
                    take(i + 1)
                    taken = True
                if j >= n:
                    break
                if g > 0:
                    out.append(("tag", g - 1))
                out.append(wait("s_full", g, NK))
                if P_SMEM:
                    out.append(arrive("s_free", g, NSB))
                out.append(("say", g))
                if P_SMEM and g >= 2:
                    out.append(wait("pv_done", g - NV, NV))
                if j == n - 1:
                    out.append(wait("v_full", g, NV))
                if j > 0 and rescale:
                    out.append(wait("pv_done", g - 1, NV))
                out.append(arrive("p_full", g, NSB))
                j += 2
            out.append(arrive("exch", i, 1))
            out.append(wait("exch", i, 1))
            if P_SMEM and last > 0:
                out.append(wait("pv_done", last - 1, NV))
            out.append(wait("pv_done", last, NV))
            out.append(arrive("o_free", i, 1))
            out.append(arrive("item_empty", i, ITEMS))
            tile += n
        return out

    def mma_qk():
        out, g = [], 0
        for i, n in enumerate(items):
            out += [wait("item_full", i, ITEMS), arrive("item_empty", i, ITEMS), q("wait", i)]
            for _ in range(n):
                if g >= NSB:
                    out.append(wait("s_free", g - NSB, NSB) if P_SMEM else wait("pv_done", g - NSB, NV))
                out += [wait("k_full", g, NK), done("s_full", g, NK)]
                g += 1
        return out + [wait("item_full", len(items), ITEMS)]

    def mma_pv():
        out, g = [], 0
        for i, n in enumerate(items):
            out += [wait("item_full", i, ITEMS), arrive("item_empty", i, ITEMS)]
            for j in range(n):
                out.append(wait("v_full", g, NV))
                if j == 0 and i > 0:
                    out.append(wait("o_free", i - 1, 1))
                out += [wait("p_full", g, NSB), done("pv_done", g, NV)]
                g += 1
        return out + [wait("item_full", len(items), ITEMS)]

    def producer(is_v):
        ns, empty, full = (NV, "pv_done", "v_full") if is_v else (NK, "s_full", "k_full")
        out, g = [], 0
        for i, n in enumerate(items + [0]):
            if is_v:
                out.append(wait("item_full", i, ITEMS))
                if n:
                    out.append(arrive("item_empty", i, ITEMS))
            else:
                if i >= ITEMS:
                    out.append(wait("item_empty", i - ITEMS, ITEMS))
                out.append(arrive("item_full", i, ITEMS))
            for _ in range(n):
                if g >= ns:
                    out.append(wait(empty, g - ns, ns))
                out.append(done(full, g, ns))
                g += 1
        return out

    return [softmax(0), softmax(1), mma_qk(), mma_pv(), producer(False), producer(True)]


q_tm = {64: 2, 128: 2, 256: 1}                       # Q buffers in tensor memory
COUNT = {"q": 2, "exch": 2, "o_free": 2, "item_empty": 5}   # arrivals that complete a phase (a softmax group counts once)


def walk(progs, limit=2_000_000):
    """None when every order ends and no wait can be misled, else what goes wrong first."""
    # a step: a wait with the arrivals behind it (nobody sees the difference before the next wait)
    steps = []
    for p in progs:
        mine, cur = [], []
        for op in p:
            if op[0] in ("wait", "tag") and cur:
                mine.append(cur)
                cur = []
            cur.append(op)
        steps.append(mine + [cur])
    # what a role has issued completes in a role of its own
    for r in range(len(steps)):
        late = [[("after", r, i + 1), ("arrive", op[1])] for i, step in enumerate(steps[r]) for op in step if op[0] == "done"]
        if late:
            steps.append(late)
    arrivals, said = [], []                          # of each role, by the number of its steps that are done
    for s in steps:
        a, t, last = [{}], [-1], -1
        for step in s:
            d = dict(a[-1])
            for op in step:
                if op[0] == "arrive":
                    d[op[1]] = d.get(op[1], 0) + 1
                elif op[0] == "say":
                    last = op[1]
            a.append(d)
            t.append(last)
        arrivals.append(a)
        said.append(t)
    start, end = (0,) * len(steps), tuple(len(s) for s in steps)
    seen, todo = {start}, [start]
    while todo:
        pcs = todo.pop()
        moved = False
        for r, pc in enumerate(pcs):
            if pc == end[r]:
                continue
            op = steps[r][pc][0]
            if op[0] == "wait":
                done = sum(a[x].get(op[1], 0) for a, x in zip(arrivals, pcs)) // COUNT.get(op[1][0], 1)
                passes = (done & 1) != op[3]
                if passes and done <= op[2]:
                    return f"role {r}: the wait for phase {op[2]} of {op[1]} passes after {done}"
                if done > op[2] + 1:
                    return f"role {r}: phase {op[2]} of {op[1]} has been overtaken ({done} are complete)"
                if not passes:
                    continue
            elif op[0] == "after":
                if pcs[op[1]] < op[2]:
                    continue
            elif op[0] == "tag":
                tag = max(t[x] for t, x in zip(said, pcs))
                if tag > op[1]:
                    return f"role {r}: the maximum of tile {op[1]} is gone"
                if tag < op[1]:
                    continue
            moved = True
            nxt = pcs[:r] + (pc + 1,) + pcs[r + 1:]
            if nxt not in seen:
                seen.add(nxt)
                todo.append(nxt)
        if not moved and pcs != end:
            return f"stuck at {pcs}"
        assert len(seen) < limit
    return None
