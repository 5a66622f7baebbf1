"""Plain form of a step's tables: requests one after another, lists and loops.

``update`` changes a state of lists in place and returns the step's tables:
block tables, free blocks as a stack, row offsets, positions, slots, and for
every row the drafts of its request that it descends from."""

from __future__ import annotations

BLOCK = 16
OK, NO_BLOCKS, INVALID = 0, 1, 2


class State:
    """``table[r]``: the blocks that request r holds, in order; ``free``: the stack,
    its top last."""

    def __init__(self, table, free):
        self.table = [list(t) for t in table]
        self.free = list(free)


def update(s: State, ctx_len, q_len, parents, max_rows, max_blocks, max_draft):
    n = len(ctx_len)
    q_start, at, refused = [], 0, [None] * n
    for r in range(n):
        q_start.append(min(at, max_rows))
        rows = max(q_len[r], 0)
        need = -(-(ctx_len[r] + q_len[r]) // BLOCK)
        if ctx_len[r] < 0 or q_len[r] < 0 or need > max_blocks or (max_draft and q_len[r] > max_draft) or \
                q_start[r] + rows > max_rows:
            refused[r] = INVALID
        at += rows
    q_start.append(min(at, max_rows))
    need = [0 if refused[r] else -(-(ctx_len[r] + q_len[r]) // BLOCK) for r in range(n)]
    # back first, so that the first to come back is on top
    back = []
    for r in range(n):
        if not refused[r]:
            back += s.table[r][need[r]:]
            del s.table[r][need[r]:]
    s.free += reversed(back)
    asked, avail = 0, len(s.free)
    for r in range(n):
        if refused[r] or need[r] == len(s.table[r]):
            continue
        asked += need[r] - len(s.table[r])
        if asked > avail:
            refused[r] = NO_BLOCKS
            continue
        while len(s.table[r]) < need[r]:
            s.table[r].append(s.free.pop())
    state = [r or OK for r in refused]
    kv_len = [0 if refused[r] else ctx_len[r] + q_len[r] for r in range(n)]
    positions, slots, seen = [], [], []
    for r in range(n):
        masks = []
        for i in range(q_start[r + 1] - q_start[r]):
            if refused[r]:
                positions.append(0)
                slots.append(-1)
                seen.append(0)
                continue
            token = ctx_len[r] + i
            slots.append(s.table[r][token // BLOCK] * BLOCK + token % BLOCK)
            if not max_draft:
                positions.append(token)
                continue
            p = i - 1 if parents is None else parents[q_start[r] + i]
            masks.append((1 << i) | (masks[p] if 0 <= p < i else 0))
            seen.append(masks[-1])
            positions.append(ctx_len[r] + bin(masks[-1]).count("1") - 1)
    return dict(q_start=q_start, kv_len=kv_len, state=state, positions=positions, slots=slots, seen=seen)
