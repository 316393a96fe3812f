"""Page tables of a step when pages run out (include/ivfpq_kv.h, ivfpq_kv_plan), request by request in numpy: the ring
holds pages only, so what an ended request never got is not put back.  Nothing here uses the library."""
import numpy as np

PAGE = 64


def plan(past, new, table, ring, state, max_tokens):
    """Arguments and result as `kv_reference.plan`'s."""
    table, ring = table.copy(), ring.copy()
    W, cap, (head, tail, _) = table.shape[1], len(ring), state
    avail = min(max(tail - head, 0), cap)
    old, left, back, missing, t = ring.copy(), avail, 0, 0, 0
    kv, start = [], [0]
    slots, reqs, poss = (np.full(max_tokens, -1, np.int64) for _ in range(3))
    for r, (p, n) in enumerate(zip(past, new)):
        p = min(max(p, 0), W * PAGE)
        held = -(-p // PAGE)
        if n < 0:
            for page in table[r, :held]:
                if page >= 0 and back < cap - avail:  # never onto a page that waits in the ring
                    ring[(tail + back) % cap] = page
                    back += 1
        total = min(p + max(n, 0), W * PAGE)
        if n >= 0:
            for c in range(held, -(-total // PAGE)):
                if left > 0:
                    table[r, c] = old[(head + avail - left) % cap]
                    left -= 1
                else:
                    table[r, c] = -1
                    missing += 1
        kv.append(total if n >= 0 else 0)
        for j in range(p, p + max(n, 0)):
            if t < max_tokens:
                page = table[r, j // PAGE] if j < W * PAGE else -1
                slots[t] = page * PAGE + j % PAGE if page >= 0 else -1
                reqs[t], poss[t] = r, j
            t += 1
        start.append(min(t, max_tokens))
    return dict(kv_lens=np.array(kv, np.int64), q_start=np.array(start, np.int64), table=table, ring=ring, slots=slots,
                requests=reqs, positions=poss, state=np.array([head + avail - left, tail + back, missing], np.int64))


def pages_of(lens, table, ring, state):
    """(pages in the tables, pages in the ring) after a step."""
    held = [int(p) for row, n in zip(table, lens) for p in row[:-(-int(n) // PAGE)] if p >= 0]
    return held, [int(ring[i % len(ring)]) for i in range(int(state[0]), int(state[1]))]


def check(lens, table, ring, state, n_pages):
    """Every page is in one table or in the ring, once."""
    held, free = pages_of(lens, table, ring, state)
    assert sorted(held + free) == list(range(n_pages)), (held, free)
