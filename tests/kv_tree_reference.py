"""Drafted tokens over the paged 4-bit cache from the definitions (include/ivfpq_kv.h), in numpy and 64 bits, token by token.
Nothing here uses the library."""
import numpy as np

from kv_reference import PAGE


def ancestors(parents, i):
    """Token i of a request, its parent, and so on; parents that are no earlier token are none."""
    path = [i]
    while 0 <= parents[path[-1]] < path[-1]:
        path.append(int(parents[path[-1]]))
    return path


def tree(parents, step, max_nodes, window=0):
    """(sees [T][max_nodes] bool, positions [T])."""
    T = len(step["positions"])
    sees, positions = np.zeros((T, max_nodes), bool), np.full(T, -1, np.int64)
    for a, b in zip(step["q_start"], step["q_start"][1:]):
        for i in range(min(b - a, max_nodes)):
            path = ancestors(parents[a:b], i)
            sees[a + i, path[:window or None]] = True
            positions[a + i] = step["positions"][a] + len(path) - 1
    return sees, positions


def words(sees):
    """Bits of rows [T][n] as int64 words."""
    n = -(-sees.shape[1] // 64) * 64
    bits = np.zeros((sees.shape[0], n), bool)
    bits[:, :sees.shape[1]] = sees
    return (bits.reshape(len(sees), -1, 64).astype(np.uint64) << np.arange(64, dtype=np.uint64)).sum(-1, dtype=np.uint64).view(np.int64)


def attention(cache, q, H, step, sees, positions, n_pages, scale, window=0):
    """As kv_reference.attention: (out, lse, mass, reach, size)."""
    T, Hq, D = q.shape
    out, mass, reach = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, size = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    for a, b in zip(step["q_start"], step["q_start"][1:]):
        for t in range(a, b):
            r, past = step["requests"][t], step["positions"][a]
            held = step["kv_lens"][r]
            here = min(max(positions[t], past), past + (b - a) - 1)
            j = np.arange(max(0, here - window + 1) if window else 0, min(past, held))
            new = past + np.nonzero(sees[t])[0]
            j = np.concatenate((j, new[new < min(held, past + (b - a))])).astype(np.int64)
            pages = step["table"][r, j // PAGE]
            there = (pages >= 0) & (pages < n_pages)
            at = pages[there].astype(np.int64) * PAGE + j[there] % PAGE
            if len(at) == 0:
                continue
            for h in range(Hq):
                hk = h // (Hq // H)
                if cache.bad[at, hk].any():
                    out[t, h], lse[t, h] = np.nan, np.nan
                    continue
                k, v = cache.k[at, hk], cache.v[at, hk]
                s = k @ q[t, h] * scale
                top = s.max()
                p = np.exp(s - top)
                lse[t, h] = top + np.log(p.sum())
                p /= p.sum()
                out[t, h], mass[t, h], reach[t, h] = p @ v, p @ np.abs(v), np.abs(v).sum(0)
                size[t, h] = (np.abs(k) @ np.abs(q[t, h])).max() * abs(scale)
    return out, lse, mass, reach, size


def path_of(sees, drafted, picked, stored):
    """Tokens that stay of one request: sees [n][n], the rest [n]."""
    best = []
    for i in range(len(sees)):
        path = np.nonzero(sees[i])[0]
        if len(path) <= len(best):
            continue
        good = True
        for p in path:
            below = np.nonzero(sees[p][:p])[0]
            good = good and (p == 0 or (stored[p] and len(below) > 0 and drafted[p] == picked[below[-1]]))
        if good:
            best = path.tolist()
    return best


def keep(caches, step, sees, drafted, picked, ring, state, n_pages):
    """Moves held values and makes boxes again in `caches`; returns (lens, rows, ring, state)."""
    R, T, W = len(step["kv_lens"]), len(step["positions"]), step["table"].shape[1]
    ring, lens, rows = ring.copy(), np.array(step["kv_lens"]), np.full(T, -1, np.int64)
    head, tail, missing = state
    avail = min(max(tail - head, 0), len(ring))
    given = 0
    for r in range(R):
        a, b = step["q_start"][r], step["q_start"][r + 1]
        if b == a:
            continue
        n, past, held = b - a, step["positions"][a], step["kv_lens"][r]
        slots = step["slots"][a:b]
        full = np.zeros((n, n), bool)
        full[:, :min(n, sees.shape[1])] = sees[a:b, :n]
        path = path_of(full, drafted[a:b], picked[a:b], (slots >= 0) & (slots < n_pages * PAGE))
        lens[r] = min(past + len(path), held)
        rows[a:a + len(path)] = a + np.array(path, np.int64)
        for c in caches:
            for i, p in enumerate(path):
                if 0 <= slots[p] < n_pages * PAGE and 0 <= slots[i] < n_pages * PAGE:
                    c.k[slots[i]], c.v[slots[i]], c.bad[slots[i]] = c.k[slots[p]], c.v[slots[p]], c.bad[slots[p]]
            for col in range(past // PAGE, min(-(-lens[r] // PAGE), W)):
                page = step["table"][r, col]
                if 0 <= page < n_pages:
                    k = c.k[page * PAGE:page * PAGE + min(PAGE, lens[r] - col * PAGE)]
                    c.boxes[page, :, 0], c.boxes[page, :, 1] = k.min(0), k.max(0)
        for col in range(-(-lens[r] // PAGE), min(-(-held // PAGE), W)):
            if 0 <= step["table"][r, col] < n_pages:
                if given < len(ring) - avail:
                    ring[(tail + given) % len(ring)] = step["table"][r, col]
                given += 1
    return lens, rows, ring, np.array([head, tail + min(given, len(ring) - avail), missing], np.int64)


def rotate(x, positions, frequencies, axes, neighbours):
    """x [T][heads][D] turned by positions [axes][T], in 64 bits: (result, |a| + |b| of each channel's pair)."""
    y, size = np.array(x, np.float64), np.zeros(x.shape)
    n = len(frequencies)
    for i, f in enumerate(frequencies):
        one, two = (2 * i, 2 * i + 1) if neighbours else (i, i + n)
        p = positions[axes[i]].astype(np.int64)
        # in extended precision: an angle of 2^31 is off by 2^-33 at most
        turn = np.fmod(np.longdouble(p) * np.longdouble(f), _TWO_PI).astype(np.float64)[:, None]
        a, b = y[..., one].copy(), y[..., two].copy()
        y[..., one], y[..., two] = a * np.cos(turn) - b * np.sin(turn), b * np.cos(turn) + a * np.sin(turn)
        size[..., one] = size[..., two] = np.abs(a) + np.abs(b)
    return y, size


# 2 pi in the 64 bits of an extended number
_TWO_PI = 2 * (np.longdouble(3.141592653589793115997963468544185161591) + np.longdouble(1.2246467991473531772e-16))
