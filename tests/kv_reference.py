"""The paged 4-bit cache from its definitions (include/ivfpq_kv.h), in numpy and 64 bits, token by token:
what the tests compare the kernels with.  Nothing here uses the library."""
import numpy as np

PAGE = 64
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """(codes [..., D] 0..15, scale bytes [..., D/32], held values) of finite rows."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(g).max(-1)
    exponent = np.frexp(np.where(top > 0, top, 1.0))[1] - 1          # floor(log2(top))
    b = np.where(top > 0, np.clip(exponent + 127 - 2, 1, 254), 1).astype(np.int64)
    unit = np.ldexp(1.0, b - 127)[..., None]
    far = np.abs(np.abs(g)[..., None] / unit[..., None] - GRID)
    # nearest; of two equally near the even code
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[np.argmin(far[..., order], -1)]
    value = np.copysign(GRID[code], g) * unit
    return (code + 8 * np.signbit(g)).reshape(x.shape), b.astype(np.uint8), value.reshape(x.shape)


class Cache:
    """Held values [n_pages * 64][H][D], a NaN flag per token and head, boxes [n_pages][H][2][D]."""

    def __init__(self, n_pages, H, D):
        self.k = np.zeros((n_pages * PAGE, H, D))
        self.v = np.zeros_like(self.k)
        self.bad = np.zeros((n_pages * PAGE, H), bool)
        self.boxes = np.zeros((n_pages, H, 2, D))

    def append(self, k, v, slots):
        k, v = np.asarray(k, np.float64), np.asarray(v, np.float64)
        bad = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))
        k, v = np.where(bad[..., None], 0.0, k), np.where(bad[..., None], 0.0, v)
        kq, vq = quantise(k)[2], quantise(v)[2]
        for i, s in enumerate(slots):
            if not 0 <= s < self.k.shape[0]:
                continue
            self.k[s], self.v[s], self.bad[s] = kq[i], vq[i], bad[i]
            box = self.boxes[s // PAGE]
            if s % PAGE == 0:
                box[:, 0], box[:, 1] = kq[i], kq[i]
            else:
                box[:, 0], box[:, 1] = np.minimum(box[:, 0], kq[i]), np.maximum(box[:, 1], kq[i])
        return np.where(bad[..., None], np.nan, kq), vq


def plan(past, new, table, ring, state, max_tokens):
    """One request after the other.  Returns a dict; table and ring are copies."""
    table, ring = table.copy(), ring.copy()
    W, (head, tail, _) = table.shape[1], state
    old, back, missing, t = ring.copy(), tail, 0, 0
    kv, start = [], [0]
    slots, reqs, poss = (np.full(max_tokens, -1, np.int64) for _ in range(3))
    for r, (p, n) in enumerate(zip(past, new)):
        p = min(max(p, 0), W * PAGE)
        held = -(-p // PAGE)
        if n < 0:
            for c in range(held):
                ring[back % len(ring)] = table[r, c]
                back += 1
        total = min(p + max(n, 0), W * PAGE)
        if n >= 0:
            for c in range(held, -(-total // PAGE)):
                if head < tail:
                    table[r, c] = old[head % len(ring)]
                    head += 1
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
                requests=reqs, positions=poss, state=np.array([head, back, missing], np.int64))


def rounded_queries(q, H):
    """q [T][Hq][D] as whole numbers, a factor per token and kv head (32-bit steps by definition)."""
    T, Hq, D = q.shape
    x = np.where(np.isfinite(q), q, 0.0).astype(np.float32).reshape(T, H, Hq // H, D)
    top = np.abs(x).max((2, 3), keepdims=True)
    with np.errstate(divide="ignore", over="ignore", invalid="ignore"):
        f = np.float32(127.0) * (np.float32(1.0) / top)
    f = np.where(np.isfinite(f), f, np.float32(0.0)).astype(np.float32)
    return np.rint(x * f).astype(np.int64)


def select(cache, q, H, step, n_pages, n, sinks, recent):
    T = len(step["positions"])
    qi = rounded_queries(q, H)
    out = np.full((T, H, n), -1, np.int64)
    for t in range(T):
        r, pos = step["requests"][t], step["positions"][t]
        if r < 0:
            continue
        W = step["table"].shape[1]
        visible = min(pos // PAGE + 1, W)
        for h in range(H):
            if visible <= n:
                out[t, h, :visible] = np.arange(visible)
                continue
            keys = []
            for c in range(visible):
                page = step["table"][r, c]
                if c < sinks or c >= visible - recent:
                    keys.append((-np.inf, c))
                elif not 0 <= page < n_pages:
                    keys.append((np.inf, c))
                else:
                    lo, hi = cache.boxes[page, h]
                    top = max(np.abs(lo).max(), np.abs(hi).max())
                    e = (max(int(np.frexp(top)[1]) - 1 + 127, 8) if top > 0 else 8) - 127 - 6
                    lo, hi = np.floor(np.ldexp(lo, -e)), np.ceil(np.ldexp(hi, -e))
                    s = max(int(np.maximum(x * lo, x * hi).sum()) for x in qi[t, h])
                    keys.append((-np.ldexp(float(s), e), c))
            out[t, h] = sorted(c for _, c in sorted(keys)[:n])
    return out


def attention(cache, q, H, step, n_pages, scale, window=0, selected=None):
    """(out, lse, mass = sum_j p_j |v_j|, reach = sum_j |v_j|, size = largest sum_d |q_d k_d|) in 64 bits."""
    T, Hq, D = q.shape
    q = np.asarray(q, np.float64)
    out, mass, reach = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, size = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    W = step["table"].shape[1]
    for t in range(T):
        r, pos = step["requests"][t], step["positions"][t]
        if r < 0:
            continue
        high = min(pos, step["kv_lens"][r] - 1)
        j = np.arange(max(0, pos - window + 1) if window else 0, high + 1)
        pages = step["table"][r, j // PAGE]
        j, pages = j[(pages >= 0) & (pages < n_pages)], pages[(pages >= 0) & (pages < n_pages)]
        for h in range(Hq):
            hk = h // (Hq // H)
            keep = np.isin(j // PAGE, selected[t, hk][selected[t, hk] >= 0]) if selected is not None else np.ones(len(j), bool)
            at = pages[keep].astype(np.int64) * PAGE + j[keep] % PAGE
            if len(at) == 0:
                continue
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


def bounds(out, lse, mass, reach, size, D, fp16):
    """How far results may be off: (of out, of lse).

    u, half a unit of the type, relative: 2^-8 for bf16 (8 significant bits: 1 + 2^-8 lies midway between neighbours), 2^-11
    for fp16 (11 bits).  Every weight is rounded to the type once, u of it
    (in fp16, whose smallest step is 2^-24, 2^-25 at least; in 32 bits and bf16 weights below 2^-126 are 0; the weights' sum, kept in 32 bits, is 1 at least), and so is the
    result.  A score in 32 bits: D products summed and scaled, 2^-24 of the sum of their sizes each; the exponential's
    argument and value a few 2^-23 of their sizes.  A score that is off by d moves its weight by d, relative, and the sum of
    weights by as much."""
    u = 2.0 ** -11 if fp16 else 2.0 ** -8
    d = (D + 4) * 2.0 ** -24 * size + 2.0 ** -21 * (1 + size)
    off = u * np.abs(out) + mass * (u + 2 * d[..., None]) * 1.01
    off = off + (2.0 ** -25 * reach + 2.0 ** -25 if fp16 else 2.0 ** -125 * reach)
    return off, d + 2.0 ** -21 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0.0)))
