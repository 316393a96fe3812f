"""The measured cases of decoding with drafted tokens over the paged 4-bit key/value cache: rotary positions with several
axes, trees of drafted tokens, their attention, keeping the accepted ones, reading held tokens back.

A case is a dict of plain values:
  op        "rotate"     queries and keys turned by their positions on one or several axes
            "tree"       from every drafted token's parent: which drafted tokens it sees, and its position
            "attention"  the drafted tokens' attention: what is held before them, and of themselves their ancestors
            "keep"       of every request the longest path that the model agrees with: its tokens move together in the caches
                         of all layers, the boxes of their pages are those of what stays, pages behind it go back
            "read"       held keys and values back as rows
  dtype     "bf16" or "fp16"
  requests, short, long   number of requests and the range of tokens that they hold before the step (spread over it)
  new       drafted tokens of the longest request (the others have fewer); tokens in all (rotate, read)
  heads, kv_heads, dim    query heads, key/value heads, channels of a head
  window    tokens that a token sees, itself among them (0: all before it)
  packed    queries and keys are views of one projection's rows
  layers    caches that keep the same tokens (keep)
  axes, turned, beside    axes of a position; channels that are turned; whether the two of a pair are neighbours (rotate)
  run       tokens that follow each other in a page (read)

A page holds 64 tokens of all kv heads, 68 dim bytes a head.  A held value is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign
(4 bits) times a power of two shared by 32 channels (8 bits).  `own` chooses between the framework's calls and plain torch operations.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
VOCABULARY = 32000
BASE = 500000.0  # of the frequencies: BASE ** (-2 i / turned)


def listed():
    base = dict(heads=32, kv_heads=8, dim=128, window=0, packed=False, layers=0, axes=0, turned=0, beside=False, run=0,
                requests=1, short=0, long=0, dtype="bf16")
    return [
        # one token of a small model: nothing but latency
        dict(base, name="rotate_one", op="rotate", dtype="fp16", new=1, long=333, heads=12, kv_heads=12, dim=64, axes=1, turned=64),
        # a prompt with images in it: time, height and width, out of the rows of one projection
        dict(base, name="rotate_images", op="rotate", new=9001, long=130000, packed=True, axes=3, turned=128),
        # the tree of a single request
        dict(base, name="tree_one", op="tree", new=26, short=1000, long=1000),
        # a full server: hundreds of requests with trees of all sizes
        dict(base, name="tree_server", op="tree", requests=700, short=0, long=60000, new=200),
        # a chat turn of a small model: a few drafted tokens behind a few hundred held
        dict(base, name="attend_one", op="attention", dtype="fp16", short=333, long=333, new=7, heads=12, kv_heads=12, dim=64),
        # a batch of ragged contexts, a tree each, eight query heads to a key head
        dict(base, name="attend_batch", op="attention", requests=24, short=700, long=33000, new=32, heads=64),
        # a tree behind a single very long context
        dict(base, name="attend_long", op="attention", short=300001, long=300001, new=16),
        # larger trees, a window over them, every head its own keys, 96 channels
        dict(base, name="attend_window", op="attention", dtype="fp16", requests=9, short=50, long=7000, new=61, heads=16,
             kv_heads=16, dim=96, window=1000),
        # a single request's tokens in the caches of a few layers
        dict(base, name="keep_one", op="keep", short=500, long=500, new=10, layers=4),
        # a batch, all layers of a model
        dict(base, name="keep_batch", op="keep", requests=48, short=0, long=250, new=64, layers=28),
        # a few hundred tokens from everywhere, as a check of what is held
        dict(base, name="read_some", op="read", dtype="fp16", new=301, dim=64, long=40000, run=1),
        # a shared prefix of many pages, to hand it on unrounded
        dict(base, name="read_prefix", op="read", new=30011, long=40000, run=64),
    ]


def _between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kv_heads = rng.choice((1, 2, 4, 5, 8))
    case = dict(op=rng.choice(("rotate", "tree", "attention", "attention", "keep", "read")), dtype=rng.choice(("bf16", "fp16")),
                kv_heads=kv_heads, heads=kv_heads * rng.choice((1, 2, 3, 4, 6, 8, 12)), dim=rng.choice((64, 96, 128, 128, 256)),
                requests=1, short=0, long=0, new=1, window=0, packed=False, layers=0, axes=0, turned=0, beside=False, run=0)
    if case["op"] == "rotate":
        case.update(new=_between(rng, 1, 8000), long=_between(rng, 100, 1000000), axes=rng.choice((1, 2, 3, 4)),
                    beside=rng.random() < 0.4, packed=rng.random() < 0.5)
        case["turned"] = rng.choice((case["dim"], case["dim"], case["dim"] // 2, 32))
    elif case["op"] == "tree":
        case.update(new=_between(rng, 2, 1000), long=_between(rng, 1, 100000), window=rng.choice((0, 0, rng.randint(1, 20))))
        case["requests"] = _between(rng, 1, max(2, min(600, 50000 // case["new"])))
    elif case["op"] == "attention":
        case["requests"] = _between(rng, 1, 32)
        case["long"] = _between(rng, 8, 200000 // case["requests"])
        case["new"] = _between(rng, 2, 300 if case["requests"] < 6 else 48)
        if rng.random() < 0.3:
            case["window"] = _between(rng, 1, 5000)
    elif case["op"] == "keep":
        case.update(requests=_between(rng, 1, 48), long=_between(rng, 1, 250), new=_between(rng, 2, 64), layers=rng.randint(1, 28))
    else:
        case.update(new=_between(rng, 1, 30000), long=_between(rng, 64, 40000), run=rng.choice((1, 3, 17, 64)))
    case["short"] = case["long"] if case["op"] in ("rotate", "read") else min(
        case["long"], rng.choice((0, case["long"], _between(rng, 1, max(1, case["long"])))))
    # no more work than the largest listed case of its kind
    most = [work(c) for c in listed() if c["op"] == case["op"]]
    size = {"rotate": "new", "tree": "requests", "attention": "long", "keep": "layers", "read": "new"}[case["op"]]
    while case[size] > 1 and any(work(case)[k] > max(m[k] for m in most) for k in ("bytes", "flops")):
        case[size] = case[size] * 3 // 4
        case["short"] = min(case["short"], case["long"])
    return case


# ---- lengths ------------------------------------------------------------------------------------


def _lengths(case):
    """(tokens held, drafted tokens) of every request."""
    i = np.arange(case["requests"])
    f, g = (0.37 + 0.6180339887 * i) % 1.0, np.where(i, (1.0 + 0.7548776662 * i) % 1.0, 1.0)
    past = np.round((case["short"] + 1.0) * ((case["long"] + 1.0) / (case["short"] + 1.0)) ** f).astype(np.int64) - 1
    return past, np.maximum(1, np.round(case["new"] * g)).astype(np.int64)


def _pages_of(tokens):
    return (tokens + PAGE - 1) // PAGE


def work(case):
    H, G, D, n = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"], case["new"]
    row, held = H * D * 2, H * (D + D // 16)  # bytes of a token's keys (or values) as rows, and of both as they are held
    if case["op"] == "rotate":
        return {"bytes": 2 * n * (G + 1) * row + 4 * n * case["axes"], "flops": 3 * n * (G + 1) * H * case["turned"]}
    if case["op"] == "read":
        return {"bytes": n * (held + 2 * row + 8), "flops": 2 * n * H * D}
    past, new = _lengths(case)
    T, words = int(new.sum()), _words(case)
    if case["op"] == "tree":
        return {"bytes": T * (4 + 4 + 4 + 8 * words), "flops": T * words}
    if case["op"] == "keep":
        # a third of a request's tokens stays at most; each moves, and the keys of its page make the new box
        kept = int((1 + new // 8).sum())
        pages = case["requests"]
        return {"bytes": T * (4 + 4 + 4 + 8 * words) + case["layers"] * (2 * kept * held + pages * (H * 17 * D + 4 * H * D)),
                "flops": case["layers"] * pages * PAGE * H * D}
    ahead = np.minimum(past, case["window"]) if case["window"] else past
    reach = np.minimum(past, case["window"] + new) if case["window"] else past
    return {"bytes": int((reach + new).sum()) * held + 2 * T * G * row + 4 * T * H * G + 8 * T * words,
            "flops": int(4 * D * H * G * (new * (ahead + 4)).sum())}


# ---- the page's layout, as the framework documents it -------------------------------------------


def _codes(x):
    """Codes (a byte each) and scale bytes of rows [...][D]."""
    g = x.float().unflatten(-1, (-1, 32))
    b = ((g.abs().amax(-1, keepdim=True).view(torch.int32) >> 23) - 2).clamp(1, 254)
    y = g.abs() * ((254 - b) << 23).view(torch.float32)
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
    return (code | ((g < 0).to(torch.uint8) << 3)).flatten(-2), b.squeeze(-1).to(torch.uint8)


def _packed(k, v):
    """Pages [P][H][68 D] of keys and values [P][64][H][D]."""
    P, _, H, D = k.shape
    (kc, ks), (vc, vs) = _codes(k.transpose(1, 2)), _codes(v.transpose(1, 2))      # [P][H][64][D], [P][H][64][D/32]
    keys = kc[..., 0::2] | (kc[..., 1::2] << 4)
    key_scale = ks.unflatten(2, (4, 16)).permute(0, 1, 3, 4, 2)                       # place: (t % 16, group, t / 16)
    vc = vc.unflatten(3, (D // 32, 2, 16)).unflatten(2, (4, 4, 4))                 # t / 16, t / 4 % 4, t % 4, group, half, channel
    values = (vc[..., 0, :] | (vc[..., 1, :] << 4)).permute(0, 1, 5, 3, 6, 2, 4)
    value_scale = vs.unflatten(2, (4, 4, 4)).permute(0, 1, 5, 3, 2, 4)
    return torch.cat([x.reshape(P, H, -1) for x in (keys, key_scale, values, value_scale)], -1)


def _values_of(code, scale):
    """Codes [...][D] and scale bytes [...][D/32] as values in 32 bits."""
    grid = torch.tensor(GRID + tuple(-x for x in GRID), device="cuda")
    return (grid[code.int()].unflatten(-1, (-1, 32)) * (scale.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _keys(pages, D):
    """Held keys [P][H][64][D] of pages [P][H][68 D]."""
    code = pages[..., :32 * D].unflatten(-1, (PAGE, D // 2))
    scale = pages[..., 32 * D:34 * D].unflatten(-1, (16, D // 32, 4)).permute(0, 1, 4, 2, 3).flatten(2, 3)
    return _values_of(torch.stack((code & 15, code >> 4), -1).flatten(-2), scale)


def _values(pages, D):
    code = pages[..., 34 * D:66 * D].unflatten(-1, (D // 32, 4, 16, 4, 4)).permute(0, 1, 5, 3, 6, 2, 4)
    scale = pages[..., 66 * D:].unflatten(-1, (D // 32, 4, 4, 4)).permute(0, 1, 4, 3, 5, 2)
    return _values_of(torch.stack((code & 15, code >> 4), -2).flatten(5).reshape(*pages.shape[:2], PAGE, D), scale.reshape(*pages.shape[:2], PAGE, D // 32))


def _bytes_of_token(D):
    """Where a page and head has the bytes of token t: [64][68 D / 64]."""
    t, byte, group, c = np.arange(PAGE)[:, None], np.arange(D // 2)[None], np.arange(D // 32)[None], np.arange(D // 2)[None]
    place = ((t // 4) % 4, (t // 16) * 4 + t % 4)
    at = np.concatenate((t * (D // 2) + byte, 32 * D + ((t % 16) * (D // 32) + group) * 4 + t // 16,
                         34 * D + (c // 16) * 1024 + (place[0] * 16 + c % 16) * 16 + place[1], 66 * D + group * 64 + place[0] * 16 + place[1]), 1)
    return torch.from_numpy(at).cuda()


# ---- inputs -------------------------------------------------------------------------------------


def _generator(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (seed + 1) + part)
    return g


def _words(case):
    return (case["new"] + 63) // 64


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _held_pages(case, seed, n_pages, part):
    """Pages as a cache holds them, keys with a few channels that are large in every token, as in trained models."""
    H, D, dtype = case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    g = _generator(seed, part)
    gain = torch.exp(0.7 * torch.randn(H, D, device="cuda", generator=g)).to(dtype)
    pages = torch.empty(n_pages, H, 68 * D, dtype=torch.uint8, device="cuda")
    piece = max(1, (1 << 26) // (PAGE * H * D))
    for a in range(0, n_pages, piece):
        shape = (min(piece, n_pages - a), PAGE, H, D)
        k = torch.randn(shape, device="cuda", generator=g, dtype=dtype) * gain
        pages[a:a + piece] = _packed(k, torch.randn(shape, device="cuda", generator=g, dtype=dtype))
    return pages


def _parents(gen, new):
    """Trees: the first token of a request is the last that is certain, each other hangs on one before it."""
    parents = np.full(int(new.sum()), -1, dtype=np.int32)
    at = 0
    for n in new:
        parents[at + 1:at + n] = np.floor(gen.random(n - 1) * np.arange(1, n))
        at += n
    return parents


def _inputs(case, seed):
    """Lengths, page tables, trees and rows, from the seed alone."""
    gen, g = np.random.default_rng([seed, 13]), _generator(seed, 1)
    H, G, D, dtype = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    x = dict(lens=())
    if case["op"] == "rotate":
        T = case["new"]
        rows = torch.randn(T, H * G + H, D, device="cuda", generator=g).to(dtype)
        x["q"], x["k"] = (rows[:, :H * G], rows[:, H * G:]) if case["packed"] else (rows[:, :H * G].contiguous(), rows[:, H * G:].contiguous())
        # time goes on, height and width stay near it, as where an image begins at the time that its text has reached
        time = np.sort(gen.integers(0, case["long"] + 1, T))
        x["positions"] = _dev(np.stack([time] + [time + gen.integers(0, 40, T) for _ in range(case["axes"] - 1)]).astype(np.int32))
        half = case["turned"] // 2
        x["frequencies"] = [BASE ** (-2.0 * i / case["turned"]) for i in range(half)]
        x["axis"] = [min(i * case["axes"] // half, case["axes"] - 1) for i in range(half)]
        return x
    if case["op"] == "read":
        n_pages = _pages_of(case["long"])
        first = gen.integers(0, n_pages * PAGE // case["run"], -(-case["new"] // case["run"]))
        slots = (first[:, None] * case["run"] + np.arange(case["run"])[None]).reshape(-1)[:case["new"]]
        return dict(x, slots=_dev(slots.astype(np.int64)), n_pages=n_pages)
    past, new = _lengths(case)
    order = gen.permutation(case["requests"])
    past, new = past[order], new[order]
    held, need = _pages_of(past), _pages_of(past + new)
    width, n_pages = int(need.max()) + 1, int(need.sum()) + 5
    ids, at = gen.permutation(n_pages).astype(np.int32), np.concatenate(([0], np.cumsum(held)))
    table = np.full((case["requests"], width), -1, dtype=np.int32)
    after = table.copy()
    taken = at[-1] + np.concatenate(([0], np.cumsum(need - held)))
    for r in range(case["requests"]):
        after[r, :held[r]] = table[r, :held[r]] = ids[at[r]:at[r + 1]]
        after[r, held[r]:need[r]] = ids[taken[r]:taken[r + 1]]
    # the pages that nobody holds, in a ring that has gone round a few times
    head, left = int(gen.integers(0, 3 * n_pages)), n_pages - int(at[-1])
    free = np.zeros(n_pages, dtype=np.int32)
    free[(head + np.arange(left)) % n_pages] = ids[at[-1]:]
    start = np.concatenate(([0], np.cumsum(new)))
    node = np.arange(start[-1]) - np.repeat(start[:-1], new)
    request, position = np.repeat(np.arange(case["requests"]), new), np.repeat(past, new) + node
    slots = after[request, position // PAGE].astype(np.int64) * PAGE + position % PAGE
    parents = _parents(gen, new)
    x.update(past=_dev(past.astype(np.int32)), new=_dev(new.astype(np.int32)), before=_dev(table), table=_dev(after), free=_dev(free),
             state=_dev(np.array([head, head + left, 0], dtype=np.int64)), tokens=int(start[-1]), n_pages=n_pages,
             taken=int(taken[-1] - at[-1]), start=_dev(start), request=_dev(request), node=_dev(node), slots=_dev(slots),
             parents=_dev(parents), lens=[(int(p), int(n)) for p, n in zip(past, new)])
    if case["op"] == "attention":
        x["q"] = torch.randn(x["tokens"], H * G, D, device="cuda", generator=g).to(dtype)
    if case["op"] == "keep":
        x["drafted"], x["picked"] = (_dev(a) for a in _agreed(gen, parents, new))
    return x


def _agreed(gen, parents, new):
    """Tokens drafted, and those that the model picks behind each: they agree along one path of every tree.  A path is
    taken none of whose tokens moves to where another of it comes from, so that a pass can be repeated."""
    drafted, picked = [], []
    at = 0
    for n in new.tolist():
        p = parents[at:at + n]
        paths = [[0]]
        for i in range(1, n):
            paths.append(paths[p[i]] + [i])
        fit = [w for w in paths if all(a == i or a >= len(w) for i, a in enumerate(w))]
        deep = max(map(len, fit))
        path = [w for w in fit if 2 * len(w) >= deep][int(gen.integers(1 << 30)) % sum(2 * len(w) >= deep for w in fit)]
        d = (int(gen.integers(VOCABULARY // 2)) + 7 * np.arange(n)) % (VOCABULARY // 2)  # no token twice in a tree of this size
        k = gen.integers(VOCABULARY // 2, VOCABULARY, n)
        k[path[:-1]] = d[path[1:]]
        drafted.append(d)
        picked.append(k)
        at += n
    return np.concatenate(drafted).astype(np.int32), np.concatenate(picked).astype(np.int32)


def prepare(case, seed):
    x = _inputs(case, seed)
    st = dict(x, case=case)
    H, D, dtype = case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    if own:
        from paper_2312_01712_amd import kv
        st["kv"] = kv
    if case["op"] == "rotate":
        st["out"] = torch.empty(x["q"].shape, dtype=dtype, device="cuda"), torch.empty(x["k"].shape, dtype=dtype, device="cuda")
        if own:
            st["rotary"] = kv.Rotary(x["frequencies"], axes=x["axis"], neighbours=case["beside"])
        else:
            st["frequencies"] = torch.tensor(x["frequencies"], dtype=torch.float64, device="cuda")
            st["axis"] = torch.tensor(x["axis"], device="cuda")
        return st
    if case["op"] == "read":
        pages = _held_pages(case, seed, x["n_pages"], 2)
        st["out"] = [torch.empty(case["new"], H, D, dtype=dtype, device="cuda") for _ in range(2)]
        if own:
            st["cache"] = kv.KvCache(x["n_pages"], H, D, dtype)
            st["cache"].pages.copy_(pages.flatten(1))
        else:
            st["pages"] = pages
        return st
    if own:
        ring = x["free"].clone()
        st["step"] = kv.plan(x["past"], x["new"], x["before"], ring, x["state"], max_tokens=x["tokens"])
        st["tree"] = kv.Tree.empty(x["tokens"], case["new"], window=case["window"])
        if case["op"] != "tree":
            kv.tree(x["parents"], st["step"], out=st["tree"])
    if case["op"] == "tree":
        return st
    if not own:
        st["masks"], st["positions"] = _tree_plain(st)
    if case["op"] == "attention":
        pages = _held_pages(case, seed, x["n_pages"], 2)
        if own:
            cache = st["cache"] = kv.KvCache(x["n_pages"], H, D, dtype)
            cache.pages.copy_(pages.flatten(1))
            st["work"] = cache.tree_attention_workspace(st["step"], case["heads"], st["tree"])
            st["to"] = torch.empty(x["q"].shape, dtype=dtype, device="cuda")
            st["lse"] = torch.empty(x["q"].shape[:2], dtype=torch.float32, device="cuda")
        else:
            st["pages"] = pages
        return st
    # the caches of all layers after the drafted tokens were appended: their boxes are those of all tokens held
    st["state"] = x["state"] + torch.tensor([x["taken"], 0, 0], device="cuda")
    stacked = [_held_pages(case, seed, x["n_pages"], 2 + n) for n in range(case["layers"])]
    boxes = [_boxes(st, p, x["past"].long() + x["new"].long(), 0) for p in stacked]
    if own:
        st["caches"] = [kv.KvCache(x["n_pages"], H, D, dtype) for _ in stacked]
        for c, p, b in zip(st["caches"], stacked, boxes):
            c.pages.copy_(p.flatten(1))
            c.boxes.copy_(b)
        st["kept"] = kv.Kept.empty(st["step"])
    else:
        st["stacked"], st["boxes"], st["places"] = torch.stack(stacked), torch.stack(boxes), _bytes_of_token(D)
    return st


# ---- the plain forms ----------------------------------------------------------------------------


def _rotate_plain(st):
    case, R = st["case"], st["case"]["turned"]
    turn = st["positions"].double()[st["axis"]].t() * st["frequencies"]                  # [T][R / 2], in 64 bits: far positions
    cos, sin = turn.cos().float()[:, None], turn.sin().float()[:, None]

    def of(x, out):
        y = x[..., :R].float()
        a, b = (y[..., 0::2], y[..., 1::2]) if case["beside"] else (y[..., :R // 2], y[..., R // 2:])
        c, d = a * cos - b * sin, b * cos + a * sin
        out[..., :R] = torch.stack((c, d), -1).flatten(-2) if case["beside"] else torch.cat((c, d), -1)
        out[..., R:] = x[..., R:]
        return out

    return [of(st["q"], st["out"][0]), of(st["k"], st["out"][1])]


def _tree_plain(st):
    """Masks [T][words] (bit j: token j of the request is seen) and positions [T]: by the tokens' ancestors, one generation a turn."""
    case, T = st["case"], st["tokens"]
    first, node = st["start"][:-1][st["request"]], st["node"]
    depth = torch.zeros(T, dtype=torch.int32, device="cuda")
    masks = torch.zeros(T, _words(case), dtype=torch.int64, device="cuda")
    at, rows, far = node.clone(), torch.arange(T, device="cuda"), 0
    while rows.numel():
        if not case["window"] or far < case["window"]:
            masks[rows, at >> 6] |= torch.ones_like(at) << (at & 63)
        up = st["parents"][first[rows] + at].long()
        rows, at, far = rows[up >= 0], up[up >= 0], far + 1
        depth[rows] += 1
    return masks, st["past"][st["request"]] + depth


def _attention_plain(st):
    case = st["case"]
    H, G, D, dtype = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    out, lse = torch.empty_like(st["q"]), torch.empty(st["q"].shape[:2], device="cuda")
    bit = torch.arange(64, device="cuda")
    t = 0
    for r, (past, new) in enumerate(st["lens"]):
        pages = st["pages"][st["table"][r, :_pages_of(past + new)].long()]
        k = _keys(pages, D).transpose(0, 1).flatten(1, 2)[:, :past + new]               # [H][past + new][D]
        v = _values(pages, D).transpose(0, 1).flatten(1, 2)[:, :past + new]
        own_part = (st["masks"][t:t + new, :, None] >> bit & 1).bool().flatten(1)[:, :new]
        key = torch.arange(past, device="cuda")
        before = key > st["positions"][t:t + new, None] - case["window"] if case["window"] else key.expand(new, -1) >= 0
        seen = torch.cat((before, own_part), 1)                                         # [new][past + new]
        q = st["q"][t:t + new].float().unflatten(1, (H, G)).permute(1, 0, 2, 3).flatten(1, 2) / math.sqrt(D)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()).unflatten(1, (new, G))
        s.masked_fill_(~seen[:, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul((p / total).flatten(1, 2), v).unflatten(1, (new, G))
        out[t:t + new] = o.permute(1, 0, 2, 3).flatten(1, 2).to(dtype)
        lse[t:t + new] = (top + torch.log(total)).squeeze(-1).permute(1, 0, 2).flatten(1, 2)
        t += new
    return [out, lse]


def _boxes(st, pages, lens, since):
    """Boxes [n_pages][H][2][D] bf16 of the keys that requests of these lengths hold; only of pages with a token from `since` on
    (a tensor, or 0 for all)."""
    case, table = st["case"], st["table"].long()
    col = torch.arange(table.shape[1], device="cuda")[None]
    wanted = (col * PAGE < lens[:, None]) & ((col + 1) * PAGE > (since[:, None] if torch.is_tensor(since) else since))
    request, column = wanted.nonzero(as_tuple=True)
    page = table[request, column]
    k = _keys(pages[page], case["dim"])                                                 # [P][H][64][D]
    there = (torch.arange(PAGE, device="cuda") < (lens[request] - column * PAGE)[:, None])[:, None, :, None]
    box = torch.stack((torch.where(there, k, math.inf).amin(2), torch.where(there, k, -math.inf).amax(2)), 2).bfloat16()
    if not torch.is_tensor(since):
        new = torch.zeros(pages.shape[0], *box.shape[1:], dtype=torch.bfloat16, device="cuda")
        new[page] = box
        return new
    return page, box


def _keep_plain(st):
    case, start, request, node = st["case"], st["start"], st["request"], st["node"]
    T, R, N = st["tokens"], case["requests"], _words(case) * 64
    first = start[:-1][request]
    seen = (st["masks"][:, :, None] >> torch.arange(64, device="cuda") & 1).bool().flatten(1)      # [T][N]
    parent = st["parents"].long()
    agrees = (node == 0) | ((parent >= 0) & (st["drafted"] == st["picked"][first + parent.clamp(min=0)]))
    padded = torch.ones(R, N, dtype=torch.bool, device="cuda")
    padded[request, node] = agrees
    good = ~(seen & ~padded[request]).any(1)
    # the deepest, the first among equals
    rank = torch.where(good, seen.sum(1) * N + N - 1 - node, -1)
    best = torch.full((R,), -1, dtype=torch.int64, device="cuda").scatter_reduce(0, request, rank, "amax")
    path = seen[start[:-1] + N - 1 - best % N]                                                     # [R][N]
    kept = path.sum(1)
    r, j = path.nonzero(as_tuple=True)
    to = start[:-1][r] + (path.cumsum(1) - 1)[r, j]
    rows = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    rows[to] = (start[:-1][r] + j).int()
    past = st["past"].long()
    lens = past + kept
    # the bytes of what stays, to where it belongs
    source, target = st["slots"][start[:-1][r] + j], st["slots"][to]
    layer = torch.arange(case["layers"], device="cuda")[:, None, None, None]
    head = torch.arange(case["kv_heads"], device="cuda")[None, None, :, None]
    at = lambda s: (layer, (s // PAGE)[None, :, None, None], head, st["places"][s % PAGE][None, :, None, :])
    st["stacked"][at(target)] = st["stacked"][at(source)]
    for pages, boxes in zip(st["stacked"], st["boxes"]):
        page, box = _boxes(st, pages, lens, past)
        boxes[page] = box
    # pages behind what stays, in the order of requests
    col = torch.arange(st["table"].shape[1], device="cuda")[None]
    back = (col >= ((lens + PAGE - 1) // PAGE)[:, None]) & (col < ((past + st["new"].long() + PAGE - 1) // PAGE)[:, None])
    given = st["table"][back]
    tail = st["state"][1]
    st["free"][(tail + torch.arange(given.numel(), device="cuda")) % st["free"].numel()] = given
    state = st["state"] + torch.stack((tail * 0, tail * 0 + given.numel(), tail * 0))
    return [lens.int(), rows, state, st["free"], [p.flatten(1) for p in st["stacked"]], list(st["boxes"])]


def _read_plain(st):
    case, slots = st["case"], st["slots"]
    D = case["dim"]
    at = _bytes_of_token(D)[slots % PAGE]                                                          # [T][68 D / 64]
    b = st["pages"][(slots // PAGE)[:, None, None], torch.arange(case["kv_heads"], device="cuda")[None, :, None], at[:, None]]
    kc, ks, vc, vs = b.split((D // 2, D // 32, D // 2, D // 32), -1)
    vc = vc.unflatten(-1, (D // 32, 16))
    st["out"][0].copy_(_values_of(torch.stack((kc & 15, kc >> 4), -1).flatten(-2), ks))
    st["out"][1].copy_(_values_of(torch.stack((vc & 15, vc >> 4), -2).flatten(-3), vs))
    return st["out"]


def run(st):
    op = st["case"]["op"]
    if own:
        if op == "rotate":
            return list(st["rotary"](st["q"], st["k"], st["positions"], out=st["out"]))
        if op == "tree":
            tree = st["kv"].tree(st["parents"], st["step"], out=st["tree"])
            return [tree.masks, tree.positions]
        if op == "attention":
            return list(st["cache"].tree_attention(st["q"], st["step"], st["tree"], out=st["to"], lse=st["lse"], workspace=st["work"]))
        if op == "read":
            return list(st["cache"].read(st["slots"], out=st["out"]))
        kept = st["kv"].keep(st["caches"], st["step"], st["tree"], st["drafted"], st["picked"], st["free"], st["state"], out=st["kept"])
        return [kept.lens, kept.rows, kept.free_state, st["free"], [c.pages for c in st["caches"]], [c.boxes for c in st["caches"]]]
    if op == "tree":
        return list(_tree_plain(st))
    return {"rotate": _rotate_plain, "attention": _attention_plain, "read": _read_plain, "keep": _keep_plain}[op](st)


# ---- from the definitions, in 64 bits -----------------------------------------------------------


def _token(page, t, D):
    """Keys and values [H][D] in 64 bits of token t of a page [H][68 D] (numpy), channel by channel as the layout says."""
    c, grid = np.arange(D), np.array(GRID + tuple(-x for x in GRID))
    k = page[:, t * (D // 2) + c // 2] >> 4 * (c & 1) & 15
    v = page[:, 34 * D + (c // 32) * 1024 + (((t // 4) % 4) * 16 + c % 16) * 16 + (t // 16) * 4 + t % 4] >> 4 * ((c // 16) & 1) & 15
    ks = page[:, 32 * D + ((t % 16) * (D // 32) + c // 32) * 4 + t // 16].astype(np.int64)
    vs = page[:, 66 * D + (c // 32) * 64 + ((t // 4) % 4) * 16 + (t // 16) * 4 + t % 4].astype(np.int64)
    return grid[k] * np.exp2(ks - 127.0), grid[v] * np.exp2(vs - 127.0)


def _ancestors(parents, i):
    path = [i]
    while parents[path[-1]] >= 0:
        path.append(int(parents[path[-1]]))
    return path


def exact(case, seed):
    x = _inputs(case, seed)
    H, G, D = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"]
    if case["op"] == "rotate":
        found, half = [], case["turned"] // 2
        for rows in (x["q"], x["k"]):
            z = rows.double().clone()
            for i in range(half):
                one, two = (2 * i, 2 * i + 1) if case["beside"] else (i, i + half)
                turn = (x["positions"][x["axis"][i]].double() * x["frequencies"][i])[:, None]
                a, b = rows[..., one].double(), rows[..., two].double()
                z[..., one], z[..., two] = a * torch.cos(turn) - b * torch.sin(turn), a * torch.sin(turn) + b * torch.cos(turn)
            found.append(z)
        return found
    if case["op"] == "read":
        pages = _held_pages(case, seed, x["n_pages"], 2).cpu().numpy()
        rows = {}
        for s in x["slots"].tolist():
            if s not in rows:
                rows[s] = _token(pages[s // PAGE], s % PAGE, D)
        return [torch.from_numpy(np.stack([rows[s][i] for s in x["slots"].tolist()])).cuda() for i in range(2)]
    parents, lens = x["parents"].tolist(), x["lens"]
    masks, positions, t = [], [], 0
    for past, new in lens:
        for i in range(new):
            path = _ancestors(parents[t:t + new], i)
            mark = [0] * _words(case)
            for j in path[:case["window"] or None]:
                mark[j // 64] |= 1 << j % 64
            masks.append([m - (1 << 64) if m >> 63 else m for m in mark])
            positions.append(past + len(path) - 1)
        t += new
    if case["op"] == "tree":
        return [_dev(np.array(masks, dtype=np.int64)), _dev(np.array(positions, dtype=np.int32))]
    if case["op"] == "attention":
        return _exact_attention(case, x, seed, positions)
    drafted, picked, table, ring = x["drafted"].tolist(), x["picked"].tolist(), x["table"].tolist(), x["free"].tolist()
    rows, kept, t, back = [-1] * x["tokens"], [], 0, int(x["state"][1])
    for r, (past, new) in enumerate(lens):
        p, best = parents[t:t + new], [0]
        for i in range(new):
            path = _ancestors(p, i)[::-1]
            if path[0] == 0 and len(path) > len(best) and all(drafted[t + b] == picked[t + a] for a, b in zip(path, path[1:])):
                best = path
        rows[t:t + len(best)] = [t + i for i in best]
        kept.append(past + len(best))
        for c in range(_pages_of(kept[-1]), _pages_of(past + new)):
            ring[back % len(ring)] = table[r][c]
            back += 1
        t += new
    state = [int(x["state"][0]) + x["taken"], back, 0]
    return [_dev(np.array(kept, dtype=np.int32)), _dev(np.array(rows, dtype=np.int32)), _dev(np.array(state, dtype=np.int64)),
            _dev(np.array(ring, dtype=np.int32)), [None] * case["layers"], _exact_boxes(case, x, seed, rows, kept)]


def _exact_boxes(case, x, seed, rows, kept):
    """Boxes after the step: of pages that the drafted tokens touch those of the tokens that stay, of the others what was there."""
    D, slots, table = case["dim"], x["slots"].tolist(), x["table"].tolist()
    found = []
    for n in range(case["layers"]):
        pages = _held_pages(case, seed, x["n_pages"], 2 + n).cpu().numpy()
        box = np.zeros((x["n_pages"], case["kv_heads"], 2, D))
        t = 0
        for r, (past, new) in enumerate(x["lens"]):
            for c in range(_pages_of(past + new)):
                tokens = []
                for position in range(c * PAGE, min((c + 1) * PAGE, past + new)):
                    page, place = table[r][c], position % PAGE
                    if position >= past and c * PAGE < kept[r]:
                        if position >= kept[r]:
                            continue
                        page, place = divmod(slots[rows[t + position - past]], PAGE)
                    tokens.append(_token(pages[page], place, D)[0])
                box[table[r][c], :, 0], box[table[r][c], :, 1] = np.min(tokens, 0), np.max(tokens, 0)
            t += new
        found.append(torch.from_numpy(box).cuda())
        if n == 2:  # the other layers: the same in tens of seconds
            return found + [None] * (case["layers"] - 3)
    return found


def _exact_attention(case, x, seed, positions):
    H, G, D = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"]
    pages, parents = _held_pages(case, seed, x["n_pages"], 2), x["parents"].tolist()
    grid = torch.tensor(GRID + tuple(-g for g in GRID), dtype=torch.float64, device="cuda")
    out, lse = torch.empty(x["tokens"], H * G, D, dtype=torch.float64, device="cuda"), torch.empty(x["tokens"], H * G, dtype=torch.float64, device="cuda")
    c, t0 = torch.arange(D, device="cuda")[None], 0
    for r, (past, new) in enumerate(x["lens"]):
        j = torch.arange(past + new, device="cuda")
        page, t = x["table"][r].long()[j // PAGE][:, None], (j % PAGE)[:, None]
        see = torch.zeros(new, past + new, dtype=torch.bool, device="cuda")
        for i in range(new):
            low = max(0, positions[t0 + i] - case["window"] + 1) if case["window"] else 0
            see[i, low:past] = True
            see[i, torch.tensor(_ancestors(parents[t0:t0 + new], i)[:case["window"] or None], device="cuda") + past] = True
        for h in range(H):
            byte = lambda at: pages[page, h, at].long()
            k = grid[byte(t * (D // 2) + c // 2) >> 4 * (c & 1) & 15]
            k = k * torch.exp2(byte(32 * D + ((t % 16) * (D // 32) + c // 32) * 4 + t // 16).double() - 127.0)
            lane = ((t // 4) % 4) * 16
            v = grid[byte(34 * D + (c // 32) * 1024 + (lane + c % 16) * 16 + (t // 16) * 4 + t % 4) >> 4 * ((c // 16) & 1) & 15]
            v = v * torch.exp2(byte(66 * D + (c // 32) * 64 + lane + (t // 16) * 4 + t % 4).double() - 127.0)
            for g in range(h * G, h * G + G):
                s = x["q"][t0:t0 + new, g].double() @ k.t() * D ** -0.5
                s.masked_fill_(~see, -math.inf)
                lse[t0:t0 + new, g] = torch.logsumexp(s, -1)
                out[t0:t0 + new, g] = torch.softmax(s, -1) @ v
        t0 += new
    return [out, lse]
