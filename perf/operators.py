"""The measured cases of the paged 4-bit key/value cache: page tables, append, page selection, attention.

A case is a dict of plain values:
  op        "plan"       page tables and slot maps of one step from the requests' lengths
            "append"     keys and values of the step's new tokens into the cache
            "select"     the pages that each new token and kv head looks at, by a score from the pages' key boxes
            "attention"  the new tokens' attention over the cache, whole or over selected pages
  dtype     "bf16" or "fp16"
  requests, short, long   number of requests and the range of tokens that they hold before the step (spread over it)
  new       new tokens of the longest request; the others have fewer, unless it is 1
  heads, kv_heads, dim    query heads, key/value heads, channels of a head
  pages     pages selected for a token and kv head (0: attention over everything)
  window    tokens that a token sees, itself among them (0: all before it)
  packed    queries, keys and values are views of one projection's rows
  width     pages a row of the page table has room for (plan); every `retire`-th request ends in this step (plan)

A page holds 64 tokens.  A held value is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign (4 bits) times a power of two
shared by 32 channels (8 bits).  `own` chooses between the framework's calls and plain torch operations.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    heads = dict(heads=32, kv_heads=8, dim=128, pages=0, window=0, packed=False, width=0, retire=0)
    return [
        # the first step of a single request: nothing but latency
        dict(heads, name="plan_one", op="plan", dtype="bf16", requests=1, short=0, long=0, new=37, width=128),
        # a full server between two steps: thousands of requests, most add a token, some a few, some end
        dict(heads, name="plan_server", op="plan", dtype="bf16", requests=4001, short=0, long=131000, new=7, width=2064,
             retire=16),
        # one decode step of a batch: a token a request lands somewhere inside a page
        dict(heads, name="append_decode", op="append", dtype="bf16", requests=48, short=100, long=3000, new=1),
        # prompts written at once, out of the rows of one projection
        dict(heads, name="append_prompt", op="append", dtype="fp16", requests=5, short=0, long=700, new=5003, packed=True),
        # pages for one token of a single very long context
        dict(heads, name="select_long", op="select", dtype="bf16", requests=1, short=262000, long=262000, new=1, pages=128),
        # pages for a decode batch of ragged contexts, eight query heads to a key head
        dict(heads, name="select_batch", op="select", dtype="fp16", requests=61, short=900, long=65000, new=1, heads=64,
             pages=48),
        # a short chat turn of a small model: one token, a few hundred held, a head of 64
        dict(heads, name="attend_one", op="attention", dtype="fp16", requests=1, short=333, long=333, new=1, heads=12,
             kv_heads=12, dim=64),
        # a decode batch of ragged contexts
        dict(heads, name="attend_batch", op="attention", dtype="bf16", requests=40, short=700, long=33000, new=1, heads=64),
        # one token of a single very long context
        dict(heads, name="attend_long", op="attention", dtype="bf16", requests=1, short=520001, long=520001, new=1),
        # a chunk of a long prompt behind what is already held, out of the rows of one projection
        dict(heads, name="attend_chunk", op="attention", dtype="bf16", requests=1, short=8190, long=8190, new=2048,
             packed=True),
        # ragged chunks of several requests, a window over them, every head its own keys, 96 channels
        dict(heads, name="attend_window", op="attention", dtype="fp16", requests=6, short=50, long=5000, new=513, heads=16,
             kv_heads=16, dim=96, window=1000),
        # a decode batch of long contexts that looks at selected pages only
        dict(heads, name="attend_selected", op="attention", dtype="bf16", requests=24, short=9000, long=131000, new=1,
             heads=64, pages=64),
    ]


def _between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kv_heads = rng.choice((1, 2, 4, 5, 8))
    case = dict(op=rng.choice(("plan", "append", "select", "attention", "attention", "attention")), dtype=rng.choice(("bf16", "fp16")),
                kv_heads=kv_heads, heads=kv_heads * rng.choice((1, 2, 3, 4, 6, 8, 12, 16)), dim=rng.choice((64, 96, 128, 128, 256)),
                requests=1, short=0, long=0, new=1, pages=0, window=0, packed=rng.random() < 0.4, width=0, retire=0)
    if case["op"] == "plan":
        case.update(requests=_between(rng, 1, 4000), long=_between(rng, 1, 130000), new=_between(rng, 1, 64),
                    retire=rng.choice((0, 2, 7, 30)))
        case["width"] = (case["long"] + case["new"]) // PAGE + rng.randint(1, 17)
    elif case["op"] == "append":
        case.update(requests=_between(rng, 1, 64), long=_between(rng, 1, 2000))
        case["new"] = rng.choice((1, _between(rng, 2, max(2, 16000 // case["requests"]))))
    elif case["op"] == "select" or rng.random() < 0.7:
        case["requests"] = _between(rng, 1, 64)
        case["long"] = _between(rng, 8, 500000 // case["requests"])
        case["new"] = rng.choice((1, 1, rng.randint(2, 9)))
        case["pages"] = _between(rng, 4, 200) if case["op"] == "select" else rng.choice((0, _between(rng, 4, 100)))
    else:
        case["requests"] = _between(rng, 1, 8)
        case["long"] = _between(rng, 8, 16000 // case["requests"])
        case["new"] = _between(rng, 10, 2048 // case["requests"])
    case["short"] = min(case["long"], rng.choice((0, case["long"], _between(rng, 1, max(1, case["long"])))))
    if case["op"] == "attention" and not case["pages"] and rng.random() < 0.3:
        case["window"] = _between(rng, 1, 5000)
    return case


# ---- lengths ------------------------------------------------------------------------------------


def _lengths(case):
    """(tokens held, new tokens) of every request; -1 new tokens: the request ends."""
    past, new = [], []
    for i in range(case["requests"]):
        f, g = (0.37 + 0.6180339887 * i) % 1.0, (1.0 + 0.7548776662 * i) % 1.0 if i else 1.0
        past.append(int(round((case["short"] + 1.0) * ((case["long"] + 1.0) / (case["short"] + 1.0)) ** f)) - 1)
        new.append(case["new"] if case["new"] == 1 else max(1, int(round(case["new"] * g))))
        if case["op"] == "plan" and case["retire"] and i % case["retire"] == case["retire"] - 1:
            new[-1] = -1
    return past, new


def _pages_of(tokens):
    return (tokens + PAGE - 1) // PAGE


def _seen(case, total, position):
    """Tokens that a token at `position` sees (of a request of `total` tokens)."""
    if case["pages"]:
        return min(position + 1, case["pages"] * PAGE)
    return min(position + 1, case["window"]) if case["window"] else position + 1


def work(case):
    past, new = _lengths(case)
    R, H, G, D = case["requests"], case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"]
    T = sum(max(0, n) for n in new)
    if case["op"] == "plan":
        fresh = sum(_pages_of(p + n) - _pages_of(p) for p, n in zip(past, new) if n >= 0)
        ended = sum(_pages_of(p) for p, n in zip(past, new) if n < 0)
        # lengths in and out, offsets, slots (8), request and position of every token, pages taken and given back
        return {"bytes": 16 * R + 16 * T + 8 * (fresh + ended), "flops": 8 * (R + T + fresh + ended)}
    rows = T * H * D * 2
    if case["op"] == "append":
        pages = sum(_pages_of(p + n) - p // PAGE for p, n in zip(past, new))
        return {"bytes": 4 * rows + T * H * (D + D // 16) + 8 * T + 4 * pages * H * D, "flops": 16 * T * H * D}
    if case["op"] == "select":
        held = sum(_pages_of(p + n) for p, n in zip(past, new))
        scored = sum((p + j) // PAGE + 1 for p, n in zip(past, new) for j in range(n))
        return {"bytes": 4 * held * H * D + rows * G + 4 * T * H * case["pages"], "flops": 4 * D * scored * H * G}
    pairs = sum(_seen(case, p + n, p + j) for p, n in zip(past, new) for j in range(n))
    if case["pages"]:
        held = sum(min((p + n), n * case["pages"] * PAGE) for p, n in zip(past, new))
    else:
        held = sum(min(p + n, case["window"] + n) if case["window"] else p + n for p, n in zip(past, new))
    return {"bytes": held * H * (D + D // 16) + 2 * rows * G + 4 * T * H * G, "flops": 4 * D * pairs * H * G}


# ---- inputs -------------------------------------------------------------------------------------


def _generator(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (seed + 1) + part)
    return g


def _inputs(case, seed):
    """Lengths, page tables and the step's rows, from the seed alone; the cache's contents come from _held."""
    gen = np.random.default_rng([seed, 11])
    past, new = (np.array(x, dtype=np.int32) for x in _lengths(case))
    order = gen.permutation(case["requests"])
    past, new = past[order], new[order]
    total = np.where(new < 0, 0, past + new)
    held, need = _pages_of(past), _pages_of(total)
    fresh = np.maximum(need - held, 0) * (new >= 0)
    width = case["width"] or int(max(held.max(), need.max())) + 1
    n_pages = int(held.sum() + fresh.sum()) + 5
    ids = gen.permutation(n_pages).astype(np.int32)
    table = np.full((case["requests"], width), -1, dtype=np.int32)
    at = 0
    for r in range(case["requests"]):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += int(held[r])
    # the pages that nobody holds, in a ring that has gone round a few times
    head = int(gen.integers(0, 3 * n_pages))
    free = np.zeros(n_pages, dtype=np.int32)
    free[(head + np.arange(n_pages - at)) % n_pages] = ids[at:]
    T = int(np.maximum(new, 0).sum())
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    x = dict(past=dev(past), new=dev(new), table=dev(table), free=dev(free), n_pages=n_pages, width=width, tokens=T,
             state=dev(np.array([head, head + n_pages - at, 0], dtype=np.int64)),
             lens=[(int(p), int(n)) for p, n in zip(past, new)])
    if case["op"] == "plan":
        return x
    H, G, D, dtype = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    g = _generator(seed, 1)
    # a few channels of the keys are large in every token, as in trained models
    x["gain"] = torch.exp(0.7 * torch.randn(H, D, device="cuda", generator=g)).to(dtype)
    rows = torch.randn(T, H * G + 2 * H, D, device="cuda", generator=g).to(dtype)
    rows[:, H * G:H * G + H] *= x["gain"]
    parts = rows[:, :H * G], rows[:, H * G:H * G + H], rows[:, H * G + H:]
    x["q"], x["k"], x["v"] = parts if case["packed"] else (p.contiguous() for p in parts)
    if case["op"] == "attention" and case["pages"]:
        # ascending pages for every token and kv head, the token's own last; -1 behind them
        sel = np.full((T, H, case["pages"]), -1, dtype=np.int32)
        t = 0
        for p, n in x["lens"]:
            for j in range(n):
                seen = (p + j) // PAGE + 1
                take = min(seen, case["pages"])
                for h in range(H):
                    sel[t, h, :take] = np.sort(np.append(gen.choice(seen - 1, take - 1, replace=False), seen - 1))
                t += 1
        x["pages"] = dev(sel)
    return x


def _held(case, x, seed):
    """The keys and values that the cache holds before the step, in pieces: (k, v, slots)."""
    H, D, dtype = case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    g = _generator(seed, 2)
    piece = max(PAGE, (1 << 27) // (H * D) // PAGE * PAGE)
    for r, (p, _) in enumerate(x["lens"]):
        for a in range(0, p, piece):
            n = min(piece, p - a)
            k = torch.randn(n, H, D, device="cuda", generator=g, dtype=dtype) * x["gain"]
            v = torch.randn(n, H, D, device="cuda", generator=g, dtype=dtype)
            at = torch.arange(a, a + n, device="cuda")
            yield k, v, x["table"][r].long()[at // PAGE] * PAGE + at % PAGE


def prepare(case, seed):
    x = _inputs(case, seed)
    st = dict(x, case=case)
    H, D = case["kv_heads"], case["dim"]
    if own:
        from paper_2312_01712_amd import kv
        st["kv"] = kv
        st["out"] = kv.Step.empty(case["requests"], x["tokens"], x["table"])
        if case["op"] == "plan":
            return st
        cache = st["cache"] = kv.KvCache(x["n_pages"], H, D, TYPES[case["dtype"]])
        for k, v, slots in _held(case, x, seed):
            cache.append(k, v, slots)
        st["step"] = kv.plan(x["past"], x["new"], x["table"], x["free"], x["state"], out=st["out"])
        if case["op"] in ("select", "attention"):
            cache.append(x["k"], x["v"], st["step"].slots)
        if case["op"] == "append":
            st["rounded"] = torch.empty(x["k"].shape, dtype=x["k"].dtype, device="cuda"), torch.empty(
                x["v"].shape, dtype=x["v"].dtype, device="cuda")
        elif case["op"] == "select":
            st["work"] = cache.select_workspace(st["step"], case["heads"])
            st["to"] = torch.empty(x["tokens"], H, case["pages"], dtype=torch.int32, device="cuda")
        else:
            st["work"] = cache.attention_workspace(st["step"], case["heads"], max_new=case["new"], n_select=case["pages"])
            st["to"] = torch.empty(x["q"].shape, dtype=x["q"].dtype, device="cuda")
            st["lse"] = torch.empty(x["q"].shape[:2], dtype=torch.float32, device="cuda")
        return st
    if case["op"] == "plan":
        return st
    N = x["n_pages"]
    st["codes"] = torch.zeros(2, N * PAGE, H, D // 2, dtype=torch.uint8, device="cuda")
    st["scales"] = torch.zeros(2, N * PAGE, H, D // 32, dtype=torch.uint8, device="cuda")
    st["boxes"] = torch.zeros(N, H, 2, D, dtype=torch.bfloat16, device="cuda")
    for k, v, slots in _held(case, x, seed):
        _append_plain(st, k, v, slots)
    st["slots"] = _plan_plain(st)["slots"]
    if case["op"] in ("select", "attention"):
        _append_plain(st, x["k"], x["v"], st["slots"])
    return st


# ---- the plain forms ----------------------------------------------------------------------------


def _plan_plain(st):
    past, new, table, free, T = st["past"].long(), st["new"].long(), st["table"], st["free"], st["tokens"]
    R, W, ring = past.numel(), table.shape[1], free.numel()
    ends = new < 0
    n = new.clamp(min=0)
    total = torch.where(ends, 0, past + n)
    held = (past + PAGE - 1) // PAGE
    take = torch.where(ends, 0, (total + PAGE - 1) // PAGE - held)
    give = torch.where(ends, held, 0)
    took, gave, q_end = take.cumsum(0), give.cumsum(0), n.cumsum(0)
    head, tail = st["state"][0], st["state"][1]
    col = torch.arange(W, device="cuda")
    # pages that ended requests give back
    row, c = ((col < give[:, None])).nonzero(as_tuple=True)
    free[(tail + gave[row] - give[row] + c) % ring] = table[row, c]
    # pages that the others take, as far as they go
    row, c = ((col >= held[:, None]) & (col < (held + take)[:, None])).nonzero(as_tuple=True)
    i = took[row] - take[row] + c - held[row]
    table[row, c] = torch.where(i < tail - head, free[(head + i) % ring], -1)
    used = torch.minimum(took[-1], tail - head)
    state = torch.stack((head + used, tail + gave[-1], took[-1] - used))
    t = torch.arange(T, device="cuda")
    request = torch.searchsorted(q_end, t, right=True)
    position = past[request] + t - (q_end - n)[request]
    page = table[request, position // PAGE].long()
    slots = torch.where(page >= 0, page * PAGE + position % PAGE, -1)
    return dict(kv_lens=total.int(), q_start=torch.cat((q_end.new_zeros(1), q_end)).int(), slots=slots,
                requests=request.int(), positions=position.int(), state=state)


def _quantise_plain(x):
    """Codes (one a byte), scale bytes and the values that they stand for."""
    g = x.float().unflatten(-1, (-1, 32))
    b = ((g.abs().amax(-1, keepdim=True).view(torch.int32) >> 23) - 2).clamp(1, 254)
    y = g.abs() * ((254 - b) << 23).view(torch.float32)
    code = (y > 0.25).to(torch.uint8)
    for k, edge in enumerate((0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (y >= edge) if k % 2 == 0 else (y > edge)
    value = torch.tensor(GRID, device="cuda")[code.int()] * (b << 23).view(torch.float32)
    value = torch.where(g < 0, -value, value).flatten(-2)
    return (code | ((g < 0).to(torch.uint8) << 3)).flatten(-2), b.squeeze(-1).to(torch.uint8), value


def _append_plain(st, k, v, slots):
    rounded = []
    for i, x in enumerate((k, v)):
        code, scale, value = _quantise_plain(x)
        st["codes"][i, slots] = code[..., 0::2] | (code[..., 1::2] << 4)
        st["scales"][i, slots] = scale
        rounded.append(value)
        if i == 0:
            # pages whose first token is written start over, the others widen
            page, lane = slots // PAGE, slots % PAGE
            fresh = page[lane == 0]
            low, high = st["boxes"][:, :, 0].float(), st["boxes"][:, :, 1].float()
            low[fresh], high[fresh] = math.inf, -math.inf
            at = page[:, None, None].expand(value.shape)
            low.scatter_reduce_(0, at, value, "amin")
            high.scatter_reduce_(0, at, value, "amax")
            st["boxes"][:, :, 0], st["boxes"][:, :, 1] = low, high
    return rounded


def _values(st, which, pages):
    """The held values of the tokens of `pages`, [pages * 64][H][D] in 32 bits."""
    N, H, half = st["codes"].shape[1] // PAGE, st["codes"].shape[2], st["codes"].shape[3]
    code = st["codes"][which].view(N, PAGE, H, half)[pages].flatten(0, 1).int()
    scale = st["scales"][which].view(N, PAGE, H, -1)[pages].flatten(0, 1).int()
    code = torch.stack((code & 15, code >> 4), -1).flatten(-2)
    grid = torch.tensor(GRID + tuple(-x for x in GRID), device="cuda")
    return (grid[code].unflatten(-1, (-1, 32)) * (scale << 23).view(torch.float32)[..., None]).flatten(-2)


def _select_plain(st):
    case, q = st["case"], st["q"].float()
    H, G, n = case["kv_heads"], case["heads"] // case["kv_heads"], case["pages"]
    q = q.unflatten(1, (H, G))
    r = 127.0 / q.abs().amax((2, 3), keepdim=True)
    q = torch.round(q * torch.where(torch.isfinite(r), r, 0.0))
    out = torch.full((st["tokens"], H, n), -1, dtype=torch.int32, device="cuda")
    t = 0
    for i, (past, new) in enumerate(st["lens"]):
        P = _pages_of(past + new)
        box = st["boxes"][st["table"][i, :P].long()].float()                        # [P][H][2][D]
        e = (box.abs().amax((2, 3)).view(torch.int32) >> 23).clamp(min=8)           # [P][H]
        box = box * ((260 - e) << 23).view(torch.float32)[:, :, None, None]
        low, high = torch.floor(box[:, :, 0]), torch.ceil(box[:, :, 1])
        rows = q[t:t + new].permute(1, 0, 2, 3).flatten(1, 2)                       # [H][new * G][D]
        s = rows.clamp(min=0) @ high.permute(1, 2, 0).contiguous() + rows.clamp(max=0) @ low.permute(1, 2, 0).contiguous()
        s = s.unflatten(1, (new, G)).amax(2) * ((e - 6) << 23).view(torch.float32).t()[:, None]
        page = torch.arange(P, device="cuda")
        last = ((past + torch.arange(new, device="cuda")) // PAGE)[:, None]         # [new][1]
        s = torch.where((page == 0) | (page == last), math.inf, s)                  # the first page and the token's own
        s = torch.where(page > last, -math.inf, s)
        best = torch.sort(s, dim=-1, descending=True, stable=True)[1][..., :n]
        best = torch.where(best > last, P, best).sort(-1)[0]
        out[t:t + new, :, :best.shape[-1]] = torch.where(best == P, -1, best).permute(1, 0, 2).int()
        t += new
    return out


def _attention_plain(st):
    case, q = st["case"], st["q"].float()
    H, G, D = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"]
    q = q.unflatten(1, (H, G)) / math.sqrt(D)
    out, lse = torch.zeros_like(q), torch.empty(q.shape[:3], device="cuda")
    t = 0
    for i, (past, new) in enumerate(st["lens"]):
        pages = st["table"][i, :_pages_of(past + new)].long()
        k, v = _values(st, 0, pages), _values(st, 1, pages)
        key = torch.arange(k.shape[0], device="cuda")
        step = max(1, (1 << 29) // (k.shape[0] * G))
        for a in range(0, new, step):
            at = (past + torch.arange(a, min(a + step, new), device="cuda"))[:, None]
            for h in range(H):
                seen = key <= at
                if case["window"]:
                    seen &= key > at - case["window"]
                if case["pages"]:
                    mark = torch.zeros(at.shape[0], pages.numel() + 1, dtype=torch.bool, device="cuda")
                    mark.scatter_(1, st["pages"][t + a:t + a + at.shape[0], h].long() % (pages.numel() + 1), True)
                    seen &= mark[:, key // PAGE]
                rows = q[t + a:t + a + at.shape[0], h].flatten(0, 1)
                s = (rows @ k[:, h].t()).unflatten(0, (-1, G))
                s = torch.where(seen[:, None], s, -math.inf)
                top = s.amax(-1, keepdim=True)
                p = torch.exp(s - top)
                total = p.sum(-1, keepdim=True)
                out[t + a:t + a + at.shape[0], h] = ((p / total).flatten(0, 1) @ v[:, h]).unflatten(0, (-1, G))
                lse[t + a:t + a + at.shape[0], h] = (top + torch.log(total)).squeeze(-1)
        t += new
    return out.flatten(1, 2).to(st["q"].dtype), lse.flatten(1, 2)


def run(st):
    case = st["case"]
    if own:
        if case["op"] == "plan":
            step = st["kv"].plan(st["past"], st["new"], st["table"], st["free"], st["state"], out=st["out"])
            return [step.kv_lens, step.q_start, step.slots, step.requests, step.positions, step.free_state, st["table"], st["free"]]
        cache = st["cache"]
        if case["op"] == "append":
            cache.append(st["k"], st["v"], st["step"].slots, rounded=st["rounded"])
            return [*st["rounded"], cache.boxes]
        if case["op"] == "select":
            return [cache.select(st["q"], st["step"], case["pages"], sinks=1, recent=1, out=st["to"], workspace=st["work"])]
        return list(cache.attention(st["q"], st["step"], window=case["window"], pages=st.get("pages"), max_new=case["new"],
                                    out=st["to"], lse=st["lse"], workspace=st["work"]))
    if case["op"] == "plan":
        x = _plan_plain(st)
        return [x["kv_lens"], x["q_start"], x["slots"], x["requests"], x["positions"], x["state"], st["table"], st["free"]]
    if case["op"] == "append":
        k, v = _append_plain(st, st["k"], st["v"], st["slots"])
        return [k.to(st["k"].dtype), v.to(st["v"].dtype), st["boxes"]]
    if case["op"] == "select":
        return [_select_plain(st)]
    return list(_attention_plain(st))


# ---- from the definitions, in 64 bits -----------------------------------------------------------


def _nearest(x):
    """Held values of rows [...][D] in 64 bits: the nearest multiple on the grid, of two equally near the one with the even code."""
    g = x.double().unflatten(-1, (-1, 32))
    unit = torch.exp2(torch.floor(torch.log2(g.abs().amax(-1, keepdim=True).clamp(min=1e-30))) - 2)
    grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")
    y = g.abs() / unit
    best, far = torch.zeros_like(y), y.clone()
    for code in (2, 4, 6, 1, 3, 5, 7):
        d = (y - grid[code]).abs()
        best, far = torch.where(d < far, grid[code], best), torch.minimum(d, far)
    return (torch.copysign(best, g) * unit).flatten(-2)


def exact(case, seed):
    x = _inputs(case, seed)
    past, new, ring, W = x["past"].tolist(), x["new"].tolist(), x["free"].tolist(), x["width"]
    table = x["table"].cpu().numpy().copy()
    head, tail, _ = x["state"].tolist()
    q_start, total, slots, requests, positions, missing = [0], [], [], [], [], 0
    first_free, size, back = list(ring), len(ring), tail
    for r, (p, n) in enumerate(zip(past, new)):
        if n < 0:
            for c in range(-(-p // PAGE)):
                ring[back % size] = int(table[r, c])
                back += 1
        total.append(p + n if n >= 0 else 0)
        for c in range(-(-p // PAGE), -(-(p + n) // PAGE) if n >= 0 else 0):
            if head < tail:
                table[r, c] = first_free[head % size]
                head += 1
            else:
                table[r, c] = -1
                missing += 1
        for j in range(p, p + n):
            page = int(table[r, j // PAGE])
            slots.append(page * PAGE + j % PAGE if page >= 0 else -1)
            requests.append(r)
            positions.append(j)
        q_start.append(q_start[-1] + max(0, n))
    dev = lambda a, t: torch.from_numpy(np.array(a, dtype=t)).cuda()
    if case["op"] == "plan":
        return [dev(total, np.int32), dev(q_start, np.int32), dev(slots, np.int64), dev(requests, np.int32),
                dev(positions, np.int32), dev([head, back, missing], np.int64), dev(table, np.int32), dev(ring, np.int32)]
    H, G, D = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"]
    slots = dev(slots, np.int64)
    keys = torch.zeros(x["n_pages"] * PAGE, H, D, dtype=torch.float32, device="cuda")       # held values are short: nothing is lost
    values = torch.zeros_like(keys) if case["op"] == "attention" else None
    valid = torch.zeros(x["n_pages"] * PAGE, dtype=torch.bool, device="cuda")
    whole = ((k, v, s) for part in (_held(case, x, seed), [(x["k"], x["v"], slots)]) for k, v, s in part)
    for k, v, s in whole:
        for a in range(0, s.numel(), 8192):
            keys[s[a:a + 8192]] = _nearest(k[a:a + 8192]).float()
            if values is not None:
                values[s[a:a + 8192]] = _nearest(v[a:a + 8192]).float()
        valid[s] = True
    if case["op"] == "append":
        by_page, seen = keys.unflatten(0, (-1, PAGE)), valid.view(-1, PAGE, 1, 1)
        box = torch.stack((torch.where(seen, by_page, math.inf).amin(1), torch.where(seen, by_page, -math.inf).amax(1)), 2)
        box = torch.where(torch.isfinite(box), box, 0.0).double()
        return [_nearest(x["k"]), _nearest(x["v"]), box]
    if case["op"] == "select":
        return [_exact_pages(case, x, keys, valid, table)]
    out, lse = torch.zeros(x["tokens"], H * G, D, dtype=torch.float64, device="cuda"), None
    lse = torch.zeros(x["tokens"], H * G, dtype=torch.float64, device="cuda")
    t = 0
    for r, (p, n) in enumerate(x["lens"]):
        at = torch.arange(p + n, device="cuda")
        at = dev(table[r], np.int64)[at // PAGE] * PAGE + at % PAGE
        position = torch.arange(p, p + n, device="cuda")[:, None]
        distance = position - torch.arange(p + n, device="cuda")[None]
        for h in range(H):
            k, v = keys[at, h].double(), values[at, h].double()
            hidden = distance < 0
            if case["window"]:
                hidden |= distance >= case["window"]
            if case["pages"]:
                chosen = (x["pages"][t:t + n, h, :, None] == torch.arange(W, device="cuda", dtype=torch.int32)).any(1)
                hidden |= ~chosen[:, torch.arange(p + n, device="cuda") // PAGE]
            for g in range(G):
                s = x["q"][t:t + n, h * G + g].double() @ k.t() * D ** -0.5
                s.masked_fill_(hidden, -math.inf)
                lse[t:t + n, h * G + g] = torch.logsumexp(s, -1)
                out[t:t + n, h * G + g] = torch.softmax(s, -1) @ v
        t += n
    return [out, lse]


def _exact_pages(case, x, keys, valid, table):
    H, G, n = case["kv_heads"], case["heads"] // case["kv_heads"], case["pages"]
    out = np.full((x["tokens"], H, n), -1, dtype=np.int32)
    by_page, seen = keys.unflatten(0, (-1, PAGE)), valid.view(-1, PAGE, 1, 1)
    low = torch.where(seen, by_page, math.inf).amin(1)
    high = torch.where(seen, by_page, -math.inf).amax(1)
    t = 0
    for r, (p, new) in enumerate(x["lens"]):
        pages = torch.from_numpy(table[r, :_pages_of(p + new)].astype(np.int64)).cuda()
        lo, hi = low[pages].double(), high[pages].double()                              # [P][H][D]
        unit = torch.exp2(torch.floor(torch.log2(torch.maximum(lo.abs(), hi.abs()).amax(-1))) - 6)
        lo, hi = torch.floor(lo / unit[..., None]), torch.ceil(hi / unit[..., None])
        for j in range(new):
            q = x["q"][t].float().unflatten(0, (H, G))
            scale = 127.0 / q.abs().amax((1, 2), keepdim=True)                          # the rounding of the queries is 32-bit by definition
            q = torch.round(q * scale).double()
            bound = torch.stack([torch.maximum(q[:, g] * lo, q[:, g] * hi).sum(-1) for g in range(G)]).amax(0) * unit
            last = (p + j) // PAGE
            for h, s in enumerate(bound.t().cpu().numpy()):
                rest = [c for c in np.lexsort((np.arange(last + 1), -s[:last + 1])) if c not in (0, last)]
                chosen = sorted({0, last} | set(int(c) for c in rest[:n - len({0, last})]))
                out[t, h, :len(chosen)] = chosen
            t += 1
    return torch.from_numpy(out).cuda()
