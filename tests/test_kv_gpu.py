"""The paged 4-bit key/value cache on the GPU against its definitions in 64 bits (tests/kv_reference.py), through the
public calls of `paper_2312_01712_amd.kv`."""
import numpy as np
import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def kv():
    from paper_2312_01712_amd import kv as module
    assert torch.cuda.is_available()
    return module


def dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()


def rows(rng, dtype, *shape, spread=1.0):
    """Rows whose values are exact in the type, as a tensor and in 64 bits."""
    t = torch.from_numpy(rng.normal(size=shape) * spread).to(TYPES[dtype])
    return t.cuda(), t.double().numpy()


class Server:
    """A cache, its reference and the lengths of a few requests; `step` adds tokens to both."""

    def __init__(self, kv, rng, dtype, H, D, n_pages, R, W, ring_start=0, held=True):
        self.kv, self.rng, self.dtype, self.H, self.D, self.n_pages = kv, rng, dtype, H, D, n_pages
        self.cache = kv.KvCache(n_pages, H, D, TYPES[dtype])
        self.ref = ref.Cache(n_pages if held else 1, H, D)
        order = rng.permutation(n_pages)
        ring = np.empty(n_pages, np.int64)
        ring[(ring_start + np.arange(n_pages)) % n_pages] = order
        self.past, self.table, self.ring = np.zeros(R, np.int64), np.full((R, W), -1, np.int64), ring
        self.state = np.array([ring_start, ring_start + n_pages, 0], np.int64)
        self.d_past, self.d_table, self.d_ring = dev(self.past, torch.int32), dev(self.table, torch.int32), dev(ring, torch.int32)
        self.d_state = dev(self.state, torch.int64)
        # per head and channel, some channels large as in trained models
        self.gain = np.exp(rng.normal(size=(H, D)) * 0.7)

    def plan(self, new, max_tokens=None):
        new = np.asarray(new, np.int64)
        T = int(np.maximum(new, 0).sum()) if max_tokens is None else max_tokens
        self.want = ref.plan(self.past, new, self.table, self.ring, self.state, T)
        self.step = self.kv.plan(self.d_past, dev(new, torch.int32), self.d_table, self.d_ring, self.d_state, max_tokens=T)
        w = self.want
        for name, got in (("kv_lens", self.step.kv_lens), ("q_start", self.step.q_start), ("slots", self.step.slots),
                          ("requests", self.step.requests), ("positions", self.step.positions), ("state", self.step.free_state),
                          ("table", self.d_table), ("ring", self.d_ring)):
            assert np.array_equal(got.cpu().numpy().astype(np.int64), w[name]), name
        self.past, self.table, self.ring, self.state = w["kv_lens"], w["table"], w["ring"], w["state"]
        self.d_past, self.d_state = self.step.kv_lens, self.step.free_state
        return T

    def fill(self, new, max_tokens=None, edit=None):
        T = self.plan(new, max_tokens)
        k, kn = rows(self.rng, self.dtype, T, self.H, self.D)
        k = (k * dev(self.gain, TYPES[self.dtype])).contiguous()
        v, vn = rows(self.rng, self.dtype, T, self.H, self.D)
        if edit is not None:
            edit(k, v)
        kr, vr = torch.zeros_like(k), torch.zeros_like(v)
        self.cache.append(k, v, self.step.slots, rounded=(kr, vr))
        wk, wv = self.ref.append(k.double().cpu().numpy(), v.double().cpu().numpy(), self.want["slots"])
        at = self.want["slots"] >= 0
        assert np.array_equal(kr.double().cpu().numpy()[at], wk[at], equal_nan=True)
        assert np.array_equal(vr.double().cpu().numpy()[at], wv[at])
        assert np.array_equal(self.cache.boxes.double().cpu().numpy(), self.ref.boxes)
        return T

    def attend(self, heads, window=0, selected=None, scale=None, max_new=None, q=None, check=True):
        T = len(self.want["positions"])
        if q is None:
            q, qn = rows(self.rng, self.dtype, T, heads, self.D)
        else:
            qn = q.double().cpu().numpy()
        sc = self.D ** -0.5 if scale is None else scale
        out, lse = self.cache.attention(q, self.step, scale=scale, window=window, max_new=max_new,
                                        pages=None if selected is None else dev(selected, torch.int32))
        want = ref.attention(self.ref, qn, self.H, self.want, self.n_pages, sc, window, selected)
        compare(out, lse, *want, self.D, self.dtype == "fp16")
        return out, lse


def compare(out, lse, w_out, w_lse, mass, reach, size, D, fp16):
    o, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    off, off_lse = ref.bounds(w_out, w_lse, mass, reach, size, D, fp16)
    assert np.array_equal(np.isnan(o), np.isnan(w_out)) and np.array_equal(np.isnan(l), np.isnan(w_lse))
    assert np.array_equal(np.isneginf(l), np.isneginf(w_lse))
    fine = np.isfinite(w_out)
    bad = np.abs(o - w_out)[fine] > off[fine]
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, by {(np.abs(o - w_out)[fine] / np.maximum(off[fine], 1e-300)).max():.2f} bounds"
    fine = np.isfinite(w_lse)
    assert (np.abs(l - w_lse)[fine] <= off_lse[fine]).all()
    assert (o[np.isneginf(w_lse)] == 0).all()


# ---- page tables ------------------------------------------------------------------------------------


@pytest.mark.parametrize("R,longest,new,seed", [(1, 0, 1, 0), (1, 5, 200, 1), (7, 300, 70, 2), (63, 200, 3, 3), (64, 200, 40, 4),
                                                (65, 1000, 9, 5), (700, 500, 2, 6), (3, 100, 5000, 7)])
def test_plan_over_steps(kv, R, longest, new, seed):
    """Steps in a row: requests grow, end and start again, the ring goes round, rows without a token at the end."""
    rng = np.random.default_rng(seed)
    W = (longest + 6 * new) // 64 + 2
    n_pages = int(R * W * 0.8) + 3
    s = Server(kv, rng, "bf16", 1, 64, n_pages, R, W, ring_start=n_pages - 2)
    first = rng.integers(0, longest + 1, R)
    s.plan(first, max_tokens=int(first.sum()) + 5)
    for i in range(4):
        n = rng.integers(0, new + 1, R)
        n[rng.random(R) < 0.15] = -1
        s.plan(n, max_tokens=int(np.maximum(n, 0).sum()) + int(rng.integers(0, 200)))


def test_plan_without_enough_pages(kv):
    """Pages run out in the middle of a request: -1 in the table, slots -1, the shortfall counted; such tokens are neither
    stored nor seen."""
    rng = np.random.default_rng(8)
    s = Server(kv, rng, "bf16", 2, 64, 5, 4, 4)
    s.fill([100, 60, 200, 70])
    assert s.state[2] == 4 and (s.want["slots"] < 0).sum() > 0
    s.attend(4)


def test_plan_cuts_at_the_tables_width(kv):
    rng = np.random.default_rng(9)
    s = Server(kv, rng, "bf16", 1, 64, 20, 3, 2)
    s.fill([130, 64, 129])
    assert (s.past == [128, 64, 128]).all()
    s.attend(2)


def test_plan_of_no_requests(kv):
    s = kv.plan(*(torch.zeros(0, dtype=torch.int32, device="cuda"),) * 2, torch.zeros(0, 3, dtype=torch.int32, device="cuda"),
                torch.zeros(4, dtype=torch.int32, device="cuda"), torch.tensor([0, 4, 0], device="cuda"), max_tokens=3)
    assert s.slots.tolist() == [-1] * 3 and s.q_start.tolist() == [0] and s.free_state.tolist() == [0, 4, 0]
    cache = kv.KvCache(4, 2, 64)
    q = torch.randn(3, 4, 64, device="cuda").bfloat16()
    out, lse = cache.attention(q, s)
    assert (out == 0).all() and torch.isneginf(lse).all()
    assert (cache.select(q, s, 2) == -1).all()


# ---- append -----------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,D", [(1, 64), (3, 96), (2, 128), (2, 256)])
def test_append_token_by_token_and_at_once(kv, dtype, H, D):
    """Prompts of every remainder, then single tokens, then a few at a time: pages that are begun, widened and crossed; the
    bytes and boxes are the same as those of one call."""
    rng = np.random.default_rng(D + H)
    s = Server(kv, rng, dtype, H, D, 40, 6, 6)
    s.fill([0, 1, 63, 64, 65, 130], max_tokens=340)
    for new in ([1] * 6, [1] * 6, [3, 0, 2, 5, 1, 66], [7, 70, 4, 1, 128, 2]):
        s.fill(new)
    s.attend(2 * H)
    again = kv.KvCache(40, H, D, TYPES[dtype])
    total = int(s.past.sum())
    slots = np.concatenate([s.table[r, np.arange(n) // 64] * 64 + np.arange(n) % 64 for r, n in enumerate(s.past)])
    k, v = (dev(x[slots], TYPES[dtype]) for x in (s.ref.k, s.ref.v))
    assert total == len(slots)
    again.append(k, v, dev(slots, torch.int64))
    assert torch.equal(again.boxes, s.cache.boxes)
    # a second rounding of held values changes nothing, so the pages agree up to the sign of zeros and the unit of groups
    # whose largest value rounded down; what they stand for is compared through attention
    held, s.cache = s.cache, again
    s.attend(2 * H)
    s.cache = held


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_append_rounding_of_every_value(kv, dtype):
    """All finite values of the type, each with companions that set its unit: ties, zeros, the smallest and the largest."""
    bits = torch.arange(0, 1 << 16, dtype=torch.int32)
    x = bits.to(torch.int16).view(TYPES[dtype])
    x = x[torch.isfinite(x)].double().numpy()
    tops = np.array([6.0, 1.0, 1.5, 1.75, 1.9375]) if dtype == "fp16" else np.array([6.0, 1.0, 1.5, 1.75, 1.9375, 2.0 ** 100, 2.0 ** -100])
    x = np.concatenate([x, *[t * np.linspace(-1, 1, 333) for t in tops]])
    x = np.concatenate([x, np.zeros(-len(x) % 64)])
    rng = np.random.default_rng(3)
    x = np.concatenate([x, rng.permutation(x)]).reshape(-1, 1, 64)
    x = torch.from_numpy(x).to(TYPES[dtype])
    n = x.shape[0] // 64 * 64
    x = x[:n].cuda()
    cache = kv.KvCache(n // 64, 1, 64, TYPES[dtype])
    kr, vr = torch.empty_like(x), torch.empty_like(x)
    cache.append(x, x.flip(0).contiguous(), torch.arange(n, device="cuda"), rounded=(kr, vr))
    want = ref.quantise(x.double().cpu().numpy())[2]
    # what the type itself cannot hold (fp16 below 2^-24) is rounded once more
    want = torch.from_numpy(want).to(TYPES[dtype])
    assert torch.equal(kr.cpu(), want)
    assert torch.equal(vr.cpu(), want.flip(0))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_tokens_that_are_not_finite(kv, dtype):
    """Infinities and NaN in a key or a value: the rows that see the token are NaN, the others are as if it were not there, also
    within one tile and with a window that has left it behind."""
    rng = np.random.default_rng(12)
    s = Server(kv, rng, dtype, 2, 128, 12, 2, 5)

    def edit(k, v):
        k[70, 0, 5] = float("nan")
        k[75, 1, 127] = float("-inf")
        v[80, 0, 64] = float("inf")
        v[3, 1, 0] = float("nan")
    s.fill([90, 40], edit=edit)
    out, _ = s.attend(6)
    assert out.isnan().any() and not out.isnan().all()
    s.attend(6, window=5)
    s.fill([1, 1])
    s.attend(6, window=9)


def test_append_leaves_out_slots_outside(kv):
    cache = kv.KvCache(2, 1, 64)
    k = torch.ones(5, 1, 64, device="cuda").bfloat16()
    slots = torch.tensor([-1, 128, 1 << 40, -(1 << 40), 64], device="cuda")
    cache.append(k, k, slots)
    assert (cache.boxes[0] == 0).all() and (cache.boxes[1] == 1).all() and (cache.pages[0] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rows_of_a_projection(kv, dtype):
    """Queries, keys and values as views of one tensor, results into a view: strides of tokens and heads."""
    rng = np.random.default_rng(13)
    s = Server(kv, rng, dtype, 2, 96, 8, 2, 4)
    T = s.plan([70, 9])
    packed, _ = rows(rng, dtype, 6 + 2 + 2, T, 96 + 8)      # heads first, padded rows
    packed = packed.transpose(0, 1)[..., :96]
    q, k, v = packed[:, :6], packed[:, 6:8], packed[:, 8:]
    s.cache.append(k, v, s.step.slots)
    s.ref.append(k.double().cpu().numpy(), v.double().cpu().numpy(), s.want["slots"])
    out = torch.full((T, 2, 6, 96), 7.0, dtype=TYPES[dtype], device="cuda")
    o, lse = s.cache.attention(q, s.step, out=out[:, 1])
    want = ref.attention(s.ref, q.double().cpu().numpy(), 2, s.want, 8, 96 ** -0.5)
    compare(o, lse, *want, 96, dtype == "fp16")
    assert (out[:, 0] == 7).all()
    sel = s.cache.select(q, s.step, 1, sinks=0, recent=1)
    assert np.array_equal(sel.cpu().numpy(), ref.select(s.ref, q.double().cpu().numpy(), 2, s.want, 8, 1, 0, 1))


# ---- selection --------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,D,new,n,sinks,recent", [(1, 1, 64, [1, 1, 1], 3, 1, 1), (2, 3, 96, [1, 5, 2], 4, 0, 2),
                                                       (2, 4, 128, [1, 1, 1], 5, 2, 0), (1, 8, 128, [9, 1, 4], 1, 0, 0),
                                                       (1, 20, 64, [1, 3, 1], 6, 1, 1), (2, 16, 256, [1, 2, 1], 7, 3, 4),
                                                       (1, 40, 128, [2, 1, 1], 4, 1, 1), (3, 2, 128, [70, 1, 13], 2, 1, 1)])
def test_select(kv, dtype, H, G, D, new, n, sinks, recent):
    rng = np.random.default_rng(H * G + D)
    s = Server(kv, rng, dtype, H, D, 60, 3, 25)
    s.fill([64 * 19 + 5, 64 * 7, 10])
    s.fill(new, max_tokens=sum(new) + 3)
    q, qn = rows(rng, dtype, sum(new) + 3, H * G, D)
    got = s.cache.select(q, s.step, n, sinks=sinks, recent=recent).cpu().numpy()
    want = ref.select(s.ref, qn, H, s.want, 60, n, sinks, recent)
    assert np.array_equal(got, want)
    s.attend(H * G, selected=got.astype(np.int64))


def test_select_many_columns_and_equal_scores(kv):
    """Thousands of columns; boxes that repeat, so that many scores are equal (lower columns win), zeros among the
    queries, and columns without a page."""
    rng = np.random.default_rng(21)
    H, D, P, n = 2, 64, 5000, 300
    cache = kv.KvCache(P, H, D)
    some = rng.integers(-6, 7, (9, H, 2, D)).astype(np.float64)
    lo, hi = np.minimum(some[:, :, 0], some[:, :, 1]), np.maximum(some[:, :, 0], some[:, :, 1])
    boxes = np.stack([lo, hi], 2)[rng.integers(0, 9, P)]
    boxes[::17] = 0
    cache.boxes.copy_(dev(boxes, torch.bfloat16))
    table = rng.permutation(P).reshape(1, P)
    table[0, 40:60] = -1
    table[0, 100] = P
    T = 3
    want = dict(kv_lens=np.array([P * 64 - 1]), table=table, requests=np.zeros(T, np.int64),
                positions=np.array([P * 64 - 4, P * 64 - 3, P * 64 - 2]), q_start=np.array([0, T]))
    step = kv.Step(dev(want["kv_lens"], torch.int32), dev(want["q_start"], torch.int32), dev(table, torch.int32),
                   torch.zeros(T, dtype=torch.int64, device="cuda"), dev(want["requests"], torch.int32),
                   dev(want["positions"], torch.int32), torch.zeros(3, dtype=torch.int64, device="cuda"))
    q, qn = rows(rng, "bf16", T, 3 * H, D)
    q[1] = 0
    q[2, :3, 7] = float("nan")
    q[2, 3:, 9] = float("inf")
    qn = q.double().cpu().numpy()
    ref_cache = ref.Cache(1, H, D)
    ref_cache.boxes = boxes
    got = cache.select(q, step, n).cpu().numpy()
    assert np.array_equal(got, ref.select(ref_cache, qn, H, want, P, n, 1, 1))


# ---- attention --------------------------------------------------------------------------------------


SHAPES = [(1, 1, 64), (2, 4, 96), (2, 8, 128), (1, 5, 256), (1, 24, 64), (1, 3, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,D", SHAPES)
def test_attention_single_tokens(kv, dtype, H, G, D):
    """Decode: contexts of 1, 63, 64, 65 and some hundred tokens, one that ends inside a page; whole, windowed, and with a
    scale of nothing."""
    rng = np.random.default_rng(D + G)
    s = Server(kv, rng, dtype, H, D, 60, 7, 20)
    s.fill([0, 62, 63, 64, 65, 400, 1000])
    s.fill([1] * 7, max_tokens=9)
    s.attend(H * G, max_new=1)
    s.attend(H * G, max_new=1, window=1)
    s.attend(H * G, max_new=1, window=100)
    s.attend(H * G, max_new=1, scale=0.0)
    s.attend(H * G, max_new=1, scale=-0.3)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,D", SHAPES)
def test_attention_chunks(kv, dtype, H, G, D):
    """Chunks of several requests, some without new tokens, over what they hold; windows that end inside pages and chunks."""
    rng = np.random.default_rng(D * G)
    s = Server(kv, rng, dtype, H, D, 60, 5, 20)
    s.fill([0, 130, 64, 7, 500])
    s.fill([150, 33, 0, 65, 5], max_tokens=260)
    s.attend(H * G)
    s.attend(H * G, max_new=150, window=1)
    s.attend(H * G, max_new=150, window=64)
    s.attend(H * G, max_new=150, window=131)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,D", SHAPES)
def test_attention_shares_across_requests(kv, dtype, H, G, D):
    """Tables wide enough that workgroups have shares of all requests' pages: shares that begin and end inside requests,
    heads and tiles, requests of one page between long ones, some without new tokens."""
    rng = np.random.default_rng(D * G + 1)
    s = Server(kv, rng, dtype, H, D, 150, 6, 50)
    s.fill([0, 2900, 5, 64, 1300, 700])
    s.fill([1, 1, 0, 1, 1, 1], max_tokens=7)
    s.attend(H * G, max_new=1)
    s.attend(H * G, max_new=1, window=700)
    s.fill([70, 33, 0, 129, 1, 5], max_tokens=240)
    s.attend(H * G)
    s.attend(H * G, window=300)
    s.attend(H * G, max_new=1)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention_long_context_is_split(kv, dtype):
    """One request long enough that many workgroups share its pages."""
    rng = np.random.default_rng(31)
    s = Server(kv, rng, dtype, 1, 128, 300, 2, 300)
    s.fill([18001, 3])
    s.fill([1, 1])
    s.attend(4, max_new=1)
    s.attend(4, max_new=1, window=9000)
    s.fill([21, 2])
    s.attend(4, max_new=21)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,D", [(2, 4, 128), (1, 20, 64), (3, 1, 96), (1, 2, 256)])
def test_attention_selected(kv, dtype, H, G, D):
    """Lists in any order, empty ones, -1 between the columns, columns in the future and outside the table."""
    rng = np.random.default_rng(G)
    s = Server(kv, rng, dtype, H, D, 60, 4, 30)
    s.fill([1500, 64, 0, 300])
    s.fill([2, 1, 3, 1], max_tokens=9)
    T, n = 9, 7
    sel = np.full((T, H, n), -1, np.int64)
    for t in range(T):
        for h in range(H):
            some = rng.permutation(26)[:rng.integers(0, n + 1)]
            sel[t, h, rng.permutation(n)[:len(some)]] = some
    sel[0, 0] = -1
    sel[1, 0, 0], sel[3, 0, 1] = 29, 40
    s.attend(H * G, selected=sel)
    s.attend(H * G, selected=sel, window=90)


@pytest.mark.parametrize("n", [20, 40, 64, 70])
def test_attention_of_many_selections(kv, n):
    """Lists short enough for a workgroup each and longer ones, of many tokens and heads."""
    rng = np.random.default_rng(n)
    s = Server(kv, rng, "bf16", 4, 64, 500, 6, 90)
    s.fill([5000, 640, 0, 4200, 64, 2500])
    s.fill([9, 4, 3, 7, 8, 5], max_tokens=37)
    q, qn = rows(rng, "bf16", 37, 8, 64)
    got = s.cache.select(q, s.step, n, sinks=2, recent=1).cpu().numpy().astype(np.int64)
    assert np.array_equal(got, ref.select(s.ref, qn, 4, s.want, 500, n, 2, 1))
    s.attend(8, selected=got)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention_of_large_scores(kv, dtype):
    """Scores of hundreds and thousands, of both signs: the running maximum moves by more than exponentials hold."""
    rng = np.random.default_rng(41)
    s = Server(kv, rng, dtype, 1, 64, 20, 2, 10)
    s.gain = s.gain * 20
    s.fill([400, 100])
    s.fill([3, 1])
    s.attend(2, scale=2.0)
    s.attend(2, scale=-2.0)


def test_infinite_and_nan_queries_stay_in_their_rows(kv):
    rng = np.random.default_rng(42)
    s = Server(kv, rng, "bf16", 1, 128, 20, 2, 10)
    s.fill([200, 70])
    s.fill([4, 1])
    q, _ = rows(rng, "bf16", 5, 4, 128)
    clean, clean_lse = s.cache.attention(q, s.step)
    q2 = q.clone()
    q2[1, 2, 9] = float("nan")
    q2[4, 0, 3] = float("inf")
    out, lse = s.cache.attention(q2, s.step)
    hit = torch.zeros(5, 4, dtype=torch.bool, device="cuda")
    hit[1, 2] = hit[4, 0] = True
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])


def test_memory_that_no_token_wrote(kv):
    """Pages full of ones (scales that are not numbers) before the tokens come: nothing of them reaches a result."""
    rng = np.random.default_rng(43)
    for dtype in TYPES:
        s = Server(kv, rng, dtype, 2, 128, 12, 3, 5)
        s.cache.pages.fill_(255)
        s.fill([1, 70, 130])
        s.attend(8)
        s.fill([1, 1, 1])
        s.attend(8, max_new=1)


def test_pages_behind_32_bits(kv):
    """A cache of more than 4 GiB: pages at its end."""
    rng = np.random.default_rng(44)
    s = Server(kv, rng, "bf16", 8, 128, 70000, 2, 8, held=False)
    assert s.cache.pages.numel() > 1 << 32
    s.ring[:16] = np.arange(69999, 69983, -1)
    s.ring[16:69984 + 16] = np.arange(69984)
    s.d_ring = dev(s.ring, torch.int32)
    T = s.plan([200, 70])
    assert s.table[0, 0] == 69999
    k, _ = rows(rng, "bf16", T, 8, 128)
    v, _ = rows(rng, "bf16", T, 8, 128)
    s.cache.append(k, v, s.step.slots)
    low = int(s.want["slots"].min()) // 64
    s.ref = ref.Cache(70000 - low, 8, 128)
    s.ref.append(k.double().cpu().numpy(), v.double().cpu().numpy(), s.want["slots"] - low * 64)
    q, qn = rows(rng, "bf16", T, 8, 128)
    out, lse = s.cache.attention(q, s.step)
    moved = dict(s.want, table=np.where(s.want["table"] >= low, s.want["table"] - low, -1))
    compare(out, lse, *ref.attention(s.ref, qn, 8, moved, 70000 - low, 128 ** -0.5), 128, False)
    sel = s.cache.select(q, s.step, 2)
    assert np.array_equal(sel.cpu().numpy(), ref.select(s.ref, qn, 8, moved, 70000 - low, 2, 1, 1))


def test_more_requests_than_are_scanned_in_a_workgroup(kv):
    rng = np.random.default_rng(45)
    R = 2300
    s = Server(kv, rng, "bf16", 1, 64, 2600, R, 2)
    s.fill(rng.integers(0, 9, R))
    s.attend(1)
    s.fill(np.ones(R, np.int64))
    s.attend(2, max_new=1)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,W", [(64, 60), (128, 60), (96, 30)])
def test_attention_of_many_rows(kv, dtype, D, W):
    """Enough rows for the largest tiles: prompts of many requests at once, some behind what they hold; odd numbers of
    pages, pages that are missing in the middle of a request."""
    rng = np.random.default_rng(D)
    R = 31
    s = Server(kv, rng, dtype, 1, D, 420, R, W)
    s.fill(rng.integers(0, 90, R))
    new = rng.integers(1, 140, R)
    new[3], new[4] = 500, 0
    s.fill(new, max_tokens=int(new.sum()) + 2)
    assert new.sum() * 32 >= 256 * 256
    for at in ((3, 1), (3, 4), (8, 0)):  # holes in the tables
        s.table[at] = -1
    s.want["table"] = s.table
    s.d_table.copy_(dev(s.table, torch.int32))
    s.attend(32)


@pytest.mark.parametrize("max_new", [1, 3, 17, 64, 1000])
def test_the_hint_does_not_change_what_is_computed(kv, max_new):
    """max_new only chooses how the work is cut; below the truth too."""
    rng = np.random.default_rng(46)
    s = Server(kv, rng, "bf16", 2, 128, 40, 3, 20)
    s.fill([300, 0, 64])
    s.fill([40, 90, 1])
    s.attend(8, max_new=max_new)


def test_streams_and_graphs(kv):
    """The whole step on a stream of its own and in a graph whose replays continue: a request grows token by token."""
    rng = np.random.default_rng(47)
    H, G, D = 2, 4, 128
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s = Server(kv, rng, "bf16", H, D, 20, 2, 8)
        s.fill([60, 10])
        s.fill([1, 1])
        s.attend(H * G, max_new=1)
        past, state = s.d_past.clone(), s.d_state.clone()
        step = kv.Step.empty(2, 2, s.d_table)
        one = torch.ones(2, dtype=torch.int32, device="cuda")
        q, k, v = (rows(rng, "bf16", 2, h, D)[0] for h in (H * G, H, H))
        ws, out = s.cache.attention_workspace(step, H * G, max_new=1), torch.empty_like(q)
        lse = torch.empty(2, H * G, device="cuda")
        sel, sel_ws = torch.empty(2, H, 3, dtype=torch.int32, device="cuda"), s.cache.select_workspace(step, H * G)

        def whole():
            kv.plan(past, one, s.d_table, s.d_ring, state, out=step)
            s.cache.append(k, v, step.slots)
            s.cache.select(q, step, 3, out=sel, workspace=sel_ws)
            s.cache.attention(q, step, max_new=1, out=out, lse=lse, workspace=ws)
            past.copy_(step.kv_lens)
            state.copy_(step.free_state)
        s.cache.select(q, s.step, 3)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            whole()
        for i in range(6):
            kn, vn, qn = (x.double().cpu().numpy() for x in (k, v, q))
            want = ref.plan(s.past, [1, 1], s.table, s.ring, s.state, 2)
            s.ref.append(kn, vn, want["slots"])
            graph.replay()
            side.synchronize()
            assert np.array_equal(step.slots.cpu().numpy(), want["slots"])
            compare(out, lse, *ref.attention(s.ref, qn, H, want, 20, D ** -0.5), D, False)
            assert np.array_equal(sel.cpu().numpy(), ref.select(s.ref, qn, H, want, 20, 3, 1, 1))
            s.past, s.table, s.ring, s.state = want["kv_lens"], want["table"], want["ring"], want["state"]
            for x in (k, v, q):
                x.copy_(torch.randn(x.shape, device="cuda"))
            side.synchronize()


def test_the_same_call_gives_the_same_bits(kv):
    rng = np.random.default_rng(48)
    s = Server(kv, rng, "bf16", 2, 128, 300, 3, 200)
    s.fill([9000, 64, 1000])
    s.fill([1, 1, 1])
    q, _ = rows(rng, "bf16", 3, 8, 128)
    first = s.cache.attention(q, s.step, max_new=1)
    for _ in range(5):
        again = s.cache.attention(q, s.step, max_new=1)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ---- refusals ---------------------------------------------------------------------------------------


def test_refusals(kv):
    rng = np.random.default_rng(50)
    s = Server(kv, rng, "bf16", 2, 64, 8, 2, 4)
    s.fill([5, 7])
    q, _ = rows(rng, "bf16", 12, 4, 64)
    from paper_2312_01712_amd.binding import ERR_INVALID_ARGUMENT, ERR_WORKSPACE, IvfpqError
    for call in (lambda: s.cache.attention(q.half(), s.step), lambda: s.cache.attention(q.cpu(), s.step),
                 lambda: s.cache.attention(q[:11], s.step), lambda: s.cache.attention(q[..., ::2], s.step),
                 lambda: s.cache.attention(q, s.step, pages=torch.zeros(12, 2, 0, dtype=torch.int32, device="cuda")),
                 lambda: s.cache.attention(q, s.step, pages=torch.zeros(12, 3, 1, dtype=torch.int32, device="cuda")),
                 lambda: s.cache.append(q, q, s.step.slots), lambda: s.cache.append(q[:, :2], q[:, :2], s.step.slots[:5]),
                 lambda: s.cache.append(q[:, :2], q[:, :2], s.step.slots.int()),
                 lambda: kv.KvCache(0, 1, 64), lambda: kv.KvCache(1, 1, 80), lambda: kv.KvCache(1, 0, 64),
                 lambda: kv.KvCache(1, 1, 64, torch.float32),
                 lambda: kv.plan(s.d_past, s.d_past, s.d_table, s.d_ring, s.d_state),
                 lambda: kv.plan(s.d_past[:1], s.d_past, s.d_table, s.d_ring, s.d_state, max_tokens=3),
                 lambda: kv.plan(s.d_past, s.d_past, s.d_table, s.d_ring, s.d_state, max_tokens=3, out=s.step)):
        with pytest.raises(ValueError):
            call()
    odd = torch.zeros(12 * 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    for call, status in (
            (lambda: s.cache.attention(q[:, :3], s.step), ERR_INVALID_ARGUMENT),
            (lambda: s.cache.attention(q, s.step, window=-1), ERR_INVALID_ARGUMENT),
            (lambda: s.cache.attention(q, s.step, scale=float("nan")), ERR_INVALID_ARGUMENT),
            (lambda: s.cache.attention(q, s.step, max_new=0, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), ERR_INVALID_ARGUMENT),
            (lambda: s.cache.attention(q, s.step, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), ERR_WORKSPACE),
            (lambda: s.cache.attention(odd[4:4 + 12 * 256].view(12, 4, 64), s.step), ERR_INVALID_ARGUMENT),
            (lambda: s.cache.attention(odd[:12 * 256 + 4].as_strided((12, 4, 64), (255, 64, 1)), s.step), ERR_INVALID_ARGUMENT),
            (lambda: s.cache.select(q, s.step, 0), ERR_INVALID_ARGUMENT),
            (lambda: s.cache.select(q, s.step, 1025), ERR_INVALID_ARGUMENT),
            (lambda: s.cache.select(q, s.step, 2, sinks=2, recent=1), ERR_INVALID_ARGUMENT),
            (lambda: s.cache.select(q, s.step, 2, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), ERR_WORKSPACE)):
        with pytest.raises(IvfpqError) as e:
            call()
        assert e.value.status == status, e.value
    torch.cuda.synchronize()


def test_the_example_runs(kv):
    """examples/kv_decode.py, small: all operators together; looking at every page is attention over everything."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import kv_decode
    whole, part = kv_decode.main(["--requests", "3", "--prompt", "300", "--steps", "3", "--pages", "8"])
    assert torch.isfinite(whole).all()
    # the same keys in another order of sums: within a few units of the weights' and results' rounding
    assert (whole - part).float().abs().max() <= 2.0 ** -5 * whole.float().abs().max()
