"""Decoding with drafted tokens over the paged 4-bit cache on the GPU, against its definitions in 64 bits (tests/kv_tree_reference.py),
through the public calls of `paper_2312_01712_amd.kv`."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import kv_tree_reference as tref
from test_kv_gpu import TYPES, Server, compare, dev, kv, rows  # noqa: F401

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def random_parents(rng, new, roots=0.0):
    """Parents of every request's tokens: the first is a root, others hang on an earlier one (or, rarely, on none)."""
    parts = []
    for n in np.maximum(new, 0):
        p = np.floor(rng.random(n) * np.arange(n)).astype(np.int64)
        p[rng.random(n) < roots] = -1
        if n:
            p[0] = -1
        parts.append(p)
    return np.concatenate(parts + [np.zeros(0, np.int64)])


class TreeServer(Server):
    """`draft` appends a step's drafted tokens, `attend_tree` compares their attention, `keep` what stays of them."""

    def draft(self, new, max_tokens=None, parents=None, max_nodes=None, window=0, roots=0.0, edit=None):
        self.before = self.past
        T = self.fill(new, max_tokens, edit)
        p = random_parents(self.rng, np.asarray(new), roots) if parents is None else np.asarray(parents)
        self.parents = np.concatenate((p, np.full(T - len(p), 7)))
        N = max(1, int(np.max(new))) if max_nodes is None else max_nodes
        self.tree = self.kv.tree(dev(self.parents, torch.int32), self.step, max_nodes=N, window=window)
        self.sees, self.positions = tref.tree(self.parents, self.want, N, window)
        assert np.array_equal(self.tree.masks.cpu().numpy(), tref.words(self.sees))
        assert np.array_equal(self.tree.positions.cpu().numpy(), self.positions)
        return T

    def attend_tree(self, heads, scale=None, q=None, tree=None):
        T = len(self.want["positions"])
        q, qn = rows(self.rng, self.dtype, T, heads, self.D) if q is None else (q, q.double().cpu().numpy())
        tree = self.tree if tree is None else tree
        sc = self.D ** -0.5 if scale is None else scale
        out, lse = self.cache.tree_attention(q, self.step, tree, scale=sc)
        want = tref.attention(self.ref, qn, self.H, self.want, self.sees, self.positions, self.n_pages, sc, tree.window)
        compare(out, lse, *want, self.D, self.dtype == "fp16")
        return out, lse

    def keep(self, agree=0.7, drafted=None, picked=None, more=()):
        """`agree`: how likely the model agrees with a request's deepest path, and not with one to any of its tokens.  more: (cache,
        reference) of further layers."""
        T = len(self.want["positions"])
        if drafted is None:
            drafted, picked = self.rng.integers(0, 1000, T), self.rng.integers(1000, 2000, T)
            start = self.want["q_start"]
            for a, b in zip(start, start[1:]):
                if b > a:
                    paths = [tref.ancestors(self.parents[a:b], i)[::-1] for i in range(b - a)]
                    path = max(paths, key=len) if self.rng.random() < agree else paths[self.rng.integers(b - a)]
                    picked[a + np.array(path[:-1], int)] = drafted[a + np.array(path[1:], int)]
        lens, kept, ring, state = tref.keep([self.ref] + [m[1] for m in more], self.want, self.sees, drafted, picked, self.ring,
                                            self.state, self.n_pages)
        got = self.kv.keep([self.cache] + [m[0] for m in more], self.step, self.tree, dev(drafted, torch.int32), dev(picked, torch.int32),
                           self.d_ring, self.d_state)
        for name, x, w in (("lens", got.lens, lens), ("rows", got.rows, kept), ("ring", self.d_ring, ring), ("state", got.free_state, state)):
            assert np.array_equal(x.cpu().numpy().astype(np.int64), w), name
        self.past, self.ring, self.state = lens, ring, state
        self.d_past, self.d_state = got.lens, got.free_state
        for c, r in [(self.cache, self.ref), *more]:
            self.check_held(c, r)
        return kept

    def check_held(self, cache, reference):
        """Every held token's values, and the boxes of the pages that hold some."""
        slots, pages = [], set()
        for r, n in enumerate(self.past):
            for j in range(int(n)):
                page = self.table[r, j // 64]
                if 0 <= page < self.n_pages:
                    slots.append(page * 64 + j % 64)
                    pages.add(int(page))
        slots, pages = np.array(slots, np.int64), np.array(sorted(pages), np.int64)
        k, v = cache.read(dev(slots, torch.int64))
        assert np.array_equal(k.double().cpu().numpy(), np.where(reference.bad[slots][..., None], np.nan, reference.k[slots]), equal_nan=True)
        assert np.array_equal(v.double().cpu().numpy(), reference.v[slots])
        assert np.array_equal(cache.boxes.double().cpu().numpy()[pages], reference.boxes[pages])


# ---- rotary positions -------------------------------------------------------------------------------


def check_rotated(got, x, positions, frequencies, axes, neighbours, dtype):
    """Off by half a unit of the type, and by |a| + |b| times what the factors are: a turn's fraction has 24 significant bits, 2 pi
    2^-25 = 2^-22.3 of an angle; sine and cosine 2^-20 and the two products' roundings 2^-23 of their sizes; 2^-19 together."""
    want, size = tref.rotate(x, positions, frequencies, axes, neighbours)
    off = U[dtype] * np.abs(want) + size * 2.0 ** -19 + (2.0 ** -25 if dtype == "fp16" else 0.0)
    real = positions[0] >= 0
    err = np.abs(got.double().cpu().numpy() - want)[real]
    assert (err <= off[real]).all(), (err / np.maximum(off[real], 1e-300)).max()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("T,H,K,D,turned,axes,far", [(1, 1, 1, 64, 64, 1, 10), (3, 5, 2, 96, 48, 2, 1000), (130, 12, 3, 128, 128, 3, 10 ** 6),
                                                     (17, 2, 0, 128, 16, 8, 100), (65, 33, 8, 256, 32, 4, 2 ** 31 - 1), (700, 32, 8, 96, 96, 1, 5000)])
def test_rotate(kv, dtype, neighbours, T, H, K, D, turned, axes, far):
    rng = np.random.default_rng(T + D)
    n = turned // 2
    frequencies = [10000.0 ** (-i / n) for i in range(n)]
    axis = sorted(rng.integers(0, axes, n).tolist())
    axis[-1] = axes - 1
    positions = rng.integers(0, far + 1, (axes, T))
    positions[1:] -= rng.integers(0, far + 1, (axes - 1, T))        # below 0 on the other axes
    positions[0, 0] = far
    qk, x = rows(rng, dtype, T, H + K, D)
    rotary = kv.Rotary(frequencies, axes=axis, neighbours=neighbours)
    # out of one projection's rows, into tensors of their own
    q, k = rotary(qk[:, :H], qk[:, H:], dev(positions, torch.int32))
    check_rotated(q, x[:, :H], positions, frequencies, axis, neighbours, dtype)
    check_rotated(k, x[:, H:], positions, frequencies, axis, neighbours, dtype)
    assert torch.equal(q[..., turned:], qk[:, :H, turned:]) and torch.equal(k[..., turned:], qk[:, H:, turned:])
    # where they are: the same bits
    rotary(qk[:, :H], qk[:, H:], dev(positions, torch.int32), out=(qk[:, :H], qk[:, H:]))
    assert torch.equal(qk[:, :H], q) and torch.equal(qk[:, H:], k)


def test_rotate_leaves_rows_without_a_token(kv):
    rng = np.random.default_rng(0)
    rotary = kv.Rotary([1.0 / (i + 1) for i in range(32)])
    x, xn = rows(rng, "bf16", 9, 3, 64)
    positions = np.array([[5, -1, 0, 7, -1, 2, 3, -2 ** 31, 2 ** 31 - 1]])
    out = torch.full_like(x, 3.0), torch.full((9, 0, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    rotary(x, x[:, :0], dev(positions[0], torch.int32), out=out)
    check_rotated(out[0], xn, positions, [1.0 / (i + 1) for i in range(32)], [0] * 32, False, "bf16")
    assert (out[0][torch.from_numpy(positions[0] < 0).cuda()] == 3.0).all()
    assert torch.equal(out[0][2], x[2])                                        # position 0


# ---- trees ------------------------------------------------------------------------------------------


@pytest.mark.parametrize("window", [0, 1, 2, 5, 64])
@pytest.mark.parametrize("new", [[1], [2, 0, 3], [64, 1, 63], [65, 64, 7, 200], [256], [257, 3], [1024, 900, 1], [5] * 300])
def test_tree(kv, new, window):
    """Random trees with several roots, chains, stars; rows without a token behind them."""
    rng = np.random.default_rng(len(new) + window)
    s = TreeServer(kv, rng, "bf16", 1, 64, 1, len(new), 40, held=False)
    s.past[:] = rng.integers(0, 100, len(new))
    s.d_past = dev(s.past, torch.int32)
    T = s.plan(new, max_tokens=sum(new) + 9)
    N = max(new)
    shapes = [random_parents(rng, np.array(new), 0.05), np.concatenate([np.arange(n) - 1 for n in new]),
              np.concatenate([np.minimum(np.arange(n) - 1, 0) for n in new]), rng.integers(-N, 2 * N, sum(new))]
    for parents in shapes:
        parents = np.concatenate((parents, np.full(9, 3)))
        got = kv.tree(dev(parents, torch.int32), s.step, max_nodes=N, window=window)
        sees, positions = tref.tree(parents, s.want, N, window)
        assert np.array_equal(got.masks.cpu().numpy(), tref.words(sees))
        assert np.array_equal(got.positions.cpu().numpy(), positions)
    assert T == len(positions)


def test_tree_of_more_tokens_than_it_has_room_for(kv):
    s = TreeServer(kv, np.random.default_rng(2), "bf16", 1, 64, 8, 2, 4, held=True)
    s.draft([70, 6], max_nodes=5, max_tokens=80)
    s.attend_tree(2)
    s.keep(agree=1.0)


# ---- attention --------------------------------------------------------------------------------------

SHAPES = [(2, 4, 128), (1, 8, 64), (3, 1, 96), (2, 3, 256), (1, 20, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,D", SHAPES)
@pytest.mark.parametrize("W", [8, 70])
def test_tree_attention(kv, dtype, H, G, D, W):
    """Trees behind contexts from nothing to some pages, whole units and shares; rows without a token."""
    rng = np.random.default_rng(H * 100 + D + W)
    s = TreeServer(kv, rng, dtype, H, D, 40, 6, W)
    s.fill([0, 1, 63, 64, 300, 131])
    s.draft([3, 1, 9, 2, 13, 0], max_tokens=31, roots=0.1)
    out, lse = s.attend_tree(H * G)
    assert (out[28:] == 0).all() and torch.isneginf(lse[28:]).all()
    s.attend_tree(H * G, scale=-0.3)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,D", [(2, 4, 128), (2, 1, 64), (1, 7, 96), (1, 2, 256)])
@pytest.mark.parametrize("W", [20, 70])
def test_large_trees(kv, dtype, H, G, D, W):
    """More rows than share a page in registers: tiles of many rows, masks of several words, trees over page borders."""
    rng = np.random.default_rng(G * 10 + D + W)
    s = TreeServer(kv, rng, dtype, H, D, 60, 4, W)
    s.fill([5, 200, 0, 700])
    s.draft([70, 150, 64, 33])
    s.attend_tree(H * G)


@pytest.mark.parametrize("n,G", [(4, 4), (5, 4), (8, 4), (9, 4), (16, 4), (17, 4), (33, 2), (3, 5), (13, 5), (64, 1), (65, 1)])
def test_tree_rows_around_tile_borders(kv, n, G):
    rng = np.random.default_rng(n * G)
    for W, past in ((12, [100, 3, 620]), (90, [4000, 70, 1])):
        s = TreeServer(kv, rng, "bf16", 2, 64, 90, 3, W)
        s.fill(past)
        s.draft([n, max(1, n - 1), 1])
        s.attend_tree(2 * G)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,G,D", [(2, 4, 128), (2, 3, 64), (1, 5, 96), (1, 2, 256)])
@pytest.mark.parametrize("new", [[9, 6, 13, 1, 8], [40, 3, 70, 16, 1]])
@pytest.mark.parametrize("window", [0, 90])
def test_trees_in_wide_tables(kv, dtype, H, G, D, new, window):
    """Tables whose width promises long contexts decide how the work is cut: units of one and of two tiles, parts of them in shares, shares
    across units and requests; a page in the middle of a request that is not there."""
    rng = np.random.default_rng(D + G + len(new) + window)
    s = TreeServer(kv, rng, dtype, H, D, 60, 5, 12000)
    s.fill([700, 64, 5, 900, 333])
    s.draft(new, window=window)
    s.attend_tree(H * G, scale=-0.2)
    s.d_table[3, 2] = s.want["table"][3, 2] = 60
    s.d_table[0, 0] = s.want["table"][0, 0] = -1
    s.attend_tree(H * G)


@pytest.mark.parametrize("D,G,new", [(128, 4, 16), (128, 1, 40), (96, 5, 13), (64, 16, 8), (256, 3, 20)])
@pytest.mark.parametrize("window", [0, 2500])
def test_one_tree_behind_a_long_context(kv, D, G, new, window):
    """One request whose units of three, four and more tiles go into parts of a few pages, some of which end between the two
    wavefronts that take a unit's pages in turn."""
    rng = np.random.default_rng(D + G + window)
    s = TreeServer(kv, rng, "bf16", 2, D, 160, 1, 30000)
    s.fill([9001])
    s.draft([new], window=window)
    s.attend_tree(2 * G)


@pytest.mark.parametrize("R,D,G", [(30, 128, 4), (31, 128, 4), (70, 128, 8), (70, 64, 3)])
def test_trees_of_requests_whose_lists_fill_the_lds(kv, R, D, G):
    """Lists of the requests beside the pages in LDS, and from a launch of their own where they do not fit there."""
    rng = np.random.default_rng(R + D + G)
    s = TreeServer(kv, rng, "fp16", 2, D, 8 * R, R, 6000)
    s.fill(rng.integers(0, 400, R))
    new = rng.integers(0, 18, R)
    s.draft(new, max_tokens=int(new.sum()) + 3)
    s.attend_tree(2 * G)
    s.keep()


@pytest.mark.parametrize("G,W", [(1, 4), (8, 4), (4, 100)])
def test_trees_of_more_requests_than_are_scanned_in_a_workgroup(kv, G, W):
    rng = np.random.default_rng(25)
    R = 530
    s = TreeServer(kv, rng, "bf16", 1, 64, 2 * R, R, W)
    s.fill(rng.integers(0, 60, R))
    s.draft(rng.integers(0, 7, R), max_tokens=7 * R)
    s.attend_tree(G)
    s.keep()


@pytest.mark.parametrize("window", [1, 2, 7, 64, 100, 1000])
@pytest.mark.parametrize("H,G,D,new", [(2, 2, 64, [9, 20, 3]), (1, 8, 128, [40, 70, 1])])
def test_tree_windows(kv, window, H, G, D, new):
    rng = np.random.default_rng(window + D)
    s = TreeServer(kv, rng, "fp16", H, D, 40, 3, 20)
    s.fill([700, 61, 0])
    s.draft(new, window=window, roots=0.05)
    s.attend_tree(H * G)


@pytest.mark.parametrize("new", [[9, 20, 3], [70, 100, 1]])
def test_any_masks(kv, new):
    """Masks that are no trees: rows that see nothing of the new tokens (and, without a past, nothing at all), later tokens, bits of
    tokens that are not there; positions that are nothing."""
    rng = np.random.default_rng(4)
    s = TreeServer(kv, rng, "bf16", 2, 64, 20, 3, 10)
    s.fill([100, 0, 64])
    T = s.draft(new)
    N = s.tree.max_nodes
    s.sees = rng.random((T, N)) < 0.3
    s.sees[::5] = False
    masks = dev(tref.words(s.sees), torch.int64)
    for window in (0, 30):
        s.positions = rng.integers(-2 ** 31, 2 ** 31, T) if window else s.positions
        tree = kv.Tree(masks, dev(s.positions, torch.int32), N, window)
        out, lse = s.attend_tree(8, tree=tree)
    nothing = new[0] + np.nonzero(~s.sees[new[0]:new[0] + new[1], :new[1]].any(1))[0]
    assert len(nothing) and (out[nothing] == 0).all() and torch.isneginf(lse[nothing]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_tree_behind_a_long_context(kv, dtype):
    rng = np.random.default_rng(6)
    s = TreeServer(kv, rng, dtype, 1, 128, 330, 1, 330)
    s.fill([20011])
    for n in (1, 4, 16, 40, 70):
        s.draft([n])
        s.attend_tree(4)
        s.keep(agree=0.0)


def test_tree_attention_is_causal_attention_for_a_chain(kv):
    """A chain is a chunk of a prompt: both calls within the bounds of the same 64-bit result."""
    rng = np.random.default_rng(7)
    s = TreeServer(kv, rng, "bf16", 2, 128, 30, 2, 12)
    s.fill([130, 5])
    s.draft([17, 40], parents=np.concatenate((np.arange(17) - 1, np.arange(40) - 1)))
    q, _ = rows(rng, "bf16", 57, 8, 128)
    s.attend_tree(8, q=q)
    s.attend(8, q=q)


def test_pages_that_are_missing(kv):
    """Pages run out in the middle of the trees; the tokens without one are neither seen nor kept."""
    rng = np.random.default_rng(8)
    s = TreeServer(kv, rng, "bf16", 1, 64, 5, 3, 4)
    s.fill([60, 60, 100])
    s.draft([10, 20, 40])
    assert s.state[2] > 0
    s.attend_tree(4)
    s.keep(agree=1.0)


def test_the_tables_width_cuts_trees(kv):
    rng = np.random.default_rng(9)
    s = TreeServer(kv, rng, "bf16", 1, 64, 8, 2, 2)
    s.fill([120, 10])
    s.draft([20, 20])
    s.attend_tree(4)
    s.keep(agree=1.0)


@pytest.mark.parametrize("new", [[8, 12], [70, 80]])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_tokens_that_are_no_numbers_stay_in_the_rows_that_see_them(kv, dtype, new):
    rng = np.random.default_rng(10)
    s = TreeServer(kv, rng, dtype, 2, 64, 12, 2, 6)
    s.fill([50, 64])

    def edit(k, v):
        k[3, 0, 5], v[new[0] + 5, 1, 0] = float("inf"), float("nan")
    s.draft(new, edit=edit)
    out, _ = s.attend_tree(4)
    assert torch.isnan(out).any() and torch.isfinite(out[0]).all()
    q, _ = rows(rng, dtype, sum(new), 4, 64)
    q[2, 1], q[new[0], 3, 0] = float("nan"), float("inf")
    got, _ = s.cache.tree_attention(q, s.step, s.tree)
    clean = torch.ones(got.shape[:2], dtype=torch.bool, device="cuda")
    clean[2, 1] = clean[new[0], 3] = False
    again, _ = s.cache.tree_attention(torch.where(clean[..., None], q, 1.0), s.step, s.tree)
    assert torch.equal(torch.nan_to_num(got[clean]), torch.nan_to_num(again[clean]))


def test_rows_of_a_projection_and_strided_results(kv):
    rng = np.random.default_rng(11)
    s = TreeServer(kv, rng, "fp16", 2, 96, 12, 2, 8)
    s.fill([200, 30])
    s.draft([7, 20])
    big, _ = rows(rng, "fp16", 27, 12, 96)
    want, want_lse = s.attend_tree(8, q=big[:, 2:10].contiguous())
    room = torch.zeros(8, 27, 104, dtype=torch.float16, device="cuda")
    out, lse = s.cache.tree_attention(big[:, 2:10], s.step, s.tree, out=room[..., :96].transpose(0, 1))
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and (room[..., 96:] == 0).all()


# ---- what stays -------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,D", [(1, 64), (5, 96), (2, 128), (2, 256)])
def test_steps_with_drafts(kv, dtype, H, D):
    """Steps in a row: trees checked and kept, requests that wait, end and start; every page is in one place throughout."""
    rng = np.random.default_rng(D)
    R, W, n_pages = 6, 6, 30
    s = TreeServer(kv, rng, dtype, H, D, n_pages, R, W, ring_start=n_pages - 3)
    s.fill(rng.integers(0, 150, R))
    for step in range(6):
        new = rng.integers(1, 30 if step % 2 else 70, R)
        new[rng.random(R) < 0.15] = 0
        new[rng.random(R) < 0.15] = -1
        s.draft(new, max_tokens=int(np.maximum(new, 0).sum()) + int(rng.integers(0, 5)), roots=0.03)
        s.attend_tree(2 * H)
        s.keep(agree=(0.3, 0.8, 1.0)[step % 3])
        head, tail, _ = s.state
        where = [s.ring[i % n_pages] for i in range(head, tail)]
        where += [p for r in range(R) for p in s.table[r, :-(-s.past[r] // 64)] if p >= 0]
        assert sorted(where) == list(range(n_pages))


@pytest.mark.parametrize("dtype,new,tiny", [("bf16", [40, 70, 30, 9], 0), ("fp16", [40, 60, 30, 9], 0), ("bf16", [40, 64, 30, 9], -129),
                                            ("fp16", [40, 64, 30, 9], -22)])
def test_keep_gives_what_appending_only_the_kept_gives(kv, dtype, new, tiny):
    """Bytes of the held tokens and boxes, page for page, against a cache that never saw the others; keys as small as the type has them."""
    rng = np.random.default_rng(13)
    s = TreeServer(kv, rng, dtype, 3, 128, 30, 4, 6)
    s.gain *= 2.0 ** tiny
    s.fill([0, 60, 64, 130])
    other = kv.KvCache(30, 3, 128, TYPES[dtype])
    other.pages.copy_(s.cache.pages), other.boxes.copy_(s.cache.boxes)
    T = s.draft(new, parents=random_parents(rng, np.array(new)))
    k, v = s.cache.read(s.step.slots)
    kept = s.keep(agree=1.0)
    q_start, slots = s.want["q_start"], s.step.slots
    to = [q_start[r] + i for r in range(4) for i in range(s.past[r] - s.before[r])]
    stay = dev(kept[to], torch.int64)
    assert len(to) > 12
    other.append(k[stay].contiguous(), v[stay].contiguous(), slots[dev(np.array(to), torch.int64)].contiguous())
    held = []
    for r in range(4):
        held += [s.table[r, j // 64] * 64 + j % 64 for j in range(s.past[r])]
    held = dev(np.array(held), torch.int64)
    for a, b in zip(s.cache.read(held), other.read(held)):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    pages = torch.unique(held // 64)
    assert torch.equal(s.cache.boxes[pages].view(torch.int16), other.boxes[pages].view(torch.int16))
    assert T == sum(new)


def test_keep_in_many_layers(kv):
    """More caches than one launch takes, each with tokens of its own."""
    rng = np.random.default_rng(14)
    s = TreeServer(kv, rng, "fp16", 2, 64, 8, 2, 4)
    s.fill([30, 100])
    s.draft([20, 40])
    more = []
    for i in range(70):
        cache, reference = kv.KvCache(8, 2, 64, torch.float16), ref.Cache(8, 2, 64)
        k, kn = rows(rng, "fp16", 60, 2, 64)
        cache.append(k, k, s.step.slots)
        reference.append(kn, kn, s.want["slots"])
        more.append((cache, reference))
    # (what the other layers hold before the step was never written: zeros)
    s.keep(agree=0.9, more=more)


@pytest.mark.parametrize("new", [[64], [65], [300, 700], [1024]])
def test_a_chain_that_agrees_stays_where_it_is(kv, new):
    rng = np.random.default_rng(15)
    n_pages = sum(n // 64 + 3 for n in new)
    s = TreeServer(kv, rng, "bf16", 1, 64, n_pages, len(new), 20)
    s.fill([10] * len(new))
    s.draft(new, parents=np.concatenate([np.arange(n) - 1 for n in new]))
    before = s.cache.pages.clone(), s.cache.boxes.clone()
    s.keep(agree=1.0)
    assert (s.past == 10 + np.array(new)).all()
    assert torch.equal(before[0], s.cache.pages) and torch.equal(before[1], s.cache.boxes)
    # and one that agrees halfway: nothing moves, pages go back
    s.draft([min(n, 200) for n in new], parents=np.concatenate([np.arange(min(n, 200)) - 1 for n in new]))
    drafted, picked = np.arange(len(s.parents)), np.arange(len(s.parents)) + 1
    picked[100:] = -5
    s.keep(drafted=drafted, picked=picked)


def test_equal_tokens_beside_each_other(kv):
    """Two children with the picked token: the one whose path goes on, the first where both do."""
    s = TreeServer(kv, np.random.default_rng(16), "bf16", 1, 64, 4, 2, 2)
    s.fill([10, 20])
    parents = [-1, 0, 0, 2, -1, 0, 0, 1, 2]
    s.draft([4, 5], parents=parents)
    kept = s.keep(drafted=np.array([5, 6, 6, 7, 5, 6, 6, 7, 7]), picked=np.array([6, 1, 7, 2, 6, 7, 7, 3, 4]))
    assert kept.tolist() == [0, 2, 3, -1, 4, 5, 7, -1, -1] and s.past.tolist() == [13, 23]


@pytest.mark.parametrize("R", [1, 5, 300, 1100])
def test_pages_go_back_in_order(kv, R):
    """Many requests, all of whose drafts are refused; a ring with room and one without."""
    rng = np.random.default_rng(R)
    s = TreeServer(kv, rng, "bf16", 1, 64, 3 * R, R, 4, held=False)
    s.past[:] = 0
    new = rng.integers(60, 130, R)
    s.plan(new)
    s.parents = random_parents(rng, new)
    s.tree = kv.tree(dev(s.parents, torch.int32), s.step, max_nodes=130)
    s.sees, s.positions = tref.tree(s.parents, s.want, 130)
    lens, kept, ring, state = tref.keep([], s.want, s.sees, np.zeros(len(s.parents)), np.ones(len(s.parents)), s.ring, s.state, 3 * R)
    got = kv.keep([s.cache], s.step, s.tree, torch.zeros_like(s.step.requests), torch.ones_like(s.step.requests), s.d_ring, s.d_state)
    for x, w in ((got.lens, lens), (got.rows, kept), (s.d_ring, ring), (got.free_state, state)):
        assert np.array_equal(x.cpu().numpy().astype(np.int64), w)
    assert (lens == 1).all()


def test_keep_of_no_requests_and_of_no_tokens(kv):
    s = TreeServer(kv, np.random.default_rng(17), "bf16", 1, 64, 4, 2, 2)
    s.fill([10, 20])
    for T in (0, 3):
        s.plan([0, -1], max_tokens=T)
        s.parents = np.zeros(T, np.int64)
        s.tree = kv.tree(dev(s.parents, torch.int32), s.step, max_nodes=4)
        s.sees, s.positions = tref.tree(s.parents, s.want, 4)
        s.keep()
        assert s.past.tolist() == [10, 0]
    table = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    step = kv.plan(none, none, table, s.d_ring, s.d_state, max_tokens=5)
    five = torch.zeros(5, dtype=torch.int32, device="cuda")
    tree = kv.tree(five, step)
    assert (tree.masks == 0).all() and (tree.positions == -1).all()
    kept = kv.keep([s.cache], step, tree, five, five, s.d_ring, step.free_state)
    assert (kept.rows == -1).all() and torch.equal(kept.free_state, step.free_state)


# ---- reading back -----------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,D", [(1, 64), (3, 96), (2, 128), (5, 256)])
def test_read(kv, dtype, H, D):
    """Any slots in any order, twice, outside; tokens that are no numbers; results in strided rows."""
    rng = np.random.default_rng(D + H)
    s = Server(kv, rng, dtype, H, D, 7, 2, 5)

    def edit(k, v):
        k[7, 0, 3], v[70, H - 1, 9] = float("nan"), float("-inf")
    s.fill([200, 100], edit=edit)
    slots = np.concatenate((s.want["slots"], rng.integers(0, 7 * 64, 41), [-1, 7 * 64, -2 ** 60, 2 ** 60, 7 * 64 - 1]))
    k, v = s.cache.read(dev(slots, torch.int64))
    inside = (slots >= 0) & (slots < 7 * 64)
    at = np.where(inside, slots, 0)
    want_k = np.where(s.ref.bad[at][..., None], np.nan, s.ref.k[at])
    assert np.array_equal(k.double().cpu().numpy(), np.where(inside[:, None, None], want_k, 0.0), equal_nan=True)
    assert np.array_equal(v.double().cpu().numpy(), np.where(inside[:, None, None], s.ref.v[at], 0.0))
    room = torch.ones(2, H, len(slots), D + 8, dtype=TYPES[dtype], device="cuda")
    s.cache.read(dev(slots, torch.int64), out=(room[0, ..., :D].transpose(0, 1), room[1, ..., 8:].transpose(0, 1)))
    assert torch.equal(torch.nan_to_num(room[0, ..., :D].transpose(0, 1)), torch.nan_to_num(k)) and torch.equal(room[1, ..., 8:].transpose(0, 1), v)
    assert (room[0, ..., D:] == 1).all() and (room[1, ..., :8] == 1).all()
    for n in (0, 1, 64, 130):
        a, b = s.cache.read(dev(slots[:n], torch.int64))
        assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(k[:n])) and torch.equal(b, v[:n])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,D", [(4, 64), (5, 96), (4, 128), (8, 256), (33, 64)])
def test_read_of_runs(kv, dtype, H, D):
    """Long lists, where a lane has four tokens: runs of all lengths that begin anywhere in a page and in the list, slots outside, tokens that
    are no numbers; the same bits as a few slots at a time, which are compared with the definitions above."""
    rng = np.random.default_rng(D + H)
    n_pages = 40
    s = Server(kv, rng, dtype, H, D, n_pages, 1, n_pages, held=False)
    s.ref = None
    step = kv.plan(s.d_past, dev(np.array([n_pages * 64]), torch.int32), s.d_table, s.d_ring, s.d_state, max_tokens=n_pages * 64)
    k, v = (rows(rng, dtype, n_pages * 64, H, D)[0] for _ in range(2))
    k[5, 0, 1], v[77, H - 1, 2], k[1000, H // 2, 0] = float("nan"), float("inf"), float("-inf")
    s.cache.append(k, v, step.slots)
    parts = []
    while sum(map(len, parts)) * H < 17000:
        n = int(rng.choice([1, 2, 3, 4, 5, 8, 13, 64, 70, 130]))
        parts.append(int(rng.integers(-3, n_pages * 64 - n + 4)) + np.arange(n))
        if rng.random() < 0.1:
            parts.append(rng.integers(0, n_pages * 64, 7))
    for shift in range(5):
        slots = dev(np.concatenate(parts)[shift:], torch.int64)
        a, b = s.cache.read(slots)
        few = 4000 // H
        small = [s.cache.read(slots[i:i + few].contiguous()) for i in range(0, len(slots), few)]
        assert len(slots) * H >= 16384
        for got, want in ((a, torch.cat([x[0] for x in small])), (b, torch.cat([x[1] for x in small]))):
            assert torch.equal(got.view(torch.int16), want.view(torch.int16))


def test_read_and_keep_behind_32_bits(kv):
    """Pages whose bytes begin behind 4 GiB."""
    rng = np.random.default_rng(20)
    n_pages = (1 << 32) // (68 * 256 * 8) + 40
    s = TreeServer(kv, rng, "bf16", 8, 256, n_pages, 1, 4, held=False)
    s.ref = None
    ids = np.array([n_pages - 1, n_pages - 3, n_pages - 20])
    s.d_ring[:3] = dev(ids, torch.int32)
    step = kv.plan(s.d_past, dev(np.array([150]), torch.int32), s.d_table, s.d_ring, s.d_state, max_tokens=150)
    k, _ = rows(rng, "bf16", 150, 8, 256)
    v, _ = rows(rng, "bf16", 150, 8, 256)
    kr, vr = torch.empty_like(k), torch.empty_like(v)
    s.cache.append(k, v, step.slots, rounded=(kr, vr))
    a, b = s.cache.read(step.slots)
    assert torch.equal(a, kr) and torch.equal(b, vr)
    parents = np.floor(np.arange(150) * 0.9).astype(np.int64) - 1
    parents[1:] = np.maximum(parents[1:], 0)
    tree = kv.tree(dev(parents, torch.int32), step, max_nodes=150)
    path = tref.ancestors(parents, 149)[::-1]
    drafted, picked = np.arange(150), np.full(150, -1)
    picked[path[:-1]] = path[1:]
    kept = kv.keep([s.cache], step, tree, dev(drafted, torch.int32), dev(picked, torch.int32), s.d_ring, step.free_state)
    n = len(path)
    assert kept.rows[:n].tolist() == path and kept.lens.tolist() == [n]
    a, b = s.cache.read(step.slots[:n])
    at = dev(np.array(path), torch.int64)
    assert torch.equal(a, kr[at]) and torch.equal(b, vr[at])


# ---- together ---------------------------------------------------------------------------------------


def test_drafting_gives_what_decoding_gives(kv):
    """Some steps of drafts and acceptance, with rotated keys, against the same tokens one by one: the cache holds the same bytes, and
    attention is within the bounds of the same 64-bit results."""
    rng = np.random.default_rng(21)
    R, H, G, D = 3, 2, 4, 128
    rotary = kv.Rotary([10000.0 ** (-i / 64) for i in range(64)])
    cache, plain = (kv.KvCache(20, H, D) for _ in range(2))
    sides = []
    for c in (cache, plain):
        ring, state = c.free_ring()
        sides.append(dict(cache=c, ring=ring, state=state, lens=torch.zeros(R, dtype=torch.int32, device="cuda"),
                          table=torch.full((R, 5), -1, dtype=torch.int32, device="cuda")))

    def plan(x, new):
        step = kv.plan(x["lens"], dev(np.array(new), torch.int32), x["table"], x["ring"], x["state"], max_tokens=int(sum(new)))
        x["lens"], x["state"] = step.kv_lens, step.free_state
        return step

    tokens = {}  # rows of token n of request r, the same on both sides

    def token(r, n):
        if (r, n) not in tokens:
            tokens[r, n] = [torch.from_numpy(rng.normal(size=(h, D))).bfloat16() for h in (H * G, H, H)]
        return tokens[r, n]

    results = {}
    past = [0] * R
    for step_no in range(5):
        new = [int(n) for n in rng.integers(2, 25, R)]
        parents = np.concatenate([np.maximum(np.floor(np.arange(n) * 0.6).astype(np.int64) - (np.arange(n) == 0), -(np.arange(n) == 0).astype(np.int64)) for n in new])
        picked, drafted, paths = [], [], []
        at = 0
        step = plan(sides[0], new)
        tree = kv.tree(dev(parents, torch.int32), step, max_nodes=25)
        q, k, v = [], [], []
        for r, n in enumerate(new):
            p = parents[at:at + n]
            path = tref.ancestors(p, int(rng.integers(n)))[::-1]
            paths.append(path)
            d, x = rng.integers(10, 1000, n), np.full(n, 5)
            x[path[:-1]] = d[path[1:]]
            d[[i for i in range(1, n) if i not in path]] = 7
            for i in range(n):
                if i in path:
                    a = token(r, past[r] + path.index(i))
                else:
                    a = [torch.from_numpy(rng.normal(size=(h, D))).bfloat16() for h in (H * G, H, H)]
                q.append(a[0]), k.append(a[1]), v.append(a[2])
            drafted.append(d), picked.append(x)
            at += n
        q, k, v = (torch.stack(y).cuda() for y in (q, k, v))
        q, k = rotary(q, k, tree.positions)
        cache.append(k, v, step.slots)
        out, lse = cache.tree_attention(q, step, tree)
        start = step.q_start.tolist()
        for r in range(R):
            for i, node in enumerate(paths[r]):
                results[r, past[r] + i] = out[start[r] + node].double(), lse[start[r] + node].double()
        kept = kv.keep([cache], step, tree, dev(np.concatenate(drafted), torch.int32), dev(np.concatenate(picked), torch.int32),
                       sides[0]["ring"], step.free_state)
        sides[0]["lens"], sides[0]["state"] = kept.lens, kept.free_state
        past = [p + len(w) for p, w in zip(past, paths)]
        assert kept.lens.tolist() == past
    # one by one
    for n in range(max(past)):
        new = [int(n < p) for p in past]
        step = plan(sides[1], new)
        who = [r for r in range(R) if new[r]]
        q, k, v = (torch.stack([token(r, n)[i] for r in who]).cuda() for i in range(3))
        q, k = rotary(q, k, step.positions)
        plain.append(k, v, step.slots)
        out, lse = plain.attention(q, step, max_new=1)
        for i, r in enumerate(who):
            a, b = results[r, n]
            # each within u (1 + 1.01) of a result below 6 * 4 at most; sizes here are normal
            assert (a - out[i].double()).abs().max() < 4 * U["bf16"] * 4 and (b - lse[i].double()).abs().max() < 1e-4
    for r in range(R):
        slots = [dev(np.array([s["table"][r, j // 64].item() * 64 + j % 64 for j in range(past[r])]), torch.int64) for s in sides]
        for a, b in zip(cache.read(slots[0]), plain.read(slots[1])):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
        pages = [torch.unique_consecutive(s // 64) for s in slots]
        assert torch.equal(cache.boxes[pages[0]].view(torch.int16), plain.boxes[pages[1]].view(torch.int16))


def test_streams_and_graphs_of_trees(kv):
    """A step captured once and replayed with other lengths, trees and rows, eager work between; two graphs, each with its workspace."""
    rng = np.random.default_rng(22)
    H, G, D, R, N = 2, 4, 64, 3, 12
    T, W, n_pages = 30, 10, 24
    rotary = kv.Rotary([10000.0 ** (-i / 32) for i in range(32)])

    def setup():
        c = kv.KvCache(n_pages, H, D)
        ring, state = c.free_ring()
        z = lambda *shape, dtype=torch.int32: torch.zeros(*shape, dtype=dtype, device="cuda")
        x = dict(cache=c, ring=ring, state=state, lens=z(R), new=z(R), parents=z(T), drafted=z(T), picked=z(T),
                 table=torch.full((R, W), -1, dtype=torch.int32, device="cuda"))
        x["q"], x["k"], x["v"] = z(T, H * G, D, dtype=torch.bfloat16), z(T, H, D, dtype=torch.bfloat16), z(T, H, D, dtype=torch.bfloat16)
        x["step"], x["tree"] = kv.Step.empty(R, T, x["table"]), kv.Tree.empty(T, N)
        x["kept"], x["turned"] = kv.Kept.empty(x["step"]), (torch.empty_like(x["q"]), torch.empty_like(x["k"]))
        x["out"], x["lse"] = torch.empty_like(x["q"]), torch.empty(T, H * G, device="cuda")
        x["ws"] = c.tree_attention_workspace(x["step"], H * G, x["tree"])
        return x

    def once(x):
        step = kv.plan(x["lens"], x["new"], x["table"], x["ring"], x["state"], out=x["step"])
        kv.tree(x["parents"], step, out=x["tree"])
        q, k = rotary(x["q"], x["k"], x["tree"].positions, out=x["turned"])
        x["cache"].append(k, x["v"], step.slots)
        x["cache"].tree_attention(q, step, x["tree"], out=x["out"], lse=x["lse"], workspace=x["ws"])
        kv.keep([x["cache"]], step, x["tree"], x["drafted"], x["picked"], x["ring"], step.free_state, out=x["kept"])
        x["lens"].copy_(x["kept"].lens)
        x["state"].copy_(x["kept"].free_state)

    def inputs(x, seed):
        g = np.random.default_rng(seed)
        new = g.integers(1, 11, R)
        x["new"].copy_(dev(new, torch.int32))
        parents = random_parents(g, new)
        x["parents"].copy_(dev(np.concatenate((parents, np.zeros(T - len(parents), np.int64))), torch.int32))
        x["drafted"].copy_(dev(g.integers(0, 2, T), torch.int32)), x["picked"].copy_(dev(g.integers(0, 2, T), torch.int32))
        for name in ("q", "k", "v"):
            x[name].copy_(dev(g.normal(size=tuple(x[name].shape)), torch.bfloat16))

    eager, graphs = setup(), [setup(), setup()]
    side = torch.cuda.Stream()
    captured = []
    for x in graphs:
        inputs(x, 99)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            once(x)                                       # warm
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            once(x)
        captured.append(g)
    inputs(eager, 99)
    once(eager)
    for i in range(6):
        inputs(eager, i)
        once(eager)
        for x, g in zip(graphs, captured):
            inputs(x, i)
            g.replay()
            torch.cuda.synchronize()
            rows_of = int(eager["step"].q_start[-1])
            for name in ("out", "lse"):
                assert torch.equal(x[name][:rows_of], eager[name][:rows_of]), (i, name)
            for name in ("lens", "state", "table", "ring"):
                assert torch.equal(x[name], eager[name]), (i, name)
            assert torch.equal(x["kept"].rows, eager["kept"].rows)
            assert torch.equal(x["cache"].boxes, eager["cache"].boxes)


def test_the_same_calls_give_the_same_bits(kv):
    rng = np.random.default_rng(23)
    s = TreeServer(kv, rng, "bf16", 2, 128, 90, 3, 80)
    s.fill([3000, 100, 1111])
    s.draft([16, 5, 30])
    q, _ = rows(rng, "bf16", 51, 8, 128)
    first = s.cache.tree_attention(q, s.step, s.tree)
    for _ in range(5):
        for a, b in zip(first, s.cache.tree_attention(q, s.step, s.tree)):
            assert torch.equal(a, b)


# ---- refusals ---------------------------------------------------------------------------------------


def test_tree_refusals(kv):
    s = TreeServer(kv, np.random.default_rng(24), "bf16", 2, 64, 6, 2, 3)
    s.fill([20, 30])
    T = s.draft([4, 5])
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")
    q = torch.zeros(T, 4, 64, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: kv.tree(i32(T + 1), s.step), lambda: kv.tree(i32(T).long(), s.step), lambda: kv.tree(i32(T), s.step, max_nodes=1025),
                 lambda: kv.tree(i32(T), s.step, max_nodes=0), lambda: kv.tree(i32(T), s.step, window=-1),
                 lambda: kv.tree(i32(T), s.step, max_nodes=7, out=s.tree), lambda: kv.tree(i32(T), s.step, out=kv.Tree.empty(T + 1, 5)),
                 lambda: kv.Tree(torch.zeros(3, 2, dtype=torch.int64, device="cuda"), i32(3), 64),
                 lambda: s.cache.tree_attention(q[:, :, :32], s.step, s.tree), lambda: s.cache.tree_attention(q.half(), s.step, s.tree),
                 lambda: s.cache.tree_attention(q[:-1], s.step, s.tree), lambda: s.cache.tree_attention(q, s.step, kv.Tree.empty(T + 1, 5)),
                 lambda: kv.keep([s.cache], s.step, s.tree, i32(T - 1), i32(T), s.d_ring, s.d_state),
                 lambda: kv.keep([s.cache], s.step, s.tree, i32(T), i32(T), s.d_ring, s.d_state, out=kv.Kept(i32(3), i32(T), s.d_state.clone())),
                 lambda: kv.Rotary([1.0] * 7), lambda: kv.Rotary([1.0] * 136), lambda: kv.Rotary([float("nan")] * 8),
                 lambda: kv.Rotary([1.0] * 8, axes=[0] * 7), lambda: kv.Rotary([1.0] * 8, axes=[8] + [0] * 7),
                 lambda: kv.Rotary([1.0] * 8)(q, q[:, :2], i32(2, T)), lambda: kv.Rotary([1.0] * 8)(q.float(), q[:, :2], i32(T)),
                 lambda: s.cache.read(i32(4)), lambda: s.cache.read(torch.zeros(4, dtype=torch.int64, device="cuda"), out=(q[:4], q[:4]))):
        with pytest.raises(ValueError):
            call()
    windowed = kv.tree(i32(T), s.step, max_nodes=5, window=3)
    other = kv.KvCache(6, 1, 64)
    for call in (lambda: s.cache.tree_attention(torch.zeros(T, 3, 64, dtype=torch.bfloat16, device="cuda"), s.step, s.tree),
                 lambda: s.cache.tree_attention(q, s.step, s.tree, scale=float("nan")),
                 lambda: s.cache.tree_attention(q, s.step, s.tree, out=q[:, :1].expand(-1, 4, -1)),
                 lambda: s.cache.tree_attention(q, s.step, s.tree, workspace=torch.zeros(0, dtype=torch.uint8, device="cuda")) if
                 s.cache.tree_attention_workspace(s.step, 4, s.tree).numel() > 1 else kv.keep([], s.step, s.tree, i32(T), i32(T), s.d_ring, s.d_state),
                 lambda: kv.keep([], s.step, s.tree, i32(T), i32(T), s.d_ring, s.d_state),
                 lambda: kv.keep([s.cache, s.cache], s.step, s.tree, i32(T), i32(T), s.d_ring, s.d_state),
                 lambda: kv.keep([s.cache, other], s.step, s.tree, i32(T), i32(T), s.d_ring, s.d_state),
                 lambda: kv.keep([s.cache], s.step, windowed, i32(T), i32(T), s.d_ring, s.d_state),
                 lambda: kv.Rotary([1.0] * 40)(q, q[:, :2], i32(T)),
                 lambda: kv.Rotary([1.0] * 8)(q[:, :, :56], q[:, :, :56], i32(T))):
        with pytest.raises(kv.IvfpqError):
            call()
