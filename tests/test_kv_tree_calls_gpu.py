"""Calls of decoding with drafted tokens that a caller may make beside the usual ones, on the GPU."""
import numpy as np
import pytest
import torch

import kv_tree_reference as tref
from test_kv_gpu import TYPES, dev, kv, rows  # noqa: F401
from test_kv_tree_gpu import TreeServer, random_parents

pytestmark = pytest.mark.gpu


def own_masks(s, sees):
    """The step's tree with masks [T][max_nodes] of the caller's own."""
    s.sees = sees
    s.tree = s.kv.Tree(dev(tref.words(sees), torch.int64), s.tree.positions, s.tree.max_nodes)


@pytest.mark.parametrize("dtype,H,D", [("bf16", 2, 128), ("fp16", 5, 64), ("bf16", 1, 96), ("fp16", 2, 256)])
@pytest.mark.parametrize("n", [3, 30, 64, 65, 200])
def test_keep_of_blocks_of_which_nothing_stays(kv, dtype, H, D, n):
    """Blocks whose tokens see each other: one that does not agree goes as a whole, the request's first token with it, and
    the box of the page that it began in is that of what was held."""
    rng = np.random.default_rng(n + D)
    s = TreeServer(kv, rng, dtype, H, D, 60, 6, 8)
    s.fill([0, 10, 64, 100, 63, 127])
    held = s.cache.boxes.clone()
    new = [n, n, n, n, n, max(n // 2, 1)]
    T = s.draft(new)
    sees = np.zeros((T, n), bool)
    drafted, picked = np.arange(T) % 7, (np.arange(T) + 1) % 7
    for r, (a, b) in enumerate(zip(s.want["q_start"], s.want["q_start"][1:])):
        first = (b - a) // 2 if r == 3 else b - a        # the fourth request has two blocks, of which the first agrees
        sees[a:a + first, :first] = True
        sees[a + first:b, :b - a] = True
        if r < 4 and b - a > 1:
            picked[b - 2] = -1
    own_masks(s, sees)
    kept = s.keep(drafted=drafted, picked=picked)
    assert s.past.tolist() == [0, 10, 64, 100 + n // 2, 63 + n, 127 + max(n // 2, 1)] and (kept[:3 * n] == -1).all()
    for r, column in ((1, 0), (2, 0)):
        page = s.table[r, column]
        assert torch.equal(s.cache.boxes[page].view(torch.int16), held[page].view(torch.int16))
    # and on from there
    s.draft([5, 40, 1, 9, 0, 70])
    s.attend_tree(2 * H)
    s.keep(agree=1.0)


@pytest.mark.parametrize("n", [20, 64, 90])
@pytest.mark.parametrize("density", [0.02, 0.3])
def test_keep_with_any_masks(kv, n, density):
    """Paths from anywhere: without the first token, with later ones, tokens that see nothing, bits of tokens that are not there."""
    rng = np.random.default_rng(n)
    s = TreeServer(kv, rng, "bf16", 3, 64, 90, 12, 8)
    s.fill(rng.integers(0, 140, 12))
    for step in range(3):
        new = rng.integers(1, n + 1, 12)
        T = s.draft(new, max_nodes=n)
        sees = rng.random((T, n)) < density
        sees[:, 0] |= rng.random(T) < 0.3
        sees[::7] = False
        own_masks(s, sees)
        s.keep(drafted=rng.integers(0, 2, T) * (step < 2), picked=rng.integers(0, 2, T) * (step < 2))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("new", [[4] * 12, [9, 1, 30, 0, 17, 2, 5, 8, 8, 8, 1, 3], [70, 3, 40] + [1] * 9])
def test_trees_made_without_a_word_on_their_size(kv, dtype, new):
    """max_nodes left out: as many as the step has rows, whatever its requests have."""
    rng = np.random.default_rng(sum(new))
    s = TreeServer(kv, rng, dtype, 2, 128, 140, 12, 70)
    s.fill(rng.integers(0, 600, 12))
    T = s.draft(new)
    small = s.tree
    s.tree = kv.tree(dev(s.parents, torch.int32), s.step)
    assert s.tree.max_nodes == T and torch.equal(s.tree.positions, small.positions)
    s.sees, _ = tref.tree(s.parents, s.want, T)
    assert np.array_equal(s.tree.masks.cpu().numpy(), tref.words(s.sees))
    s.attend_tree(8)
    s.keep(agree=0.8)


def test_boxes_of_zeros_of_both_signs(kv):
    """The box after `keep` has the zeros of either sign that appending only the kept gives."""
    rng = np.random.default_rng(5)

    def edit(k, v):
        k.copy_(dev(np.where(rng.random(tuple(k.shape)) < 0.5, -0.0, 0.0), TYPES["bf16"]))
    s = TreeServer(kv, rng, "bf16", 2, 64, 30, 4, 5)
    s.fill([0, 1, 64, 66], edit=edit)
    other = kv.KvCache(30, 2, 64)
    other.pages.copy_(s.cache.pages), other.boxes.copy_(s.cache.boxes)
    new = np.array([7, 9, 12, 5])
    s.draft(new, parents=random_parents(rng, new), edit=edit)
    k, v = s.cache.read(s.step.slots)
    kept = s.keep(agree=1.0)
    start, slots = s.want["q_start"], s.step.slots
    to = [start[r] + i for r in range(4) for i in range(s.past[r] - s.before[r])]
    stay = dev(kept[to], torch.int64)
    other.append(k[stay].contiguous(), v[stay].contiguous(), slots[dev(np.array(to), torch.int64)].contiguous())
    pages = np.unique([s.table[r, j // 64] for r in range(4) for j in range(s.past[r])])
    a, b = (c.boxes[dev(pages, torch.int64)].view(torch.int16) for c in (s.cache, other))
    assert torch.equal(a, b) and (a == 0).any() and (a != 0).any()


def test_trees_into_buffers_with_a_window(kv):
    """Nothing said: the window of `out`; the same said; none, or another, refused."""
    rng = np.random.default_rng(6)
    s = TreeServer(kv, rng, "bf16", 1, 64, 8, 2, 4)
    s.fill([20, 30])
    s.draft([9, 14], window=3)
    parents = dev(s.parents, torch.int32)
    for window in (None, 3):
        out = kv.Tree.empty(len(s.parents), 14, 3)
        assert kv.tree(parents, s.step, window=window, out=out) is out
        assert torch.equal(out.masks, s.tree.masks) and torch.equal(out.positions, s.tree.positions)
    for window in (0, 2):
        with pytest.raises(ValueError):
            kv.tree(parents, s.step, window=window, out=out)
    assert kv.tree(parents, s.step, max_nodes=14).window == 0


def test_projections_with_weights_that_need_gradients(kv):
    """Under no_grad, in place in the rows of a projection, the results are those of detached tensors; outside they are refused."""
    rng = np.random.default_rng(7)
    s = TreeServer(kv, rng, "bf16", 2, 64, 8, 2, 4)
    s.fill([20, 30])
    T = s.draft([9, 14])
    x, weight = rows(rng, "bf16", T, 32)[0], rows(rng, "bf16", 32, 6 * 64, spread=0.2)[0].requires_grad_()
    rotary = kv.Rotary([10000.0 ** (-i / 32) for i in range(32)])
    made = (x @ weight).unflatten(-1, (6, 64))
    with pytest.raises(ValueError, match="gradient"):
        rotary(made[:, :4], made[:, 4:], s.tree.positions)
    with pytest.raises(ValueError, match="gradient"):
        s.cache.tree_attention(made[:, :4], s.step, s.tree)
    q, k = made[:, :4].detach(), made[:, 4:].detach()
    want = rotary(q, k, s.tree.positions)
    lse = torch.zeros(T, 4, device="cuda")
    held = made.detach().clone()
    for call in (lambda: rotary(q, k, s.tree.positions, out=(made[:, :4], k.clone())), lambda: rotary(q, k, s.tree.positions, out=(q.clone(), made[:, 4:])),
                 lambda: s.cache.tree_attention(q, s.step, s.tree, out=made[:, :4]),
                 lambda: s.cache.tree_attention(q, s.step, s.tree, lse=lse.requires_grad_())):
        with pytest.raises(ValueError, match="gradient"):      # nor are results written into what a graph holds
            call()
    assert torch.equal(made, held)
    with torch.no_grad():
        made = (x @ weight).unflatten(-1, (6, 64))
        got = rotary(made[:, :4], made[:, 4:], s.tree.positions, out=(made[:, :4], made[:, 4:]))
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(s.cache.tree_attention(got[0], s.step, s.tree)[0], s.cache.tree_attention(want[0], s.step, s.tree)[0])


def test_the_example_checks_a_step_without_drafts(kv):
    """Server.check of examples/kv_decode.py where no request has new tokens: nothing changes."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import kv_decode
    server = kv_decode.Server(kv_decode.Layer(64, heads=2, kv_heads=1, head_dim=64), 2, 128, n_pages=4)
    x = torch.randn(5, 64, device="cuda").bfloat16()
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    server.step(x, [2, 3])
    y, kept = server.check(x[:0], none, [0, 0], none, lambda y: none)
    assert y.shape == (0, 64) and kept.rows.numel() == 0 and server.lens.tolist() == [2, 3] and int(server.free_state[2]) == 0
