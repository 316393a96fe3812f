"""Page tables on the GPU in steps after pages ran out, against tests/kv_ring_reference.py: every page is in one table or in
the ring, once, whatever ended in which order."""
from unittest import mock

import numpy as np
import pytest
import torch

import kv_reference as ref
import kv_ring_reference as ring
from test_kv_gpu import Server, dev, kv  # noqa: F401
from test_kv_ring_host import STEPS

pytestmark = pytest.mark.gpu


class RingServer(Server):
    def plan(self, new, max_tokens=None):
        with mock.patch.object(ref, "plan", ring.plan):
            T = super().plan(new, max_tokens)
        ring.check(self.past, self.table, self.ring, self.state, self.n_pages)
        return T


@pytest.mark.parametrize("R,W,n_pages,steps,missing", STEPS)
def test_steps_after_a_shortage(kv, R, W, n_pages, steps, missing):
    """Tokens too: what a request appends and looks at is its own."""
    s = RingServer(kv, np.random.default_rng(1), "bf16", 1, 64, n_pages, R, W)
    for new, short in zip(steps, missing):
        if max(new) > 0:
            s.fill(new)
            s.attend(2)
        else:
            s.plan(new)
        assert s.state[2] == short


@pytest.mark.parametrize("R,longest,share,seed", [(3, 400, 0.15, 0), (15, 900, 0.2, 1), (16, 900, 0.2, 2), (63, 300, 0.25, 3),
                                                  (64, 2000, 0.25, 4), (300, 300, 0.25, 5), (9, 30000, 0.2, 6), (70, 12000, 0.2, 7)])
def test_random_steps_short_of_pages(kv, R, longest, share, seed):
    """Fewer pages than the requests need, from a few requests that every workgroup counts to many, rows of a few columns to
    hundreds; the ring goes round, and requests end that have some of their pages."""
    rng = np.random.default_rng(seed)
    W = 3 * longest // 64 + 4
    n_pages = int(R * W * share) + 1
    s = RingServer(kv, rng, "bf16", 1, 64, n_pages, R, W, ring_start=n_pages - 1, held=False)
    partly = 0
    for i in range(8):
        new = rng.integers(0, longest + 1, R)
        new[s.past + new > 64 * W] = 0
        new[rng.random(R) < 0.3] = -1
        rows = [s.table[r, :-(-int(s.past[r]) // 64)] for r in np.flatnonzero(new < 0)]
        partly += sum(bool((x < 0).any() and (x >= 0).any()) for x in rows)
        s.plan(new, max_tokens=int(np.maximum(new, 0).sum()) + 3)
    assert partly > 0


@pytest.mark.parametrize("R", [3, 40, 80, 300])
def test_a_step_without_room_to_count(kv, R):
    """`counts` of the step NULL: the same step."""
    rng = np.random.default_rng(R)
    s = RingServer(kv, rng, "bf16", 1, 64, R * 4, R, 12, held=False)
    s.plan(rng.integers(0, 700, R))
    new = np.where(rng.random(R) < 0.5, -1, 3)
    T = int(np.maximum(new, 0).sum())
    step = kv.Step.empty(R, T, s.d_table.clone())
    step._c.counts = None
    free, table = s.d_ring.clone(), step.table
    kv.plan(s.d_past, dev(new, torch.int32), table, free, s.d_state, out=step)
    s.plan(new)
    assert torch.equal(table, s.d_table) and torch.equal(free, s.d_ring) and torch.equal(step.free_state, s.step.free_state)
    assert torch.equal(step.slots, s.step.slots) and torch.equal(step.kv_lens, s.step.kv_lens)


def test_a_step_done_again_after_a_shortage(kv):
    """From the same lengths and state with fewer new tokens: as if the first had not been."""
    s = RingServer(kv, np.random.default_rng(2), "bf16", 1, 64, 6, 3, 6)
    s.plan([200, 64, 0])
    past, table, pages, state = s.past, s.table, s.ring, s.state
    d_past, d_state = s.d_past, s.d_state
    s.plan([100, -1, 200])
    assert s.state[2] == 4
    s.past, s.table, s.ring, s.state, s.d_past, s.d_state = past, s.table, s.ring, state, d_past, d_state
    s.plan([0, -1, 60])
    assert s.state[2] == 0


def test_a_ring_without_room_keeps_what_it_has(kv):
    """A ring smaller than the pages that come back: pages that wait in it stay, the others are dropped."""
    table = torch.tensor([[7, 8, 9], [-1, -1, -1]], dtype=torch.int32, device="cuda")
    free = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device="cuda")
    past, new = dev([192, 0], torch.int32), dev([-1, 64], torch.int32)
    step = kv.plan(past, new, table, free, dev([0, 3, 0], torch.int64), max_tokens=64)
    assert step.free_state.tolist() == [1, 4, 0] and free.tolist() == [1, 2, 3, 7] and table[1, 0] == 1
    step = kv.plan(past, new, table, free, dev([0, 9, 0], torch.int64), max_tokens=64)  # counters that claim too much
    assert step.free_state.tolist() == [1, 9, 0] and free.tolist() == [1, 2, 3, 7]
