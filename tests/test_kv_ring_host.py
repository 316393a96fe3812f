"""The ring of free pages without a GPU: the reference of tests/test_kv_ring_gpu.py keeps every page in one place, and the
check that says so finds a rule that puts back what was never taken."""
import numpy as np
import pytest

import kv_reference
import kv_ring_reference as ring

STEPS = [
    # two pages, a request that needs three and ends, three requests of a page each
    (4, 4, 2, [[130, 0, 0, 0], [-1, 0, 0, 0], [0, 64, 0, 0], [0, 0, 64, 0], [0, 0, 0, 64]], [1, 0, 0, 0, 1]),
    # a request that lacked all its pages ends before the one that has them all; both places are taken again
    (3, 9, 8, [[512, 192, 0], [0, -1, 0], [-1, 0, 0], [256, 512, 0]], [3, 0, 0, 4]),
    # pages come free between a request's shortages: -1 between its pages
    (3, 9, 6, [[200, 128, 0], [130, 0, 0], [0, -1, 64], [130, 0, 0], [-1, 0, -1], [384, 0, 0], [-1, 0, 0]], [0, 2, 1, 0, 0, 0, 0]),
]


def run(R, W, n_pages, steps, plan=ring.plan):
    lens, table, pages, state = np.zeros(R, np.int64), np.full((R, W), -1), np.arange(n_pages), np.array([0, n_pages, 0])
    missing = []
    for new in steps:
        x = plan(lens, new, table, pages, state, 4000)
        lens, table, pages, state = x["kv_lens"], x["table"], x["ring"], x["state"]
        missing.append(int(state[2]))
        ring.check(lens, table, pages, state, n_pages)
    return missing


@pytest.mark.parametrize("R,W,n_pages,steps,missing", STEPS)
def test_every_page_is_in_one_place(R, W, n_pages, steps, missing):
    assert run(R, W, n_pages, steps) == missing


@pytest.mark.parametrize("R,W,n_pages,steps,missing", STEPS)
def test_a_ring_of_columns_instead_of_pages_is_found(R, W, n_pages, steps, missing):
    """`kv_reference.plan` puts the columns that a length covers into the ring: right as long as no page is missing."""
    with pytest.raises(AssertionError):
        run(R, W, n_pages, steps, plan=kv_reference.plan)


def test_random_steps_keep_every_page():
    rng = np.random.default_rng(0)
    for _ in range(200):
        R, n_pages = int(rng.integers(1, 9)), int(rng.integers(1, 30))
        steps = [np.where(rng.random(R) < 0.25, -1, rng.integers(0, 200, R)) for _ in range(8)]
        run(R, 8 * 4, n_pages, steps)
