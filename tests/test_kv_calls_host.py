"""Sizes and limits that the host side of the paged 4-bit cache (include/ivfpq_kv.h) promises, without a GPU: addresses are
never read."""
import ctypes

import numpy as np
import pytest

from paper_2312_01712_amd import binding, kv
from test_kv_host import P, attention, cache, rows, step


def workspace(T, R, W, H, G, D, max_new, window=0, n_select=0):
    return kv._lib().ivfpq_kv_attention_workspace_bytes(
        ctypes.byref(cache(kv_heads=H, head_dim=D)), ctypes.byref(step(max_tokens=T, requests=R, table_width=W)),
        ctypes.byref(attention(heads=H * G, max_new=max_new, window=window, n_select=n_select)))


@pytest.mark.parametrize("T,R,W,H,G,max_new,window", [(4000, 4000, 45000, 8, 8, 1, 5000), (256, 256, 1 << 20, 8, 8, 1, 5000),
                                                      (2048, 1, 1 << 20, 8, 4, 2048, 70000)])
def test_workspace_without_a_window_is_enough_with_one(T, R, W, H, G, max_new, window):
    assert workspace(T, R, W, H, G, 128, max_new) >= workspace(T, R, W, H, G, 128, max_new, window) > 0


def test_workspace_without_a_window_is_enough_at_random():
    rng = np.random.default_rng(0)
    wide = lambda low, high: int(np.exp(rng.uniform(np.log(low), np.log(high))))
    for _ in range(40000):
        T, R, W = wide(1, 1 << 20), wide(1, 60000), wide(1, (1 << 20) + 1)
        H, G, D = int(rng.choice([1, 2, 5, 8, 64])), int(rng.choice([1, 3, 8, 16, 40])), int(rng.choice([64, 96, 128, 256]))
        max_new, window = wide(1, T + 1), wide(1, 1 << 27)
        free = workspace(T, R, W, H, G, D, max_new)
        assert free >= workspace(T, R, W, H, G, D, max_new, window) > 0, (T, R, W, H, G, D, max_new, window)


@pytest.mark.parametrize("T,R,W,H,G,D,max_new,n_select", [
    (1 << 21, 1 << 16, 8, 8, 1, 128, 1, 4),      # selected pages: 2^24 units of 256 threads
    (1 << 24, 1 << 16, 8, 1, 16, 64, 1, 4),
    (1 << 24, 1, 8, 16, 1, 64, 1, 0),            # a tile of 16 rows each
    (1 << 24, 1 << 16, 8, 130, 1, 64, 4096, 0),  # 256 rows, 512 threads
    (1 << 22, 1 << 16, 8, 260, 1, 256, 4096, 0)])  # 128 rows, 512 threads
def test_attention_refuses_launches_of_2_32_threads(T, R, W, H, G, D, max_new, n_select):
    a = attention(heads=H * G, max_new=max_new, n_select=n_select, selected=P if n_select else None)
    c, s = cache(kv_heads=H, head_dim=D), step(max_tokens=T, requests=R, table_width=W)
    rc = kv._lib().ivfpq_kv_attention(ctypes.byref(c), ctypes.byref(s), ctypes.byref(a), 0x10000, 1 << 50, None)
    assert rc == binding.ERR_UNSUPPORTED and "one launch" in binding.last_error()


@pytest.mark.parametrize("T,R,W,H,G", [(1 << 24, 1 << 16, 8, 1, 1),     # 2^24 workgroups pick, of 256 threads
                                       (1 << 22, 1 << 16, 2000, 1, 1),  # 2^22 of 1024
                                       (1 << 21, 1 << 16, 8, 128, 16),  # scores: a workgroup a token and head
                                       (1 << 20, 1, 20000, 8, 8)])
def test_select_refuses_launches_of_2_32_threads(T, R, W, H, G):
    c, s = cache(kv_heads=H), step(max_tokens=T, requests=R, table_width=W)
    rc = kv._lib().ivfpq_kv_select(ctypes.byref(c), ctypes.byref(s), rows(), H * G, 4, 1, 1, P, 0x10000, 1 << 60, None)
    assert rc == binding.ERR_UNSUPPORTED and "one launch" in binding.last_error()
