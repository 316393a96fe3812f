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
    a = attention(heads=H * G, max_new=max_new, n_select=n_select, selected=P if n_select else None, out_token_stride=H * G * D,
                  out_head_stride=D)
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


@pytest.mark.parametrize("T,heads,D,token,head,meet", [
    (3, 8, 128, 0, 128, True), (3, 8, 128, 1024, 0, True), (3, 8, 128, 1016, 128, True), (3, 8, 128, 1024, 120, True),
    (3, 8, 128, 128, 128, True), (1, 8, 128, 0, 120, True), (2, 1, 128, 64, 0, True), (3, 8, 128, -1016, 128, True),
    (3, 8, 64, 192, 192 * 2, True), (3, 8, 64, 168, 256, False), (3, 8, 64, 168, 200, True),
    (3, 8, 128, 1024, 128, False), (3, 8, 128, 128, 384, False), (3, 8, 128, -1024, 128, False), (1, 8, 128, 0, 128, False),
    (1, 1, 128, 0, 0, False), (2, 1, 128, 128, 0, False), (5, 8, 128, 1 << 60, 1 << 61, True), (2, 8, 128, 1 << 60, 1 << 61, False), (3, 8, 64, 1 << 62, 64, False)])
def test_rows_of_results_must_not_overlap(T, heads, D, token, head, meet):
    """Refused before the workspace is looked at; what does not overlap gets that far.  The expectations are those of all
    addresses written out."""
    at = [t * token + h * head for t in range(T) for h in range(heads)]
    at.sort()
    assert meet == any(b - a < D for a, b in zip(at, at[1:]))
    a = attention(heads=heads, out_token_stride=token, out_head_stride=head)
    rc = kv._lib().ivfpq_kv_attention(ctypes.byref(cache(kv_heads=1, head_dim=D)), ctypes.byref(step(max_tokens=T)), ctypes.byref(a),
                                      None, 0, None)
    assert rc == (binding.ERR_INVALID_ARGUMENT if meet else binding.ERR_WORKSPACE)
    assert ("overlap" in binding.last_error()) == meet


def test_calls_go_to_the_device_of_their_tensors(monkeypatch):
    """Another device is current: the tensors' one is while the library is called, with its stream."""
    current, log = [1], []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.was, current[0] = current[0], self.index

        def __exit__(self, *_):
            current[0] = self.was

    monkeypatch.setattr(kv, "_current_device", lambda: current[0])
    monkeypatch.setattr(kv.torch.cuda, "device", Device)
    monkeypatch.setattr(kv, "_raw_stream", lambda device: 0x100 + device)

    def call(*args):
        log.append((current[0], args))
        return binding.OK
    kv._launch(0, call, 7, 8)
    kv._launch(1, call, 9)
    assert log == [(0, (7, 8, 0x100)), (1, (9, 0x101))] and current == [1]
