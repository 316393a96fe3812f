"""Decoding with drafted tokens without a GPU: structs match the header's, the host side refuses what the kernels could not take, phases
of rotary positions are the fractions of a turn that they stand for, and the reference of the GPU tests agrees with itself."""
import ctypes
import os
import subprocess
from decimal import Decimal, getcontext

import numpy as np
import pytest

import kv_tree_reference as tref
from paper_2312_01712_amd import binding, kv
from test_kv_host import BAD, P, ROOT, UNSUPPORTED, WORKSPACE, attention, cache, rows, step


def test_structs_match(tmp_path):
    src, exe = tmp_path / "use.c", tmp_path / "use"
    src.write_text('#include <stdio.h>\n#include "ivfpq_kv.h"\nint main(void) {\n'
                   '  printf("%zu %zu %zu %d %d\\n", sizeof(ivfpq_kv_rotary), sizeof(ivfpq_kv_tree), sizeof(ivfpq_kv_out_rows),\n'
                   "         IVFPQ_KV_MAX_NODES, IVFPQ_KV_MAX_AXES);\n  return 0;\n}\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"),
                    str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(kv._Rotary), ctypes.sizeof(kv._Tree), ctypes.sizeof(kv._Rows), kv.MAX_NODES, kv.MAX_AXES]


def tree(**over):
    return kv._Tree(**{**dict(max_nodes=70, window=0, masks=P, positions=P + 64), **over})


def rotary(**over):
    return kv._Rotary(**{**dict(head_dim=128, turned=64, neighbours=0, dtype=0, axes=3, phases=P, axis=P), **over})


@pytest.mark.parametrize("s,t,status", [
    (dict(requests=-1), {}, BAD), (dict(max_tokens=-1), {}, BAD), (dict(q_start=None), {}, BAD), (dict(positions=None), {}, BAD),
    ({}, dict(max_nodes=0), BAD), ({}, dict(max_nodes=1025), BAD), ({}, dict(window=-1), BAD), ({}, dict(masks=None), BAD),
    ({}, dict(masks=P + 4), BAD), ({}, dict(positions=None), BAD), ({}, dict(positions=P), BAD)])
def test_tree_plan_refuses(s, t, status):
    lib = kv._lib()
    assert lib.ivfpq_kv_tree_plan(ctypes.byref(step(**s)), P, ctypes.byref(tree(**t)), None) == status and binding.last_error() != ""
    assert lib.ivfpq_kv_tree_plan(ctypes.byref(step()), None, ctypes.byref(tree()), None) == BAD
    assert lib.ivfpq_kv_tree_plan(None, P, ctypes.byref(tree()), None) == BAD
    assert lib.ivfpq_kv_tree_plan(ctypes.byref(step()), P, None, None) == BAD
    assert lib.ivfpq_kv_tree_plan(ctypes.byref(step(max_tokens=0)), None, ctypes.byref(tree(masks=None)), None) == 0


@pytest.mark.parametrize("c,s,a,t,status", [
    (dict(head_dim=80), {}, {}, {}, UNSUPPORTED), (dict(pages=None), {}, {}, {}, BAD), ({}, dict(table=None), {}, {}, BAD),
    ({}, {}, dict(heads=7), {}, BAD), ({}, {}, dict(scale=float("nan")), {}, BAD), ({}, {}, dict(selected=P, n_select=1), {}, BAD),
    ({}, {}, dict(n_select=1), {}, BAD), ({}, {}, dict(q=rows(P + 2)), {}, BAD), ({}, {}, dict(out=None), {}, BAD),
    ({}, {}, dict(out_token_stride=8), {}, BAD), ({}, {}, {}, dict(max_nodes=0), BAD), ({}, {}, {}, dict(masks=None), BAD),
    ({}, {}, {}, dict(window=-5), BAD), ({}, dict(max_tokens=1 << 24, table_width=1 << 20), dict(heads=2048), {}, UNSUPPORTED),
    ({}, dict(table_width=100), {}, {}, WORKSPACE)])
def test_tree_attention_refuses(c, s, a, t, status):
    lib = kv._lib()
    rc = lib.ivfpq_kv_tree_attention(ctypes.byref(cache(**c)), ctypes.byref(step(**s)), ctypes.byref(attention(**a)), ctypes.byref(tree(**t)),
                                     None, 0, None)
    assert rc == status and binding.last_error() != ""


def keep(caches=None, n=None, s=None, t=None, drafted=P, picked=P, free=P, capacity=4, state=P, state_out=P + 64, lens=P + 128, kept=P, counts=P + 256):
    caches = [cache()] if caches is None else caches
    s, t = step() if s is None else s, tree() if t is None else t
    return kv._lib().ivfpq_kv_keep((kv._Cache * len(caches))(*caches), len(caches) if n is None else n, ctypes.byref(s), ctypes.byref(t), drafted,
                                   picked, free, capacity, state, state_out, lens, kept, counts, None)


@pytest.mark.parametrize("over", [
    dict(n=0), dict(n=-1), dict(n=1025), dict(caches=[cache(), cache()]), dict(caches=[cache(), cache(pages=2 * P, boxes=2 * P, kv_heads=3)]),
    dict(caches=[cache(), cache(pages=2 * P, boxes=P)]), dict(caches=[cache(dtype=7)]), dict(s=step(requests=-1)), dict(s=step(slots=None)),
    dict(s=step(kv_lens=None)), dict(t=tree(window=4)), dict(t=tree(masks=None)), dict(drafted=None), dict(picked=None), dict(free=None),
    dict(capacity=0), dict(capacity=1 << 26), dict(state=None), dict(state_out=None), dict(state_out=P), dict(lens=None), dict(kept=None),
    dict(counts=None), dict(lens=P), dict(counts=P), dict(counts=P + 128)])
def test_keep_refuses(over):
    assert keep(**over) == BAD and binding.last_error() != ""


@pytest.mark.parametrize("r,q,heads,k,kv_heads,positions,tokens,q_out,status", [
    (dict(head_dim=80), rows(), 8, rows(), 2, P, 4, rows(), UNSUPPORTED), (dict(turned=0), rows(), 8, rows(), 2, P, 4, rows(), BAD),
    (dict(turned=24), rows(), 8, rows(), 2, P, 4, rows(), BAD), (dict(turned=144), rows(), 8, rows(), 2, P, 4, rows(), BAD),
    (dict(dtype=2), rows(), 8, rows(), 2, P, 4, rows(), BAD), (dict(axes=0), rows(), 8, rows(), 2, P, 4, rows(), BAD),
    (dict(axes=9), rows(), 8, rows(), 2, P, 4, rows(), BAD), (dict(phases=None), rows(), 8, rows(), 2, P, 4, rows(), BAD),
    (dict(axis=None), rows(), 8, rows(), 2, P, 4, rows(), BAD), ({}, rows(None), 8, rows(), 2, P, 4, rows(), BAD),
    ({}, rows(P + 8), 8, rows(), 2, P, 4, rows(), BAD), ({}, rows(P, 1028), 8, rows(), 2, P, 4, rows(), BAD),
    ({}, rows(), -1, rows(), 2, P, 4, rows(), BAD), ({}, rows(), 8, rows(), -2, P, 4, rows(), BAD), ({}, rows(), 8, rows(), 2, None, 4, rows(), BAD),
    ({}, rows(), 8, rows(), 2, P, -1, rows(), BAD), ({}, rows(), 8, rows(), 2, P, (1 << 24) + 1, rows(), BAD),
    ({}, rows(), 8, rows(), 2, P, 4, rows(P, 0, 128), BAD), ({}, rows(), 8, rows(None), 2, P, 4, rows(), BAD)])
def test_rotate_refuses(r, q, heads, k, kv_heads, positions, tokens, q_out, status):
    lib = kv._lib()
    rc = lib.ivfpq_kv_rotate(ctypes.byref(rotary(**r)), q, heads, k, kv_heads, positions, 4, tokens, q_out, rows(), None)
    assert rc == status and binding.last_error() != ""


def test_rotate_of_nothing():
    lib = kv._lib()
    assert lib.ivfpq_kv_rotate(ctypes.byref(rotary()), rows(None), 8, rows(None), 2, None, 0, 0, rows(None), rows(None), None) == 0
    assert lib.ivfpq_kv_rotate(ctypes.byref(rotary()), rows(None), 0, rows(None), 0, None, 0, 9, rows(None), rows(None), None) == 0


@pytest.mark.parametrize("c,slots,tokens,k,v,status", [
    (dict(head_dim=80), P, 4, rows(), rows(), UNSUPPORTED), (dict(boxes=None), P, 4, rows(), rows(), BAD), ({}, None, 4, rows(), rows(), BAD),
    ({}, P, -1, rows(), rows(), BAD), ({}, P, (1 << 24) + 1, rows(), rows(), BAD), ({}, P, 4, rows(None), rows(), BAD),
    ({}, P, 4, rows(), rows(P + 4), BAD), ({}, P, 4, rows(P, 64), rows(), BAD), ({}, P, 4, rows(), rows(P, 1024, 0), BAD)])
def test_read_refuses(c, slots, tokens, k, v, status):
    assert kv._lib().ivfpq_kv_read(ctypes.byref(cache(**c)), slots, tokens, k, v, None) == status and binding.last_error() != ""
    assert kv._lib().ivfpq_kv_read(ctypes.byref(cache()), None, 0, rows(None), rows(None), None) == 0


def test_phases():
    """round(f / (2 pi) 2^64) against 60 decimal digits."""
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    frequencies = [1.0, 500000.0 ** (-1 / 3), 1e-7, -0.25, 6.283185307179586, 12345.678, 0.0, 2.0 ** -60]
    try:
        got = kv.Rotary(frequencies, device="cpu")
    except Exception as e:  # pragma: no cover
        pytest.fail(f"tables need no GPU: {e}")
    for f, x in zip(frequencies, got._phases.tolist()):
        want = Decimal(f) / (2 * pi) * (1 << 64)
        want = int(want.to_integral_value()) % (1 << 64)
        assert min((x - want) % (1 << 64), (want - x) % (1 << 64)) <= 1


def test_reference_trees():
    """Masks are closed under ancestors, depths count them, words hold the bits; a window cuts from the far end."""
    rng = np.random.default_rng(0)
    n = 150
    parents = np.floor(rng.random(n) * np.arange(n)).astype(int) - (rng.random(n) < 0.1)
    parents[0] = -1
    s = dict(positions=np.arange(n) + 20, q_start=[0, n])
    sees, positions = tref.tree(parents, s, n)
    for i in range(n):
        p = parents[i] if 0 <= parents[i] < i else -1
        own = np.zeros(n, bool)
        own[i] = True
        assert np.array_equal(sees[i], own | (sees[p] if p >= 0 else False)) and positions[i] == 20 + sees[i].sum() - 1
    w = tref.words(sees)
    assert all(bool(int(w[i, j // 64]) >> (j % 64) & 1) == sees[i, j] for i in range(0, n, 7) for j in range(n))
    near, _ = tref.tree(parents, s, n, window=3)
    assert (near.sum(1) == np.minimum(sees.sum(1), 3)).all() and (near <= sees).all()


def test_reference_paths():
    sees, _ = tref.tree(np.array([-1, 0, 0, 2, 2, 3]), dict(positions=np.arange(6), q_start=[0, 6]), 6)
    stored = np.ones(6, bool)
    drafted = np.array([9, 1, 2, 3, 4, 5])
    assert tref.path_of(sees, drafted, np.array([2, 0, 3, 5, 0, 0]), stored) == [0, 2, 3, 5]
    assert tref.path_of(sees, drafted, np.array([2, 0, 4, 5, 0, 0]), stored) == [0, 2, 4]
    assert tref.path_of(sees, drafted, np.array([7, 0, 4, 5, 0, 0]), stored) == [0]
    stored[3] = False
    assert tref.path_of(sees, drafted, np.array([2, 0, 3, 5, 0, 0]), stored) == [0, 2]


def test_reference_rotation():
    """Turning by p and then by -p is nothing; lengths stay; one whole turn in four steps."""
    rng = np.random.default_rng(1)
    x, f = rng.normal(size=(5, 2, 16)), [1.0, 0.5, 0.1, 0.01, 2.0, 3.0, 4.0, 5.0]
    p = rng.integers(0, 10 ** 6, (1, 5))
    for neighbours in (False, True):
        y, _ = tref.rotate(x, p, f, [0] * 8, neighbours)
        z, _ = tref.rotate(y, -p, f, [0] * 8, neighbours)
        assert np.allclose(z, x, atol=1e-12) and np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    quarter, _ = tref.rotate(x, np.full((1, 5), 1), [np.pi / 2] * 8, [0] * 8, False)
    assert np.allclose(quarter[..., :8], -x[..., 8:]) and np.allclose(quarter[..., 8:], x[..., :8])
