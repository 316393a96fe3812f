"""The paged 4-bit cache without a GPU: the library exports what include/ivfpq_kv.h declares, the header is plain C, the
host side refuses what the kernels could not take, the reference of the GPU tests agrees with itself, and the page layout
has a place of its own for every value."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

import kv_reference as ref
from paper_2312_01712_amd import binding, kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BAD, UNSUPPORTED, WORKSPACE = binding.ERR_INVALID_ARGUMENT, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "ivfpq_kv.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(ivfpq_kv_[a-z_0-9]+)\s*\(", text)))
    assert sorted(kv.SYMBOLS) == names
    lib = kv._lib()
    for n in names:
        assert getattr(lib, n) is not None


def test_header_is_plain_c_and_structs_match(tmp_path):
    src, exe = tmp_path / "use.c", tmp_path / "use"
    src.write_text('#include <stdio.h>\n#include "ivfpq_kv.h"\nint main(void) {\n'
                   '  printf("%zu %zu %zu %zu %d %d %d\\n", sizeof(ivfpq_kv_cache), sizeof(ivfpq_kv_step), sizeof(ivfpq_kv_rows),\n'
                   "         sizeof(ivfpq_kv_attention_args), IVFPQ_KV_PAGE, IVFPQ_KV_MAX_REQUESTS, IVFPQ_KV_MAX_SELECT);\n  return 0;\n}\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"),
                    str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(kv._Cache), ctypes.sizeof(kv._Step), ctypes.sizeof(kv._Rows), ctypes.sizeof(kv._Attention),
                   kv.PAGE, kv.MAX_REQUESTS, kv.MAX_SELECT]


# addresses that are never read: every call below is refused before anything is enqueued
P = 0x10000


def cache(**over):
    return kv._Cache(**{**dict(n_pages=4, kv_heads=2, head_dim=128, dtype=0, pages=P, boxes=P), **over})


def step(**over):
    return kv._Step(**{**dict(requests=2, max_tokens=3, table_width=4, kv_lens=P, q_start=P, table=P, slots=P, token_req=P,
                              positions=P), **over})


def rows(data=P, token=1024, head=128):
    return kv._Rows(data, token, head)


def attention(**over):
    return kv._Attention(**{**dict(q=rows(), heads=8, max_new=1, scale=0.1, window=0, selected=None, n_select=0, out=P,
                                   out_token_stride=1024, out_head_stride=128, lse=P), **over})


@pytest.mark.parametrize("c,s,a,status", [
    (dict(head_dim=80), {}, {}, UNSUPPORTED), (dict(kv_heads=0), {}, {}, BAD), (dict(n_pages=0), {}, {}, BAD),
    (dict(n_pages=1 << 26), {}, {}, BAD), (dict(dtype=2), {}, {}, BAD), (dict(pages=None), {}, {}, BAD),
    (dict(pages=P + 8), {}, {}, BAD), (dict(boxes=P + 2), {}, {}, BAD),
    ({}, dict(requests=-1), {}, BAD), ({}, dict(requests=65537), {}, BAD), ({}, dict(max_tokens=-1), {}, BAD),
    ({}, dict(table_width=0), {}, BAD), ({}, dict(table=None), {}, BAD), ({}, dict(positions=None), {}, BAD),
    ({}, {}, dict(heads=7), BAD), ({}, {}, dict(heads=0), BAD), ({}, {}, dict(max_new=0), BAD), ({}, {}, dict(window=-1), BAD),
    ({}, {}, dict(scale=float("inf")), BAD), ({}, {}, dict(n_select=3), BAD), ({}, {}, dict(selected=P), BAD),
    ({}, {}, dict(selected=P, n_select=1025), BAD), ({}, {}, dict(q=rows(None)), BAD), ({}, {}, dict(q=rows(P + 2)), BAD),
    ({}, {}, dict(q=rows(P, 1023)), BAD), ({}, {}, dict(q=rows(P, 1024, 4)), BAD), ({}, {}, dict(out=None), BAD),
    ({}, {}, dict(out_token_stride=4), BAD), ({}, {}, {}, WORKSPACE)])
def test_attention_refuses(c, s, a, status):
    lib = kv._lib()
    rc = lib.ivfpq_kv_attention(ctypes.byref(cache(**c)), ctypes.byref(step(**s)), ctypes.byref(attention(**a)), None, 0, None)
    assert rc == status and binding.last_error() != ""


@pytest.mark.parametrize("n,sinks,recent,status", [(0, 0, 0, BAD), (1025, 1, 1, BAD), (2, 3, 0, BAD), (2, 1, 2, BAD),
                                                   (2, -1, 1, BAD), (2, 1, -1, BAD), (2, 1, 1, WORKSPACE)])
def test_select_refuses(n, sinks, recent, status):
    rc = kv._lib().ivfpq_kv_select(ctypes.byref(cache()), ctypes.byref(step()), rows(), 8, n, sinks, recent, P, None, 0, None)
    assert rc == status and binding.last_error() != ""


def test_append_and_plan_refuse():
    lib = kv._lib()
    c = ctypes.byref(cache())
    assert lib.ivfpq_kv_append(c, rows(), rows(), None, 3, None, None, None) == BAD
    assert lib.ivfpq_kv_append(c, rows(), rows(P + 4), P, 3, None, None, None) == BAD
    assert lib.ivfpq_kv_append(c, rows(), rows(), P, -1, None, None, None) == BAD
    assert lib.ivfpq_kv_append(c, rows(), rows(), P, 3, P + 2, None, None) == BAD
    assert lib.ivfpq_kv_append(None, rows(), rows(), P, 3, None, None, None) == BAD
    assert lib.ivfpq_kv_append(c, rows(None), rows(None), None, 0, None, None, None) == binding.OK
    args = dict(past=P, new=P, ring=P, capacity=8, state=P, state_out=P + 64)
    def plan(over_step={}, **over):
        return lib.ivfpq_kv_plan(ctypes.byref(step(kv_lens=P + 64, **over_step)), *{**args, **over}.values(), None)
    for over in (dict(requests=-1), dict(table=None), dict(q_start=None), dict(slots=None), dict(table_width=0), dict(max_tokens=-1)):
        assert plan(over) == BAD, over
    for over in (dict(past=None), dict(ring=None), dict(capacity=0), dict(state=None), dict(state_out=P), dict(past=P + 64)):
        assert plan(**over) == BAD, over
    assert lib.ivfpq_kv_plan(None, *args.values(), None) == BAD
    assert lib.ivfpq_kv_select_workspace_bytes(None, None, 1) == 0
    assert lib.ivfpq_kv_attention_workspace_bytes(None, None, None) == 0
    assert lib.ivfpq_kv_page_bytes(8, 128) == 8 * 68 * 128 and lib.ivfpq_kv_page_bytes(8, 100) == 0 and lib.ivfpq_kv_page_bytes(0, 64) == 0


@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_page_layout_has_a_place_for_every_value(D):
    """The addresses of include/ivfpq_kv.h: no two nibbles or scale bytes of a page and head meet, none is left over, and no
    byte belongs to two tokens."""
    seen, owner = set(), {}
    for t in range(64):
        for c in range(D):
            for nib, at in ((c & 1, t * D // 2 + c // 2),
                            ((c // 16) & 1, 34 * D + (c // 32) * 1024 + (((t // 4) % 4) * 16 + c % 16) * 16 + (t // 16) * 4 + t % 4)):
                assert (at, nib) not in seen
                seen.add((at, nib))
                assert owner.setdefault(at, t) == t
        for p in range(D // 32):
            for at in (32 * D + ((t % 16) * (D // 32) + p) * 4 + t // 16, 66 * D + p * 64 + ((t // 4) % 4) * 16 + (t // 16) * 4 + t % 4):
                assert (at, 0) not in seen
                seen.update({(at, 0), (at, 1)})
    assert seen == {(at, n) for at in range(68 * D) for n in (0, 1)}


def test_reference_rounds_to_the_nearest():
    """The reference's rounding against all eight candidates, ties by hand."""
    rng = np.random.default_rng(0)
    x = rng.normal(size=(50, 64)) * np.exp2(rng.integers(-20, 20, (50, 1)))
    code, b, value = ref.quantise(x)
    unit = np.repeat(np.ldexp(1.0, b.astype(int) - 127), 32, -1)
    best = np.abs(np.abs(x)[..., None] / unit[..., None] - ref.GRID).min(-1)
    assert np.allclose(np.abs(x - value) / unit, best)
    top = np.abs(x).reshape(50, -1, 32).max(-1) / np.ldexp(1.0, b.astype(int) - 127)
    assert ((top >= 4) & (top < 8)).all()
    row = np.zeros(32)
    row[:9] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0]
    assert ref.quantise(row)[2][:9].tolist() == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -4.0]
    row[0] = 7.9
    assert ref.quantise(row)[2][0] == 6.0


def test_reference_attention_is_a_softmax():
    """The reference over a tiny cache against a softmax written out for one row, and a score by hand."""
    rng = np.random.default_rng(1)
    c = ref.Cache(3, 1, 64)
    step = ref.plan([0], [70], np.full((1, 2), -1), np.array([2, 0, 1]), np.array([0, 3, 0]), 70)
    k, v = rng.normal(size=(70, 1, 64)), rng.normal(size=(70, 1, 64))
    c.append(k, v, step["slots"])
    assert step["table"].tolist() == [[2, 0]] and step["slots"][69] == 5
    q = rng.normal(size=(70, 2, 64))
    out, lse, *_ = ref.attention(c, q, 1, step, 3, 0.125)
    kk, vv = ref.quantise(k[:, 0])[2], ref.quantise(v[:, 0])[2]
    w = np.exp(q[69, 1] @ kk.T * 0.125)
    assert np.allclose(out[69, 1], w @ vv / w.sum()) and np.isclose(lse[69, 1], np.log(w.sum()))
    assert np.allclose(out[0, 0], vv[0])
    assert (ref.select(c, q, 1, step, 3, 1, 0, 1)[:64] == 0).all() and (ref.select(c, q, 1, step, 3, 1, 0, 1)[64:] == 1).all()
