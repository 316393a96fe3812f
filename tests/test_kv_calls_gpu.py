"""What the calls of `paper_2312_01712_amd.kv` take and refuse, on the GPU: tensors that a server's steps bring with them."""
import numpy as np
import pytest
import torch

import kv_reference as ref
from test_kv_gpu import TYPES, Server, compare, dev, kv, rows  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_step_without_tokens(kv):
    """Requests that wait or end only: rows of no tokens, whatever their strides."""
    s = Server(kv, np.random.default_rng(0), "bf16", 2, 64, 6, 2, 3)
    s.fill([70, 3])
    before = s.cache.pages.clone()
    s.plan([0, -1])
    for q in (torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda"),
              torch.empty_strided((0, 4, 64), (0, 0, 0), dtype=torch.bfloat16, device="cuda"),
              torch.empty(9, 64, 4, dtype=torch.bfloat16, device="cuda")[9:].transpose(1, 2)):
        s.cache.append(q[:, :2], q[:, 2:], s.step.slots)
        assert s.cache.select(q, s.step, 2).shape == (0, 2, 2)
        out, lse = s.cache.attention(q, s.step, max_new=1)
        assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    assert torch.equal(s.cache.pages, before)


def test_a_window_over_a_very_wide_table(kv):
    """So many columns that pages are counted in 31 bits only with the window: the calls' own workspace is enough."""
    rng = np.random.default_rng(1)
    R, H, G = 256, 8, 8
    s = Server(kv, rng, "bf16", H, 64, 2 * R, R, 2)
    s.fill(rng.integers(1, 100, R))
    s.fill([1] * R)
    wide = torch.full((R, 1 << 20), -1, dtype=torch.int32, device="cuda")
    wide[:, :2] = s.d_table
    t = s.step
    step = kv.Step(t.kv_lens, t.q_start, wide, t.slots, t.requests, t.positions, t.free_state)
    q, qn = rows(rng, "bf16", R, H * G, 64)
    for window in (0, 50, 5000):
        out, lse = s.cache.attention(q, step, window=window, max_new=1)
        compare(out, lse, *ref.attention(s.ref, qn, H, s.want, 2 * R, 64 ** -0.5, window), 64, False)


@pytest.mark.parametrize("W,max_new,new", [(12, 1, 1), (400, 1, 1), (12, 70, 70), (400, 70, 70), (12, 300, 300)])
@pytest.mark.parametrize("dtype,gap", [("fp16", 14.0), ("fp16", 17.5), ("bf16", 17.5)])
def test_a_key_far_ahead_of_many(kv, dtype, gap, W, max_new, new):
    """One key's score is `gap` above the others', its value is 0: the result is the others' alone, each with a weight below
    half the smallest step of fp16.  Weights are rounded once, u of each; fp16 weights are held times 2^7 at least, so that what
    its smallest step loses of one is 2^-32 of the largest at most."""
    rng = np.random.default_rng(int(gap) + new)
    s = Server(kv, rng, dtype, 1, 64, 14, 1, W)
    s.gain[:] = 0.05

    def first_ahead(k, v):
        k[:, 0, 0], v[:] = 0.0, (1 + v.abs()) * 40
        k[0, 0, 0], v[0] = 4.0, 0.0

    def others(k, v):
        k[:, 0, 0], v[:] = 0.0, (1 + v.abs()) * 40
    s.fill([500], edit=first_ahead)
    s.fill([new], edit=others)
    q, _ = rows(rng, dtype, new, 2, 64)
    q[:, :, 0] = gap / 4
    qn = q.double().cpu().numpy()
    out, lse = s.cache.attention(q, s.step, scale=1.0, max_new=max_new)
    w_out, w_lse, mass, reach, size = ref.attention(s.ref, qn, 1, s.want, 14, 1.0)
    off, off_lse = ref.bounds(w_out, w_lse, mass, reach, size, 64, dtype == "fp16")
    if dtype == "fp16":
        off = off - 2.0 ** -25 * reach + 2.0 ** -32 * reach
    assert (np.abs(out.double().cpu().numpy() - w_out) <= off).all()
    assert (np.abs(lse.double().cpu().numpy() - w_lse) <= off_lse).all()
    assert (w_out > 4 * off).all()


def test_results_into_rows_that_overlap_are_refused(kv):
    from paper_2312_01712_amd.binding import ERR_INVALID_ARGUMENT, IvfpqError
    s = Server(kv, np.random.default_rng(2), "bf16", 2, 64, 6, 2, 3)
    s.fill([5, 3])
    q, _ = rows(s.rng, "bf16", 8, 4, 64)
    for out in (torch.empty(1, 4, 64, dtype=torch.bfloat16, device="cuda").expand(8, 4, 64),
                torch.empty(8, 1, 64, dtype=torch.bfloat16, device="cuda").expand(8, 4, 64)):
        with pytest.raises(IvfpqError) as e:
            s.cache.attention(q, s.step, out=out)
        assert e.value.status == ERR_INVALID_ARGUMENT
    # rows between each other's, heads outside
    out = torch.empty(4, 8, 64 + 8, dtype=torch.bfloat16, device="cuda").transpose(0, 1)[..., :64]
    got, lse = s.cache.attention(q, s.step, out=out)
    want = ref.attention(s.ref, q.double().cpu().numpy(), 2, s.want, 6, 64 ** -0.5)
    compare(got, lse, *want, 64, False)


def test_every_call_makes_its_device_the_current_one(kv, monkeypatch):
    entered, real = [], torch.cuda.device
    s = Server(kv, np.random.default_rng(3), "bf16", 2, 64, 6, 2, 3)
    monkeypatch.setattr(kv, "_current_device", lambda: 1)  # as if another one were
    monkeypatch.setattr(torch.cuda, "device", lambda index: entered.append(index) or real(index))
    T = s.plan([70, 9])
    q, _ = rows(s.rng, "bf16", T, 4, 64)
    s.cache.append(q[:, :2], q[:, 2:], s.step.slots)
    s.cache.select(q, s.step, 2)
    s.cache.attention(q, s.step)
    assert entered == [0] * 4


def test_numbers_beyond_32_bits_are_refused(kv):
    """Not cut to what is left of them: a window of 2^32 + 1 is not one of 1."""
    s = Server(kv, np.random.default_rng(4), "bf16", 2, 64, 6, 2, 3)
    s.fill([5, 3])
    q, _ = rows(s.rng, "bf16", 8, 4, 64)
    big = (1 << 32) + 1
    for call in (lambda: s.cache.attention(q, s.step, window=big), lambda: s.cache.attention(q, s.step, window=-big),
                 lambda: s.cache.attention(q, s.step, max_new=big), lambda: s.cache.attention_workspace(s.step, 4, max_new=big),
                 lambda: s.cache.attention_workspace(s.step, 4, n_select=big), lambda: s.cache.select(q, s.step, big),
                 lambda: s.cache.select(q, s.step, 2, sinks=big), lambda: s.cache.select(q, s.step, 2, recent=big),
                 lambda: kv.KvCache(1, big, 64), lambda: kv.KvCache(1, 1, big + 63)):
        with pytest.raises(ValueError):
            call()
    s.attend(4, window=(1 << 31) - 1)
    s.attend(4, max_new=(1 << 31) - 1)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("H,D", [(1, 64), (3, 96), (2, 128), (2, 256)])
def test_append_writes_the_same_bytes_in_any_pieces(kv, dtype, H, D):
    """Prompts of every remainder, single tokens, a few at a time, against the same tokens in one call: pages and boxes bit for
    bit, tokens that are not finite among them, rounded rows too."""
    rng = np.random.default_rng(D + H)
    steps = [[0, 1, 63, 64, 65, 130], [1] * 6, [1] * 6, [3, 0, 2, 5, 1, 66], [1] * 6, [7, 70, 4, 1, 128, 2], [2] * 6]
    s = Server(kv, rng, dtype, H, D, 40, 6, 8)
    kept = []
    for new in steps:
        T = s.plan(new)
        k, v = (rows(rng, dtype, T, H, D)[0] for _ in range(2))
        k[T // 2, 0, 5] = float("nan")
        to = torch.zeros_like(k), torch.zeros_like(v)
        s.cache.append(k, v, s.step.slots, rounded=to)
        kept.append((k, v, *to, s.step.slots, s.step.requests, s.step.positions))
    k, v, kr, vr, slots, request, position = (torch.cat(x) for x in zip(*kept))
    order = torch.argsort(request.long() * 10000 + position)
    once = kv.KvCache(40, H, D, TYPES[dtype])
    to = torch.zeros_like(k), torch.zeros_like(v)
    once.append(k[order], v[order], slots[order], rounded=to)
    assert torch.equal(once.pages, s.cache.pages) and torch.equal(once.boxes, s.cache.boxes)
    assert torch.equal(to[0].view(torch.int16), kr[order].view(torch.int16)) and torch.equal(to[1].view(torch.int16), vr[order].view(torch.int16))
    assert int((once.pages != 0).sum()) > 0 and to[0].isnan().any()
