"""What the calls of `paper_2312_01712_amd.kv` take and refuse, on the GPU: tensors that a server's steps bring with them."""
import numpy as np
import pytest
import torch

from test_kv_gpu import Server, kv  # noqa: F401

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
