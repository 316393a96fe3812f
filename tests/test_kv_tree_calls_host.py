"""What calls of decoding with drafted tokens refuse before they touch a GPU."""
from types import SimpleNamespace

import pytest
import torch

from paper_2312_01712_amd import kv


@pytest.mark.parametrize("over", [dict(window=0), dict(window=4), dict(max_nodes=6), dict(max_nodes=5, window=0)])
def test_a_tree_that_out_was_not_made_for(over):
    """A window of 0 is none, not whatever `out` has."""
    with pytest.raises(ValueError, match="out was made for"):
        kv.tree(None, None, out=SimpleNamespace(max_nodes=5, window=3), **over)


def needing(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16, requires_grad=True)


def test_inputs_that_need_a_gradient_are_refused():
    """There is no backward pass: results without a graph would lose the gradient without a word."""
    rotary, cache = kv.Rotary([1.0] * 8, device="cpu"), kv.KvCache(2, 1, 64, device="cpu")
    plain, positions = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    some = SimpleNamespace(max_tokens=3, _checked=None)
    calls = [lambda: rotary(needing(3, 2, 64), plain, positions), lambda: rotary(plain, needing(3, 2, 64), positions),
             lambda: cache.tree_attention(needing(3, 2, 64), some, some)]
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="expected a CUDA tensor"):  # the next check
            call()
