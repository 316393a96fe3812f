"""What calls of decoding with drafted tokens refuse before they touch a GPU."""
from types import SimpleNamespace

import pytest

from paper_2312_01712_amd import kv


@pytest.mark.parametrize("over", [dict(window=0), dict(window=4), dict(max_nodes=6), dict(max_nodes=5, window=0)])
def test_a_tree_that_out_was_not_made_for(over):
    """A window of 0 is none, not whatever `out` has."""
    with pytest.raises(ValueError, match="out was made for"):
        kv.tree(None, None, out=SimpleNamespace(max_nodes=5, window=3), **over)
