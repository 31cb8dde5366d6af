"""The serving operators' binding and argument checks at their edges, on the
CPU (nothing is launched)."""
import os

import pytest
import torch

from paper_2609_39361_amd import lamp

pytestmark = pytest.mark.skipif(not os.path.exists(lamp.LIB_PATH), reason="liblamp.so not built")


@pytest.mark.parametrize("shape", [(0, 64), (4, 0), (0, 0)])
def test_an_empty_rope_table_is_refused(shape):
    """(An empty tensor has no address, which the library takes as "not rotated".)"""
    with pytest.raises(ValueError, match="rope"):
        lamp._rope(torch.empty(shape), -1)
    with pytest.raises(ValueError, match="rope"):
        lamp._rope(torch.ones(4, 64)[:shape[0], :shape[1]].contiguous(), -1)
    assert lamp._rope(None, -1) == (None, 0, 0)


def test_workspace_size_of_tables_without_columns():
    """attn_cache accepts them, so the size says what such a call needs: the plan of more than 256 sequences."""
    size = lamp.attn_cache_workspace_size
    assert size(256, 256, 4, 1, 64, 16, 0) == 0 and size(3, 2, 4, 1, 64, 16, 0) == 0
    assert size(300, 300, 4, 1, 64, 16, 0) == size(300, 300, 4, 1, 64, 16, 1) > 0
    assert size(300, 300, 4, 1, 64, 16, -1) == 0
