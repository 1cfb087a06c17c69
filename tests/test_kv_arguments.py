"""What the binding of the cache and sampling calls does with arguments before the library sees them (no GPU)."""
import pytest

import paper_2602_01027_amd as S


def test_a_workspace_has_to_be_contiguous_memory_of_the_gpu():
    import torch
    for bad in (torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8).expand(1 << 16), 1 << 20):
        with pytest.raises(ValueError, match="workspace has to be"):
            S.kv._workspace(bad)
    assert S.kv._workspace(None) == (None, 0) and S.kv._workspace(torch.zeros(0)) == (None, 0)
