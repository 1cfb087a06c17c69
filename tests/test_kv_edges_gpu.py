"""The cache and sampling calls on the GPU where sizes and arguments end."""
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _torch():
    import torch
    assert torch.cuda.is_available()
    import paper_2602_01027_amd as S
    return torch, S


def test_workspaces_that_are_not_contiguous_gpu_memory_are_refused():
    torch, S = _torch()
    layout = S.sfmp_kv_query(4, 2, 64)
    cache, tables = S.make_kv_cache(layout), S.make_kv_tables(layout, 2, 3)
    x = torch.zeros((2, 2, 64), dtype=torch.float16, device=DEV)
    i, f = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV)
    calls = (lambda w: S.sfmp_kv_attention(cache, 0, tables, i, None, x, x.clone(), 1, 64, 1.0, w),
             lambda w: S.sfmp_kv_reserve(cache, tables, i[:0], None, i[:1], w), lambda w: S.sfmp_kv_compact(cache, tables, i[:1], w),
             lambda w: S.sfmp_sample(torch.zeros((2, 9), device=DEV), None, None, None, None, f, i, f.clone(), w))
    host = torch.zeros((1 << 16) + 256, dtype=torch.uint8)
    host = host[-host.data_ptr() % 256:][:1 << 16]  # (on an address that the library would take)
    for call in calls:
        call(torch.zeros(1 << 16, dtype=torch.uint8, device=DEV))
        for bad in (host, torch.zeros(1, dtype=torch.uint8, device=DEV).expand(1 << 16)):
            with pytest.raises(ValueError, match="workspace has to be"):
                call(bad)
    torch.cuda.synchronize()
