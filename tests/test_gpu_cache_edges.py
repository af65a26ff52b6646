"""Where a cache's attention can go wrong at the ends of what it takes: scales of pages without a token."""
import pytest
import torch

from test_gpu_cache_attn import _attend

pytestmark = pytest.mark.gpu


# ---- scales of pages that hold no token

@pytest.mark.parametrize("byte", [255, 0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_scales_of_pages_without_a_token_are_not_used(dtype, D, byte):
    """What a program has not set yet: of the page behind a sequence's end, in the same block of keys, and of page 0, which stands in for
    those that are not there."""
    seed = next(s for s in range(200) if 0 not in torch.randperm(10, generator=torch.Generator().manual_seed(s))[[0, 1, 2, 4, 5, 6]])
    change = lambda case: case.spoil_scales(byte)
    for counts in ([1, 1], [5, 3], [40, 20], [41, 1]):
        how = dict(Hq=4, Hkv=1, D=D, seed=seed, change=change)
        case, *_ = _attend(dtype, "e4m3", [41, 33], counts, **how)
        assert not (case.scales[0][0] != byte).any()
        table = case.table.clone()
        table[0, 1], table[1, 0] = -1, 10 ** 6
        _attend(dtype, "e4m3", [41, 33], counts, table=table, **how)
        _attend(dtype, "e4m3", [41, 33], counts, causal=False, window=20, **how)
    how = dict(Hq=4, Hkv=1, D=D, change=change)
    _attend(dtype, "e4m3", [200, 130], [110, 90], **how)
    _attend(dtype, "e4m3", [5001, 1200], [1, 1], **how)                           # walks in shares
