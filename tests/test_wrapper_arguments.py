"""Arguments that the wrapper hands to the C ABI as numbers: what does not fit is refused, not cut off (CPU)."""
import pytest
import pytest
import torch

import paper_2407_00611_amd as st
from paper_2407_00611_amd import api


def test_a_workspace_that_ends_before_its_first_boundary_is_empty():
    """A negative number of bytes would be taken for more than any call needs, and the kernels would write behind the buffer."""
    buf = torch.empty(2048, dtype=torch.uint8)
    start = -buf.data_ptr() % 256
    for skip in (0, 1, 100, 255):
        for n in (0, 1, 10, 156, 255, 256, 300):
            ptr, size = api._aligned(buf[start + skip:start + skip + n], 256)
            end = buf.data_ptr() + start + skip + n
            assert ptr % 256 == 0 and size >= 0 and (size == 0 or ptr + size == end), (skip, n)


def test_numbers_beyond_the_fields_of_the_structs():
    x = torch.zeros((1, 8, 4, 64), dtype=torch.bfloat16)
    long = x[:, :1].expand(1, (1 << 32) + 64, 4, 64)          # no memory behind it: a cut-off size would be 64
    wide = x[:, :, :1].expand(1, 8, (1 << 32) + 4, 64)
    score = lambda q=x, k=x, where=0, k0=0: api._score_desc(q, k, k, where, k0, False, 0.1, 0.0, None, None)
    assert score()[0].Sk == 8 and score(where=(5, 3, 100))[0].q_seg == 3
    for bad in (dict(k=long), dict(q=long), dict(k=wide), dict(q=wide), dict(where=1 << 63), dict(where=-(1 << 63) - 1), dict(where=(0, (1 << 32) + 3, 100)),
                dict(where=(0, 3, 1 << 64)), dict(where=(1 << 64, 3, 100)), dict(k0=1 << 64)):
        with pytest.raises(ValueError, match="does not fit"):
            score(**bad)
    assert score(where=(1 << 63) - 1, k0=-(1 << 63))[0].k_offset == -(1 << 63)
    f = torch.zeros(32, dtype=torch.float64)
    rope = lambda q=x, k=x, offset=0, axes=None: api._rope_desc(q, k, f, offset, None, axes, "halves", True, 1e-6, None, None)
    assert rope(axes=[20, 12]).axis_pairs[1] == 12
    for bad in (dict(q=long, k=long), dict(q=long, k=None), dict(k=wide), dict(offset=(0, (1 << 32) + 3, 100)), dict(axes=[(1 << 32) + 20, 12 - (1 << 32)])):
        with pytest.raises(ValueError, match="does not fit"):
            rope(**bad)


@pytest.mark.gpu
def test_more_rows_of_spans_than_a_field_holds():
    bounds = torch.tensor([[0, 8]]).cuda()
    with pytest.raises(ValueError, match="does not fit"):
        st.st_mask_spans(bounds, (1 << 32) + 8, 0, True)
    with pytest.raises(ValueError, match="does not fit"):
        st.st_mask_spans(bounds, 8, (0, (1 << 32) + 3, 9), True)
