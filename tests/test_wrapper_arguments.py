"""Arguments that the wrapper hands to the C ABI as numbers: what does not fit is refused, not cut off (CPU)."""
import pytest
import torch

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
