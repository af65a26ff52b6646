"""What the kernels of the paged cache ask of the machine: no list of theirs lives in scratch memory."""
from test_kernel_resources import _kernels


def test_the_kernels_of_the_cache_stay_in_registers():
    kernels = _kernels()
    # (an address or a row's span that waits in memory, read once a block or outside the loops)
    for part, most in (("cache_stream_kernel", 28), ("cache_prompt_kernel", 24), ("cache_combine_kernel", 0), ("cache_combine_many_kernel", 0),
                       ("cache_append_kernel", 40), ("cache_read_kernel", 0)):
        found = {name: k for name, k in kernels.items() if part in name}
        assert found, part
        for name, k in found.items():
            assert k[".private_segment_fixed_size"] <= most, (name, k[".private_segment_fixed_size"])
