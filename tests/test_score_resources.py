"""What the kernels of modified scores, norms and rotations ask of the machine: no list of theirs lives in scratch memory, and the
accumulators of their loops stay in registers."""
from test_kernel_resources import _kernels


def test_the_kernels_of_modified_scores_and_rotations_stay_in_registers():
    kernels = _kernels()
    # capped and biased scores of head size 128 have an address waiting in memory, read outside the inner loops
    for part, most in (("score_fwd_kernel", 0), ("score_bwd_kernel", 16), ("score_rows_kernel", 0), ("score_combine_kernel", 0),
                       ("score_add_parts_kernel", 0), ("mask_spans_kernel", 0), ("score_fwd_f32_kernel", 0), ("score_dq_f32_kernel", 0),
                       ("score_dkv_f32_kernel", 8), ("rope_fwd_kernel", 0), ("rope_bwd_kernel", 0),
                       ("rope_dw_kernel", 0)):
        found = {name: k for name, k in kernels.items() if part in name}
        assert found, part
        for name, k in found.items():
            assert k[".private_segment_fixed_size"] <= most, name
