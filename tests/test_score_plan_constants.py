"""What the sizes of GPU tests rest on in the kernels of modified scores (CPU): a change of these constants asks for new sizes there."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_00611_amd", "csrc")


def constant(name, source="st_score_bf16.hip"):
    with open(os.path.join(CSRC, source)) as f:
        found = re.findall(rf"\b{name} = (\d+)", f.read())
    assert len(found) == 1, name
    return int(found[0])


def _row_tiles(B, Hq, Hkv, Sq):
    rows = constant("kScoreRows", "st_score.h")
    return (Sq * (Hq // Hkv) + rows - 1) // rows * Hkv * B


def test_launches_whose_row_tiles_are_put_in_order():
    """test_more_row_tiles_than_the_chip_holds and test_documents_of_unlike_lengths: 526 and 576 workgroups."""
    assert constant("kOrderFrom") < _row_tiles(1, 32, 2, 2100) == 526 <= constant("kOrderUpTo")
    assert constant("kOrderFrom") < _row_tiles(3, 24, 24, 1000) == 576 <= constant("kOrderUpTo")


def test_key_tiles_that_go_through_their_list_twice():
    """test_row_blocks_beyond_one_list: 520 row blocks of a KV head."""
    assert constant("kBlockList") < 1040 * 16 // 32
