"""What attn_fwd_cached_workspace_bytes asks for, which follows the launches that a call may make."""
import pytest

import paper_2603_24517_b200 as lib
from paper_2603_24517_b200 import build as lib_build


@pytest.fixture(scope="module", autouse=True)
def _library():
    lib_build.build()
    lib.load_library()


def _bytes(group, max_new, heads=2):
    return lib.attn_fwd_cached_workspace_bytes(group * heads, heads, max_new)


@pytest.mark.parametrize("group", [17, 32, 100])
def test_large_groups_have_no_launch_for_single_tokens(group):
    """A token of more than 16 heads a key head has too many rows for the decoding kernel: no place for its parts."""
    assert _bytes(group, 1) == _bytes(group, 500) == _bytes(17, 64)
    assert _bytes(group, 500) < _bytes(16, 500) and _bytes(group, 500) < _bytes(1, 500)


@pytest.mark.parametrize("group", [9, 12, 16])
def test_tokens_of_9_to_16_rows_have_tiles_of_16(group):
    """16 rows a tile and one CTA an SM instead of 8 and two: the same number of part rows, but half as many pieces (32 bytes each)."""
    parts = _bytes(group, 500) - _bytes(17, 500)
    assert parts == _bytes(group, 1) and parts < _bytes(8, 1)


def test_sizes_do_not_depend_on_the_length():
    for group in (1, 4, 8, 12, 16):
        assert _bytes(group, 300) == _bytes(group, 300000) == _bytes(group, 300, heads=7)
