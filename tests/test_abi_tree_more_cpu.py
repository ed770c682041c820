"""More of the tree operators' host side, without a GPU."""
import pytest

from test_abi_tokens_cpu import lib  # noqa: F401


def test_row_tiles_refuses_what_the_call_refuses(lib):  # noqa: F811
    from paper_2606_13426_gb300 import binding as B
    good = [32, 32, 32, 8, 128, 64, 250]
    assert B.sdv_tree_attend_row_tiles(*good) >= 0
    for at, x in ((0, 0), (1, 0), (1, 65), (2, 31), (3, 0), (4, 96), (5, 8), (5, 24), (5, 144), (6, 0), (6, 1 << 25)):
        args = list(good)
        args[at] = x
        assert B.sdv_tree_attend_row_tiles(*args) == B.SDV_EINVAL, args


@pytest.mark.parametrize("rot", [0, 1, 7, -2])
def test_rotary_freqs_of_no_pairs_are_refused(rot):
    """An odd rot would give one pair more, of frequencies that no rotation of rot elements has."""
    from paper_2606_13426_gb300 import api
    with pytest.raises(ValueError):
        api.rotary_freqs(rot, device="cpu")
