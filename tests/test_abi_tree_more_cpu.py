"""More of the tree operators' host side, without a GPU."""
import pytest

from test_abi_tokens_cpu import CACHE, check, lib  # noqa: F401


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


def test_turned_queries_of_shared_memory_are_refused(lib):  # noqa: F811
    """An output of which several rows are one would be written by several threads, in no order."""
    from paper_2606_13426_gb300 import binding as B
    names = ("k v sb st_ sh q qb qt qh qo ob ot oh dtype B W Hq H D block freqs rot halves pos kc vc ks vs pages tab M n cnt st s").split()
    base = dict(CACHE, k=0x1000, v=0x2000, sb=256, st_=128, sh=64, q=0x3000, qb=512, qt=256, qh=64, qo=0x4000, ob=512, ot=256, oh=64,
                dtype=B.SDV_F32, B=2, W=2, Hq=4, H=2, D=64, block=16, freqs=0x5000, rot=64, halves=1, pos=0, s=None)
    check(lib, "sdv_cache_append_rotary", names, base, [
        (dict(ob=0), B.SDV_EINVAL), (dict(ot=0), B.SDV_EINVAL), (dict(oh=0), B.SDV_EINVAL),
        (dict(qo=0x3000, ob=0, qb=0), B.SDV_EINVAL)])
