"""What the tree attention's kernels for many rows do when a wait gives up (tree_rows_check.cu), and that a workspace's
earlier contents tell nothing."""
import os
import subprocess

import pytest
import torch

from test_gpu_tokens import BF16, api, gen, make_cache  # noqa: F401
from test_gpu_tree_attend import tree_of, widened

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def said(tmp_path_factory):
    from paper_2606_13426_gb300 import buildlib
    exe = str(tmp_path_factory.mktemp("rows") / "tree_rows_check")
    subprocess.run([buildlib._nvcc()] + buildlib.ARCH + ["-O2", "-std=c++17", os.path.join(HERE, "tree_rows_check.cu"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    return dict(line.split(": ", 1) for line in r.stdout.splitlines())


def test_what_a_block_that_gave_up_was_to_write_is_nan(said):
    """Sequence 0 in runs 0 to 2, sequence 1 in run 2, sequence 2 in runs 2 and 3: output and status of each."""
    assert said["join -1"] == "joined/0 kept/0 joined/0"
    assert said["join 0"] == "nan/128 kept/0 joined/0"
    assert said["join 2"] == "nan/128 nan/128 nan/128"
    assert said["join 3"] == "joined/0 kept/0 nan/128"


def test_copies_have_landed_when_the_copying_warp_gives_up(said):
    assert said["copies"] == "there"


def test_a_wait_ends(said):
    assert said["wait"] == "0 1 0"


def test_a_workspace_tells_nothing_of_its_past(api):
    from paper_2606_13426_gb300 import binding as B
    g = gen(3)
    for D, W, G in ((64, 64, 2), (128, 60, 3)):
        cache = make_cache(api, g, 90, 2, 32, D)
        pages = widened(torch.randperm(90, generator=g, device="cuda").to(torch.int32).view(3, 30))
        n = torch.tensor([900, W, 333], device="cuda", dtype=torch.int32)
        q = torch.randn(3, W, 2 * G, D, generator=g, device="cuda").to(BF16)
        par = torch.tensor([tree_of("tree", W)] * 3, device="cuda", dtype=torch.int32)
        assert B.sdv_tree_attend_row_tiles(3, W, 2 * G, 2, D, 32, pages.shape[1]) == (W * G + 127) // 128
        got = []
        for byte in (0, 0xff):
            ws = torch.full((B.sdv_tree_attend_workspace_bytes(3, W, 2 * G, 2, D),), byte, dtype=torch.uint8, device="cuda")
            status = torch.zeros(3, dtype=torch.int32, device="cuda")
            got.append(api.tree_attend(q, cache, pages, n, par, status=status, workspace=ws))
            assert status.tolist() == [0, 0, 0]
        assert all(torch.equal(got[0][k], got[1][k]) and got[0][k].isfinite().all() for k in ("out", "lse"))
