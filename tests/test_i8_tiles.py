"""The products' ragged test shapes reach every tile (CPU only)."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2102_08481_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not installed")
def test_ragged_shapes_reach_every_tile(tmp_path):
    """Each tile comes up with rows and channels that end inside it, inside the 32 or 16 of a matrix instruction too, and with channels in
    eights, which by their pitch are written 16 bytes at a time or one by one."""
    from test_gpu_i8 import RAGGED_WIDE
    exe = str(tmp_path / "tiles")
    subprocess.run(["g++", "-O1", "-std=c++17", os.path.join(CSRC, "linear_i8_tiles_driver.cpp"), "-o", exe], check=True, timeout=120)
    out = subprocess.run([exe], input="".join("%d %d %d\n" % s for s in RAGGED_WIDE), capture_output=True, text=True, check=True, timeout=60).stdout.split()
    assert len(out) == len(RAGGED_WIDE)
    some = set()
    for (rows, k, n), tile in zip(RAGGED_WIDE, out):
        r, c = map(int, tile.split("x"))
        if rows % r and n % c and rows % 16 and n % 16 and n % 8 == 0:
            some.add(tile)
    assert some == {"16x16", "32x32", "32x64", "64x64", "96x64", "128x64", "128x128", "192x256", "256x256"}
