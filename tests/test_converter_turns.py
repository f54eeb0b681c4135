"""The ring between TMA, the two teams of converter warps and the tensor cores: whatever the order in which the warps get on, no warp may
find a barrier a phase further than it can tell, and no tile may be read or overwritten at the wrong time.  A host program runs the turns that
the kernel is compiled from in random orders."""
import os
import subprocess

import pytest

from paper_2607_27735_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("model") / "converter_turns_model")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-x", "c++", "-I", build.CSRC, os.path.join(HERE, "converter_turns_model.cpp"), "-o", exe])
    return exe


@pytest.mark.parametrize("n_raw", [2, 3])
@pytest.mark.parametrize("n_slots", [3, 4, 5, 6, 7])
@pytest.mark.parametrize("n_tiles,units", [(2, 40), (6, 15), (58, 3)])
def test_every_tile_comes_through(model, n_raw, n_slots, n_tiles, units):
    r = subprocess.run([model, str(n_raw), str(n_slots), str(n_tiles), str(units), "60"], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0
    assert r.stdout.split() == ["0", "0"]  # runs that got stuck, runs that met a wrong tile
