"""CPU test of what the products of the step for matrices ask memory for: every request of every kind of tile within its operand (tests/host/muon_ranges_host.cpp goes through csrc/zc_muon_ask.h)."""
import os
import subprocess

import pytest


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path_factory.mktemp("ranges") / "muon_ranges_host")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", os.path.join(root, "tests", "host", "muon_ranges_host.cpp"), "-o", exe], check=True)
    return exe


def test_requests_stay_within_their_operands(exe):
    run = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0, run.stdout
    assert int(run.stdout.split()[0]) > 1000000


def test_an_order_that_goes_on_behind_the_last_tile_is_found(exe):
    run = subprocess.run([exe, "on"], capture_output=True, text=True, timeout=100)
    assert run.returncode != 0 and "a tile behind the last one" in run.stdout
