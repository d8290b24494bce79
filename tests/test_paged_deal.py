"""The dealing of the paged attention's tiles, run on the host."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("deal") / "deal")
    subprocess.check_call(["g++", "-O1", "-std=c++20", "-pthread", os.path.join(HERE, "paged_deal_host.cpp"), "-o", out])
    return out


def run(program, what):
    r = subprocess.run([program, what], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout


def test_every_tile_is_dealt_once_and_in_order(program):
    run(program, "lines")


def test_rows_that_become_shorter_meanwhile_end_the_dealing_and_are_recorded(program):
    run(program, "shorter")
