"""How the blocks of paged attention agree (csrc/attn_count.h), under random orders of their threads
on the host (tests/count_probe.cpp)."""
import os
import subprocess

import pytest

from paper_2609_37241_gb300 import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("count") / "count_probe")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.CSRC, os.path.join(HERE, "count_probe.cpp"), "-o", exe], check=True)

    def run(name, runs=4000):
        return subprocess.run([exe, name, str(runs)], capture_output=True, text=True, check=True, timeout=120).stdout.strip()
    return run


def test_parts_of_few_rows_are_joined_once(probe):
    assert probe("rows") == "ok"


def test_parts_of_many_rows_are_joined_once(probe):
    """Without block barriers before the join: what the other blocks wrote has to be known by then."""
    assert probe("tile") == "ok"


def test_one_word_for_two_answers_is_found(probe):
    """A thread that reads the first answer late finds the second one in its place."""
    assert probe("rows-one-word") != "ok"


def test_a_block_that_starts_late_takes_its_share(probe):
    """The second kernel's blocks, started before and after its block 0 has put the start word back."""
    assert probe("start") == "ok"
    assert probe("start-reads-again") != "ok"  # the form that goes by the word it reads after the wait


def test_a_part_that_failed_is_not_joined(probe):
    """A wait that runs out in one thread of a block: nobody reads the part that it did not write."""
    assert probe("tile-failed") == "ok"
    assert probe("tile-failed-counts") != "ok"  # the form whose failed block counts, and is completed by another
