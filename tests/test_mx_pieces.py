"""Rows of x that more than 16 rows against 4-bit weights bring to LDS: no
thread of the kernel forms an address outside of its row, whatever the number
of rows, planes and columns, and each piece comes from where its place in LDS
says. Enumerated with the kernel's own index functions; no GPU is needed."""

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("pieces") / "pieces")
    subprocess.check_call(["g++", "-std=c++17", "-O2", f"-I{os.path.join(ROOT, 'tests', 'hoststub')}",
                           f"-I{os.path.join(ROOT, 'paper_2201_07705_amd', 'csrc')}",
                           os.path.join(ROOT, "tests", "answerstub", "pieces.cpp"), "-o", out])
    return out


def run(*argv):
    return [int(v) for v in subprocess.check_output(argv, text=True).split()]


def test_no_read_leaves_its_row(program):
    outside, displaced, _, some, every_form = run(program)
    assert some and every_form
    assert outside == 0 and displaced == 0


def test_the_enumeration_finds_a_column_that_is_another_threads(program):
    """Up to 120 elements beyond the last row, in forms of 48 rows."""
    outside, _, most, _, _ = run(program, "mistaken")
    assert outside > 0 and most == 120
