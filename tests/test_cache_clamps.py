"""CPU: the clamps of the cache kernels' tables (csrc/clamp.h), compiled for the
host, at values that no table should hold: what they give stays inside the
caller's buffers, and is the table's own where that is in range."""

from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2606_09441_amd", "csrc")
SOURCE = """
#include "clamp.h"
extern "C" int within(int x, int most) { return sift::within(x, most); }
extern "C" int rows_between(int row0, int end, int rows, int max_rows) {
  return sift::rows_between(row0, end, rows, max_rows);
}
extern "C" int keys_of_page(int page_len, int in, int left) {
  return sift::keys_of_page(page_len, in, left);
}
"""
LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module")
def clamps(tmp_path_factory):
    d = tmp_path_factory.mktemp("clamps")
    (d / "clamps.cpp").write_text(SOURCE)
    # -ftrapv: an overflow ends the process
    subprocess.run(["g++", "-std=c++17", "-ftrapv", "-shared", "-fPIC", "-I", CSRC,
                    str(d / "clamps.cpp"), "-o", str(d / "clamps.so")], check=True)
    return ctypes.CDLL(str(d / "clamps.so"))


def test_row_pointers(clamps):
    for rows in (0, 1, 10, HIGH):
        ends = [LOW, LOW + 1, -1, 0, 1, 5, rows - 1, rows, min(rows + 1, HIGH), HIGH]
        for first in ends:
            row0 = clamps.within(first, rows)
            assert row0 == min(max(first, 0), rows)
            for end in ends:
                for most in (1, 8, HIGH):
                    n = clamps.rows_between(row0, end, rows, most)
                    assert 0 <= n <= most and row0 + n <= rows
                    assert n == max(0, min(min(end, rows) - row0, most))


def test_page_lengths(clamps):
    for at in (0, 16, 112):
        for page_len in (LOW, LOW + 1, -1, 0, 1, at + 1, at + 16, 128, HIGH):
            for left in (LOW + 256, -1, 0, 1, 16, HIGH):
                n = clamps.keys_of_page(page_len, at, left)
                assert n == min(max(min(page_len - at, left), 0), 16)
