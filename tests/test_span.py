"""Rows that a CTA of the row kernels takes, for every end that a caller's offsets may hold (the function that the kernels use, compiled for the host)."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_12934_b200", "csrc")


@pytest.fixture(scope="module")
def rows_before(tmp_path_factory):
    at = tmp_path_factory.mktemp("span")
    src, lib = at / "span.cpp", at / "span.so"
    src.write_text('#include "aif_span.h"\nextern "C" int rows_before(int64_t end, int64_t row0, int most) { return aif::rows_before(end, row0, most); }\n')
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-shared", "-fPIC", "-I", CSRC, "-o", str(lib), str(src)], check=True)
    f = C.CDLL(str(lib)).rows_before
    f.argtypes, f.restype = [C.c_int64, C.c_int64, C.c_int], C.c_int
    return f


ENDS = [-2 ** 63, -2 ** 63 + 1, -2 ** 40, -2 ** 33 + 7, -2 ** 32 - 1, -2 ** 32, -2 ** 32 + 5, -2 ** 32 + 10 ** 5, -2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1, -1, 0, 1, 5, 255, 256, 257, 1000,
        2 ** 31 - 1, 2 ** 31, 2 ** 32 + 5, 2 ** 40, 2 ** 63 - 1]


def test_rows_before(rows_before):
    for end in ENDS:
        for row0 in [0, 1, 255, 256, 10 ** 6, 2 ** 31 - 256, 2 ** 31, 2 ** 32 - 5, 2 ** 32 + 256, 2 ** 40]:
            for most in (1, 7, 256):
                assert rows_before(end, row0, most) == min(max(end - row0, 0), most), (end, row0, most)
