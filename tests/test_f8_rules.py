"""The rules that give a call of the 8-bit operators to one launch or another (csrc/gemm_rules.h), compiled for the host."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "gemm_rules.h"
extern "C" {
int wide(int M, int N) { return sjd::f8_wide_before_tiles(M, N); }
int gate_wide(int M, int F) { return sjd::f8_gate_fills(M, F); }
int read_lanes(int width, int n_rows) { return sjd::f8_read_lanes(width, n_rows); }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.cpp").write_text(SOURCE)
    subprocess.run([shutil.which("g++"), "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2505_24791_amd", "csrc"),
                    str(d / "rules.cpp"), "-o", str(d / "rules.so")], check=True)
    return ctypes.CDLL(str(d / "rules.so"))


def _rounds(M, N):
    """Of the kernel that stays on its CU: row panels are dealt to eight XCDs of 32 CUs, tiles of 256 x 256."""
    return -(--(-(-(-M // 256)) // 8) * -(-N // 256) // 32)


def test_few_row_panels_leave_the_walking_kernel_alone(rules):
    """One to three panels of 256 rows have tiles for one to three of the eight XCDs: with any number of outputs the tiles that spread over the chip take them."""
    for M in (1, 16, 64, 200, 256, 257, 512, 600, 768):
        for N in (8192, 16384, 32768, 65536, 128256, 600000):
            assert not rules.wide(M, N), (M, N)
    for M in (1, 64, 256, 512):
        for F in (4096, 8192, 16384, 32768):
            assert not rules.gate_wide(M, F), (M, F)
    # as measured beside the rules
    for M, N in ((1024, 16384), (1280, 13312), (1536, 16640), (2816, 8448), (4352, 5632), (8448, 4096), (32768, 4096), (8192, 8192), (1280, 8192), (9945, 4096)):
        assert rules.wide(M, N), (M, N)
    for M, F in ((1024, 8192), (900, 8192), (2304, 4224), (4352, 2816), (4096, 2816), (16384, 2816), (4100, 2304)):
        assert rules.gate_wide(M, F), (M, F)


def test_the_fullest_xcd_decides(rules):
    """Wherever the rule takes the kernel, the rounds of the XCD with the most tiles are at most two and a half (of the gate three) times what the same products spread
    over the chip would be; a call with a full round and less than that much more is taken."""
    for M in list(range(100, 6000, 171)) + [16640, 33000, 66000]:
        for N in (260, 1000, 2304, 4096, 8448, 16384, 40000):
            small, large, rounds = -(-M // 128) * -(-N // 128), -(-M // 256) * -(-N // 256), _rounds(M, N)
            one_round = rounds == 1 and small > 512
            assert rules.wide(M, N) == (one_round or (large >= 256 and rounds <= 2.5 * small / 1024)), (M, N)
            assert rules.gate_wide(M, N // 2) == (large >= 256 and rounds <= 3 * small / 1024), (M, N)


def _whole_rows(width):
    """Threads a row that the library counts before it accepts a call over whole rows."""
    return 16 if width <= 128 else 32 if width <= 256 else 64 if width <= 1024 else 256 if width <= 2048 else 512 if width <= 8192 else 1024


def test_reading_back_launches_no_more_threads_than_are_counted(rules):
    """Threads of a launch are counted in 32 bits: up to as many rows as the library accepts, a launch of whole workgroups of 256 has at most 2^31."""
    for width in (1, 8, 64, 65, 128, 129, 256, 257, 512, 513, 640, 1000, 1024, 1025, 2048, 2049, 8192, 32768, 1 << 20):
        most = (2 ** 31 - 1) // _whole_rows(width)
        for n in (1, 5, 4096, 100000, most // 3, most - 1, most):
            lanes = rules.read_lanes(width, n)
            assert 8 <= lanes <= 256 and lanes & (lanes - 1) == 0
            assert -(-n // (256 // lanes)) * 256 <= 2 ** 31, (width, n, lanes)
    # rows that are not so many: a lane for every eight values, up to a workgroup
    for width, lanes in ((1, 8), (64, 8), (65, 16), (512, 64), (513, 128), (1024, 128), (1025, 256), (32768, 256)):
        assert rules.read_lanes(width, 100000) == lanes
