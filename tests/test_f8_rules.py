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
