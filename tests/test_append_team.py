"""Every 16-byte piece of every row that the cache's append stores is taken by one lane, once: the division of csrc/append_team.cuh, compiled
for the host, at every page, head dimension, width of a value and number of tokens."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_08971_b200", "csrc")
SOURCE = r"""
#include "append_team.cuh"
extern "C" int team(int page, int T, int row_shift) { return append_team(page, T, row_shift); }
extern "C" int warps() { return kAppThreads / 32; }
// how often each piece of each of the block's teams is taken, as cache_append_kernel walks them
extern "C" void walk(int team, int pieces, int* taken) {
    for (int warp = 0; warp < kAppThreads / 32; ++warp)
        for (int lane = 0; lane < 32; ++lane) {
            const int me = append_place(warp, lane, team), lanes = 32 * team;
            int* mine = taken + warp / team * pieces;
            for (int i = 0; i < kHold; ++i)
                if (i * lanes + me < pieces) ++mine[i * lanes + me];
            for (int p = kHold * lanes + me; p < pieces; p += lanes) ++mine[p];
        }
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    at = tmp_path_factory.mktemp("append_team")
    (at / "host.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, str(at / "host.cpp"), "-o", str(at / "host.so")], check=True)
    return ctypes.CDLL(str(at / "host.so"))


@pytest.mark.parametrize("values", [4, 8])          # of a piece: fp32, 16 bits
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_every_piece_once(host, page, d, values):
    row_shift = (d // values).bit_length() - 1
    for T in list(range(1, page + 1)) + [page + 1, 10 * page + 3]:
        team = host.team(page, T, row_shift)
        assert host.warps() % team == 0 and team & team - 1 == 0
        teams = host.warps() // team
        for n in {1, (T + 1) // 2, min(page, T)}:          # tokens that fall into the page
            taken = np.zeros((teams, n << row_shift), np.int32)
            host.walk(team, n << row_shift, taken.ctypes.data_as(ctypes.c_void_p))
            assert (taken == 1).all(), (T, n)
