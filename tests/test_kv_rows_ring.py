"""The ring of tiles of serving attention for few rows (csrc/kv_rows_ring.cuh, compiled for the host): whatever the order in which copies land and
warps get on, a warp that stops waiting for a tile finds that tile, and everybody comes to an end."""
import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_08971_b200", "csrc")
SOURCE = r"""
#include "kv_rows_ring.cuh"
extern "C" int stages(int tile_bytes) { return rows_stages(tile_bytes); }
extern "C" int warps() { return kRowsWarps; }
extern "C" int keys() { return kRowsKeys; }
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    at = tmp_path_factory.mktemp("kv_rows_ring")
    (at / "host.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, str(at / "host.cpp"), "-o", str(at / "host.so")], check=True)
    return ctypes.CDLL(str(at / "host.so"))


class Barrier:
    """Phases of one arrival each, of which a wait sees the parity alone: it ends where the phase now open has the other one."""

    def __init__(self):
        self.phase = 0

    def passed(self, parity):
        return self.phase & 1 != parity


def walk(stages, warps, tiles, seed):
    """One run of the ring, whoever can move moving in random order; what went wrong, or None."""
    rng = random.Random(seed)
    slow = rng.choice([0.01, 0.1, 0.5])                     # how soon a copy lands
    full, empty = ([[Barrier() for _ in range(stages)] for _ in "kv"] for _ in range(2))
    holds = [[None] * stages for _ in "kv"]                 # which tile's copy has landed
    flying, taken = [], [0] * warps                         # copies on their way; steps that a warp has done (K, then V, of its tiles in turn)
    issued, last = 0, 2 * tiles
    for _ in range(200 * tiles * 20):
        actor = rng.randrange(warps + 2)
        if actor == warps and issued < last:                # the copying warp: K, V of one tile after the other
            n, part = divmod(issued, 2)
            if empty[part][n % stages].passed(n // stages & 1 ^ 1):
                flying.append((part, n))
                issued += 1
        elif actor == warps + 1 and flying and rng.random() < slow:
            part, n = flying.pop(rng.randrange(len(flying)))
            holds[part][n % stages] = n
            full[part][n % stages].phase += 1
        elif actor < warps:
            i, part = divmod(taken[actor], 2)
            n = actor + i * warps
            if n < tiles and full[part][n % stages].passed(n // stages & 1):
                if holds[part][n % stages] != n:
                    return "tile %d of %s: %s" % (n, "KV"[part], holds[part][n % stages])
                empty[part][n % stages].phase += 1
                taken[actor] += 1
        if issued == last and not flying and all(2 * len(range(w, tiles, warps)) == t for w, t in enumerate(taken)):
            return None
    return "no end"


@pytest.mark.parametrize("row_bytes", [16, 32, 64, 128, 256])
def test_every_warp_finds_its_tile(host, row_bytes):
    stages, warps = host.stages(max(1024, host.keys() * row_bytes)), host.warps()
    for seed in range(150):
        assert walk(stages, warps, 5 + seed % 40, seed) is None, (stages, seed)


def test_a_ring_that_its_warps_do_not_divide_is_found_out():
    assert any(walk(6, 4, 40, seed) for seed in range(150))
