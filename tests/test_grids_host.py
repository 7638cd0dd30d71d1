"""How work is cut into grids: the host's arithmetic, compiled by itself and called here."""
import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2005_10761_b200", "csrc")
SHIM = """
#include "grids.h"
using namespace rtopk::mat;
extern "C" {
void dropout_grid(int64_t rows, int64_t units, int64_t per, int64_t* out) {
  const DropoutGrid g(rows, units, per);
  out[0] = g.band, out[1] = g.bands, out[2] = g.blocks;
}
void divisor_of(uint32_t d, uint32_t* out) {
  const Divisor v = divisor(d);
  out[0] = v.m, out[1] = v.d, out[2] = v.shift;
}
int fit(int64_t tiles, int64_t split, int64_t tile_bytes) { return parts_fit(tiles, split, tile_bytes); }
int64_t limit(int which) { return which ? kPartsBytes : kSplitTiles; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("grids")
    src, so = d / "grids.cpp", d / "grids.so"
    src.write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-fPIC", "-shared", "-I", CSRC, "-o", str(so), str(src)], check=True)
    return ctypes.CDLL(str(so))


def dropout_grid(lib, rows, units, per):
    out = (ctypes.c_int64 * 3)()
    lib.dropout_grid(ctypes.c_int64(rows), ctypes.c_int64(units), ctypes.c_int64(per), out)
    return tuple(out)


def most(lo, hi, rng):
    return int(lo * (hi / lo) ** rng.random())


def test_dropout_takes_every_row_within_the_grid_and_31_bits(lib):
    """Up to 2^30 rows and columns: pieces of eight columns in blocks of 256 threads, or of 256 in blocks of eight warps."""
    rng = random.Random(1)
    cols = [1, 7, 8, 9, 255, 256, 257, 1500, 16384, 66076416, 66076424, 1 << 26, (1 << 26) + 8, 67900000, 100000000, (1 << 27) + 8, 1 << 29, (1 << 30) - 8, 1 << 30]
    rows = [1, 2, 3, 4, 5, 63, 64, 65, 8192, 131075, 1 << 20, (1 << 30) - 1, 1 << 30]
    cases = [(r, c) for r in rows for c in cols] + [(most(1, 1 << 30, rng), most(1, 1 << 30, rng)) for _ in range(2000)]
    for r, c in cases:
        for units, per in ((-(-c // 8), 256), (-(-c // 256), 8)):
            band, bands, blocks = dropout_grid(lib, r, units, per)
            assert band >= 4 and band % 4 == 0 and bands >= 1 and blocks >= 1, (r, c)
            assert (bands - 1) * band < r <= bands * band, (r, c)                   # every row has a band, no band is empty
            assert blocks * per >= band // 4 * units, (r, c)                        # every piece a thread or warp
            assert blocks * per <= 1 << 31, (r, c)                                  # whose number 31 bits hold
            assert bands <= 65535 or r * c >= 1 << 46, (r, c)                       # as documented


def test_quotients_by_multiplication(lib):
    rng = random.Random(2)
    out = (ctypes.c_uint32 * 3)()
    for d in [1, 2, 3, 4, 5, 7, 8, 188, 2048, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, (1 << 27) - 1, 1 << 27] + [most(1, 1 << 27, rng) for _ in range(500)]:
        lib.divisor_of(ctypes.c_uint32(d), out)
        m, same, shift = out
        assert same == d
        top = ((1 << 31) - 1) // d
        for q in [0, 1, 2, top - 1, top] + [rng.randint(0, top) for _ in range(20)]:
            for k in (q * d - 1, q * d, q * d + 1, (1 << 31) - 1):
                if 0 <= k < 1 << 31:
                    assert (k if d == 1 else (k * m >> 32) >> shift) == k // d, (k, d)


def test_parts_stay_within_their_counters_and_their_room(lib):
    lib.limit.restype = ctypes.c_int64
    counters, room = lib.limit(0), lib.limit(1)

    def fit(tiles, split, tile_bytes):
        return bool(lib.fit(ctypes.c_int64(tiles), ctypes.c_int64(split), ctypes.c_int64(tile_bytes)))
    for lanes, cols in ((128, 64), (128, 128), (256, 128), (256, 192), (256, 256)):
        size = lanes * cols * 4
        for tiles in (1, 2, 3, 37, 74, 148, 160, 640, 1023, 1024, 1025, 1078, 1 << 30, 1 << 40):
            assert fit(tiles, 1, size)
            for split in (2, 3, 8, 160, 1 << 20, 1 << 40):
                assert fit(tiles, split, size) == (tiles <= counters and tiles * split * size <= room), (lanes, cols, tiles, split)
