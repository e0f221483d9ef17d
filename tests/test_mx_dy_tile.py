"""Who brings which 16 bytes of a stage of dY to LDS in the microscaled gradients: the map of csrc/lp_mx_tile.h, enumerated by a
plain C++ program.  A piece has one lane whichever way it comes, so that a wave's wait for its own loads orders all writes to it."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1711_04713_amd", "csrc")
# rows of dY's tile (columns where the reduction goes down the rows), waves of a workgroup
TILES = [(ti, waves, weights) for ti, waves in ((64, 4), (128, 4), (256, 8)) for weights in (0, 1)]

PROGRAM = """
#include <cstdio>
#include "lp_mx_tile.h"
template <int TI, int WAVES, bool W> void print()
{
    typedef lp::DyTile<TI, WAVES, W> T;
    for (int w = 0; w < WAVES; ++w)
        for (int q = 0; q < T::PER; ++q)
            for (int l = 0; l < 64; ++l) {
                const int k = T::number(w, q, l);
                std::printf("%d %d %d %d %d %d %d %d\\n", TI, int(W), w, q, l, k, T::row(k), T::piece(k));
            }
    for (int r = 0; r < TI * 8 / T::PIECES; ++r)
        for (int s = 0; s < T::PIECES; ++s) std::printf("%d %d -1 0 0 %d %d %d\\n", TI, int(W), r * T::PIECES + T::turned(r, s), r, s);
}
int main()
{
    print<64, 4, false>(); print<64, 4, true>(); print<128, 4, false>(); print<128, 4, true>(); print<256, 8, false>(); print<256, 8, true>();
}
"""


@pytest.fixture(scope="module")
def maps(tmp_path_factory):
    d = tmp_path_factory.mktemp("tile")
    (d / "tile.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I" + CSRC, str(d / "tile.cpp"), "-o", str(d / "tile")], check=True)
    rows = [tuple(map(int, l.split())) for l in subprocess.run([str(d / "tile")], check=True, stdout=subprocess.PIPE, text=True).stdout.splitlines()]
    brings, reads = {}, {}
    for ti, weights, wave, q, lane, number, row, piece in rows:
        if wave < 0:
            reads.setdefault((ti, weights), {})[(row, piece)] = number
        else:
            brings.setdefault((ti, weights), []).append((wave, q, lane, number, row, piece))
    return brings, reads


def of_two_waves(brings, per):
    """Pieces that a load to LDS of one wave fills and another wave writes.  Load q of wave w fills the 1024 bytes from
    (w * per + q) * 1024 on, lane l's 16 bytes at 16 l."""
    loads = {(w * per + q) * 64 + l: w for w, q, l, *_ in brings}
    return sum(loads[number] != w for w, _, _, number, *_ in brings)


@pytest.mark.parametrize("ti,waves,weights", TILES)
def test_a_piece_has_one_lane_and_one_place(maps, ti, waves, weights):
    brings, reads = maps[0][ti, weights], maps[1][ti, weights]
    pieces = ti * 8
    per = pieces // 64 // waves
    assert sorted(b[3] for b in brings) == list(range(pieces))                       # every 16 bytes of the tile, once
    assert len({(row, piece) for *_, row, piece in brings}) == pieces                # every piece of dY, once
    rows, in_row = (64, ti // 8) if weights else (ti, 8)
    assert all(0 <= row < rows and 0 <= piece < in_row for *_, row, piece in brings)
    assert all(reads[row, piece] == number for *_, number, row, piece in brings)     # where the products look for it
    assert of_two_waves(brings, per) == 0


@pytest.mark.parametrize("ti,waves,weights", TILES)
def test_the_check_sees_pieces_of_two_waves(maps, ti, waves, weights):
    """Pieces numbered through the whole workgroup, load by load: the place of a piece is the same, its lane is not."""
    reads = maps[1][ti, weights]
    in_row, per = (ti // 8 if weights else 8), ti * 8 // 64 // waves
    brings = []
    for wave in range(waves):
        for q in range(per):
            for lane in range(64):
                k = q * waves * 64 + wave * 64 + lane
                row, piece = k // in_row, k % in_row
                brings.append((wave, q, lane, reads[row, piece], row, piece))
    assert of_two_waves(brings, per) == ti * 8 * (waves - 1) // waves
