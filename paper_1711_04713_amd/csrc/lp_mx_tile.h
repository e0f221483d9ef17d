// Where a stage of dY lies in LDS, and which lane brings what of it (gradient_kernel).  Nothing but constant expressions: any C++
// compiler can enumerate them.
#pragma once

namespace lp {

// A stage is TI x 64 elements of 2 bytes: TI rows of 64 positions of the reduction, or, WEIGHTS, 64 rows of TI.  In units of 16 bytes
// (pieces), number k of the tile in LDS belongs to row k / PIECES; the row's pieces change places so that what a read takes
// together lies in different banks: single pieces by r % 8 in rows of 128 bytes, 64 bytes by r % 4 (r % 2 where a row has two)
// where the read goes down the columns.
//
// Every piece has one lane, whichever way it comes: a load to LDS puts lane l's at 16 l from its first byte, so load q of a wave
// fills the 64 pieces from 64 (PER w + q) on, and what comes through registers is written by the same lane.  That order matters where a
// stage is brought through registers after loads to LDS that left zeros there: a wave waits for its own loads only.
template <int TI, int WAVES, bool WEIGHTS>
struct DyTile {
    static constexpr int ROW = WEIGHTS ? TI * 2 : 128, PIECES = ROW / 16; // of a row: bytes, pieces
    static constexpr int PER = TI * 128 / 1024 / WAVES;                   // a wave's loads per stage, and a lane's pieces
    static constexpr int TURN = (ROW < 256 ? ROW / 64 : 4) - 1;           // 64-byte parts that change places
    static_assert((ROW & (ROW - 1)) == 0 && 64 % PIECES == 0, "places are exchanged within a row, and a load takes whole rows");
    static_assert(PER * WAVES * 1024 == TI * 128, "whole loads");

    // number in LDS of piece q of a lane
    static constexpr int number(int wave, int q, int lane) { return (wave * PER + q) * 64 + lane; }
    static constexpr int row(int k) { return k / PIECES; }
    // place of piece s of row r, and the piece that lies at place s: the exchange is its own inverse
    static constexpr int turned(int r, int s) { return WEIGHTS ? (((s >> 2) ^ (r & TURN)) << 2) + (s & 3) : s ^ (r & 7); }
    // the piece of its row that number k holds
    static constexpr int piece(int k) { return turned(row(k), k % PIECES); }
};

} // namespace lp
