// Sizes and index arithmetic of the 8-bit logits kernels: plain code, also built into the tests,
// which check the CPU model of the many-row kernel's addresses and rings against it.
#pragma once

namespace dcd {

constexpr int kGroup = 128;  // elements of K that share a scale

// Half a tile (8 rows x 128 columns) loads into LDS at byte 16 l of lane l.  A tile is 16 rows of
// 128 bytes; the 16-byte column c of row r lies at c ^ (r % 8), so that the 16 rows of a matrix operand
// fall into different banks.
constexpr int TILE = 16 * kGroup;  // bytes of 16 rows x 128 columns
constexpr int half_row(int lane) { return lane / 8; }
constexpr int half_column(int lane) { return (lane % 8 ^ lane / 8) * 16; }
// Offset of a lane's first piece of a matrix operand in such a tile.  (Its second piece, 64 columns
// on, lies at the address with bit 6 flipped: tiles start at multiples of 128.)
constexpr int piece_at(int lane) { return lane % 16 * kGroup + (lane / 16 ^ lane % 16 % 8) * 16; }
// The column that is loaded for column `col` of a block: past the end of a row its last ones.
constexpr unsigned load_column(int block, unsigned col, unsigned K) {
    return (unsigned)block * kGroup + col < K - 16 ? (unsigned)block * kGroup + col : K - 16;
}

// The many-row kernel.
constexpr int TT = 256;              // tokens per workgroup
constexpr int VB = 4;                // token blocks per wave
constexpr int WT = 16 * VB;          // tokens per wave
constexpr int WSTAGE = TT * kGroup;  // bytes of a weight stage
constexpr int WL = WT / 8;           // a loading wave's instructions per weight stage
constexpr int SB = 4;                // blocks whose scales are loaded together

template <int RB>
struct TileGeo {
    static constexpr int QB = RB / 2;          // row blocks per wave and hidden-state stage
    static constexpr int TR = 32 * RB;         // rows per workgroup
    static constexpr int HALF = 16 * QB;       // rows of a stage that one half of the waves multiplies
    static constexpr int HL = QB;              // a loading wave's instructions per stage
    static constexpr int HSTAGE = 2 * HALF * kGroup;
    static constexpr int NW = 2, NH = 5;       // stages of the rings
    // stages that may still be under way when the next one is needed: of weights at the end of the
    // products of a block's second part, of hidden states at the end of a slot of reads
    static constexpr int WAHEAD = NW - 1, HAHEAD = NH - 2;
    // scales of SB blocks, two stages; each wave loads those of 64 rows, the last one past the tile's
    static constexpr int SROWS = 8 * RB;       // rows from one wave's to the next one's
    static constexpr int SSTAGE = (TR + 64 - SROWS) * SB * 4;
    static constexpr int SAT = NW * WSTAGE + NH * HSTAGE;
    static constexpr int BAT = SAT + 2 * SSTAGE;   // bias of the tokens
    static constexpr int LDS = BAT + TT * 4;
    static_assert(RB == 4 || RB == 6, "operands of two or three row blocks");
};

// The token (of a wave's 64) at row r of its tiles in LDS.  Block v = 16 rows, and a lane's results
// are rows 4 g .. 4 g + 3 of each: this way those of two blocks are 8 tokens in a row, and the four
// lanes of a row of logits write 64 (bf16) or 128 bytes in a row.
constexpr int token_of(int r) { return r / 32 * 32 + r % 16 / 4 * 8 + r / 16 % 2 * 4 + r % 4; }

// The first row of a tile that loading wave wv (of four) asks for; part `par` of the rows is HALF on.
// Waves 0, 1 load the rows of the first half of the waves, 2, 3 those of the second.
constexpr int first_row(int rb, int wv) { return wv / 2 * 16 * rb + wv % 2 * 8 * (rb / 2); }

// The b-th block of the walk along K from block `start`; past the last one: that one again (never read).
constexpr int walk_block(int b, int nb, int start) {
    return (b < nb - 1 ? b : nb - 1) + start < nb ? (b < nb - 1 ? b : nb - 1) + start
                                                  : (b < nb - 1 ? b : nb - 1) + start - nb;
}
// Where a tile of tokens starts.  Where every weight is read once (one tile of rows), the walk along K
// starts at another block for each tile of tokens, so that the chip does not ask all HBM channels for the
// same columns at once (scales are loaded SB blocks at a time, so only where their number divides).
constexpr int walk_start(int tile, int nrow, int groups) {
    return nrow == 1 && groups % SB == 0 ? (int)((unsigned)tile * SB % (unsigned)groups) : 0;
}

}  // namespace dcd
