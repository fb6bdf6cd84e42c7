// The 8-bit logits kernels' index arithmetic (csrc/logits_fp8_geo.h) for the tests.
#include "logits_fp8_geo.h"

using namespace dcd;

namespace {
template <int RB>
void fill(int *out) {
    using Q = TileGeo<RB>;
    const int all[] = {Q::TR, Q::HSTAGE, Q::NW,  Q::NH,  Q::WAHEAD, Q::HAHEAD, Q::SROWS, Q::SSTAGE,
                       Q::SAT, Q::BAT,   Q::LDS, Q::HL, Q::HALF};
    for (int v : all) *out++ = v;
}
}  // namespace

extern "C" {
void geo_constants(int *out) {
    const int all[] = {kGroup, TILE, TT, VB, WT, WSTAGE, WL, SB};
    for (int v : all) *out++ = v;
}
void geo_tile(int rb, int *out) { rb == 4 ? fill<4>(out) : fill<6>(out); }
int geo_token_of(int r) { return token_of(r); }
int geo_half_row(int lane) { return half_row(lane); }
int geo_half_column(int lane) { return half_column(lane); }
int geo_piece_at(int lane) { return piece_at(lane); }
int geo_load_column(int block, int col, int K) { return (int)load_column(block, (unsigned)col, (unsigned)K); }
int geo_first_row(int rb, int wv) { return first_row(rb, wv); }
int geo_walk_block(int b, int nb, int start) { return walk_block(b, nb, start); }
int geo_walk_start(int tile, int nrow, int groups) { return walk_start(tile, nrow, groups); }
}
