// Logits of a head in 8 bits:
//   z[r, v] = sum_b hs[r, b] ws[v / 128, b] sum_{k in block b} h[r, k] w[v, k] + bias[v]
// with e4m3 codes and fp32 scales per 128 columns (and, of the weights, 128 tokens).
//
// Up to 64 rows here, more in logits_fp8_tile.hip.  The codes are widened to bf16 in registers
// (exactly) and multiplied there, with sums in fp32; the matrix cores' 8-bit instructions lose bits
// (there).  Both files take a block's product alike, and the type of the logits changes nothing
// but the last rounding; the order of the blocks depends on the number of rows.
//
// A = weights (tokens), B = hidden states (rows), so a lane's four results belong to one row
// and the block's scale is one number per lane and row block.  Each block's product starts
// from zero and is added to the fp32 sum with one fused multiply-add per element.  A lane
// supplies columns 16 g .. and 64 + 16 g .. (g = lane / 16) of both operands: any order of
// the columns will do that is the same for both.
#include <type_traits>

#include "logits_fp8.h"

namespace dcd {
namespace {

// Geometry of the weight stream for RB blocks of 16 rows and TB tiles of 16 tokens per wave.
// KS = 1: four waves of different tokens share the hidden states; KS = 4: four waves share
// their tokens and take a quarter of K each, with hidden states of their own.
template <int RB, int TB, int KS>
struct StreamGeo {
    static constexpr int SLOTS = RB == 4 ? 6 : 8;                  // weight tiles per wave
    static constexpr int SHARE = KS == 1 ? 4 : 1;                  // waves per ring of hidden states
    static constexpr int HT = 2 * RB > SHARE ? 2 * RB / SHARE : 1;  // a wave's loads per block: halves of tiles,
    static constexpr int HL = HT + (KS == 1 ? 1 : 2);               // and scales
    // a block in the ring: tiles, then scales (KS = 1: of each wave 16 rows' and its tokens';
    // KS = 4: all rows', the tokens')
    static constexpr int SSTEP = KS == 1 ? 80 : 64;
    static constexpr int HSLOT = (RB * TILE + (KS == 1 ? 4 * SSTEP : RB * SSTEP + 4) + 127) / 128 * 128, NH = 3;
    static constexpr int HRING = NH * HSLOT;
    static constexpr int LDS = (KS == 1 ? HRING : 4 * HRING) + 4 * SLOTS * TILE;
    // two workgroups share a CU's LDS, or (KS = 4) one has it to itself
    static_assert(SLOTS > TB && (KS == 1 ? 2 : 1) * LDS <= 160 * 1024, "ring");
};

// The weight stream: up to 64 rows, bound by HBM: 82 to 85 us for one row and 96 to 98 us for 64
// rows of 128,256 tokens at d = 4096 (6.3 and 5.8 TB/s; each wave reading its matrix operands
// straight from memory took 116 and 339 us).  A wave owns 16 TB tokens x 16 RB rows.
// Weights go straight into LDS (8 rows x 128 bytes per instruction, the shape that streams
// fastest), into a ring of the wave's own: a slot is filled again as soon as its tile has
// been read.  The workgroup's four waves share the hidden states, in a ring of three blocks
// filled the same way, two blocks ahead, and meet once per block.  A wave's loads
// complete in the order of their issue, so hidden states asked for later than weights (from
// registers one block ahead, say) would wait for all of those: 140 against 96 us at 64 rows
// of 128,256 tokens, d = 4096.
//
// Lanes past the end of a row re-read its last columns, and the hidden states there count as
// zero.  Each workgroup walks K from a block of its own, so that they do not ask all HBM
// channels for the same columns at once.
//
// A vocabulary too small to fill the chip that way takes KS = 4: 16 tokens per workgroup,
// a quarter of K per wave, the four sums added in their order at the end.
template <int RB, int TB, int KS, int DT>
__device__ __forceinline__ void stream_body(const Fp8Problem &P, char *lds) {
    using G = StreamGeo<RB, TB, KS>;
    constexpr int S = G::SLOTS, HT = G::HT, HL = G::HL;
    const int lane = threadIdx.x % 64, n = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    // a wave past the vocabulary goes along with the last token
    const int tok0 = (KS == 1 ? blockIdx.x * 4 + wave : blockIdx.x) * 16 * TB, base = min(tok0, P.N - 1);
    char *rows = KS == 1 ? lds : lds + wave * G::HRING;
    char *mine = lds + (KS == 1 ? 1 : 4) * G::HRING + wave * S * TILE;
    const int b0 = KS == 1 ? 0 : P.groups * wave / KS, b1 = KS == 1 ? P.groups : P.groups * (wave + 1) / KS;
    const int nb = b1 - b0, rot = nb > 0 ? (int)(7u * blockIdx.x % (unsigned)nb) : 0;
    auto block = [&](int i) { return b0 + (i + rot < nb ? i + rot : i + rot - nb); };

    const uint8_t *w = P.w + (size_t)base * P.K;
    const uint32_t col = half_column(lane);
    uint32_t woff[2 * TB], hoff[HT];
#pragma unroll
    for (int q = 0; q < 2 * TB; ++q) woff[q] = (uint32_t)min(8 * q + half_row(lane), P.N - 1 - base) * (uint32_t)P.K;
    const int half0 = KS == 1 ? wave * HT % (2 * RB) : 0;  // this wave's halves of the hidden-state tiles
#pragma unroll
    for (int q = 0; q < HT; ++q) hoff[q] = (uint32_t)min(8 * (half0 + q) + half_row(lane), P.M - 1) * (uint32_t)P.K;
    // the scales it loads: lanes 0-15 those of 16 rows, lane 16 its tokens' (KS = 4: all rows')
    const float *wscale = P.ws + (size_t)(base / kGroup) * P.groups;
    const float *rscale = P.hs + (size_t)min(KS == 1 ? wave % RB * 16 + n : lane, P.M - 1) * P.groups;
    const float *scale = KS == 1 && lane >= 16 ? wscale : rscale;
    auto column = [&](int i) { return load_column(block(i), col, (uint32_t)P.K); };
    int fill = 0, hfill = 0;  // the slots to be filled next
    auto fetch = [&](int t, uint32_t k) {
#pragma unroll
        for (int q = 0; q < 2; ++q) load_half<2>(w, woff[2 * t + q] + k, mine + fill * TILE + q * TILE / 2);
        fill = fill + 1 == S ? 0 : fill + 1;
    };
    auto fetch_rows = [&](int i) {
        const uint32_t k = column(i);
        char *to = rows + hfill * G::HSLOT;
#pragma unroll
        for (int q = 0; q < HT; ++q) load_half<0>(P.h, hoff[q] + k, to + (half0 + q) * (TILE / 2));
        to += RB * TILE;
        if (lane < (KS == 1 ? 17 : 16 * RB))
            __builtin_amdgcn_global_load_lds(scale + block(i), (lds_ptr)(to + (KS == 1 ? wave * G::SSTEP : 0)), 4, 0, 0);
        if (KS > 1 && lane == 0)
            __builtin_amdgcn_global_load_lds(wscale + block(i), (lds_ptr)(to + RB * G::SSTEP), 4, 0, 0);
        hfill = hfill + 1 == G::NH ? 0 : hfill + 1;
    };

    f32x4 acc[TB][RB] = {};
    const int ntiles = nb * TB;
    if (nb > 0) fetch_rows(0);
    if (nb > 1) fetch_rows(1);
#pragma unroll
    for (int j = 0; j < S; ++j)
        if (j < ntiles) fetch(j % TB, column(j / TB));
    wait_loads<0>();
    __syncthreads();
    const uint32_t wat = lds_address(mine) + piece_offset(), hat = lds_address(rows) + piece_offset(),
                   sat = lds_address(rows) + RB * TILE;
    int slot = 0, hslot = 0;
    // One block.  STEADY: every tile read in it is followed by another one, so the counts of
    // what was asked for since hold.
    auto step = [&](int i, auto STEADY) {
        constexpr bool steady = decltype(STEADY)::value;
        const int b = block(i);
        if (steady || i + 2 < nb) fetch_rows(i + 2);
        const uint32_t hs0 = hslot * G::HSLOT;
        const float wsb = read_float(sat + hs0 + (KS == 1 ? wave * G::SSTEP + 64 : RB * G::SSTEP));
        float s[RB];
        Wide xb[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            u32x4 x0, x1;
            read_rows(x0, x1, s[r], hat + hs0 + r * TILE, sat + hs0 + r * G::SSTEP + n * 4);
            s[r] *= wsb;
            if (b * kGroup + kGroup > P.K) {
                if (b * kGroup + 16 * g >= P.K) x0 = u32x4{0, 0, 0, 0};
                if (b * kGroup + 64 + 16 * g >= P.K) x1 = u32x4{0, 0, 0, 0};
            }
            xb[r].set(x0, x1);
        }
        hslot = hslot + 1 == G::NH ? 0 : hslot + 1;
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            // this tile has landed: after it at least S - 1 tiles and one block of hidden states
            // were asked for
            wait_loads<steady ? 2 * (S - 1) + HL : 0>();
            u32x4 a0, a1;
            read_tile(a0, a1, wat + slot * TILE);
            slot = slot + 1 == S ? 0 : slot + 1;
            if (steady || i * TB + t + S < ntiles) fetch((t + S) % TB, column(i + (t + S) / TB));
            Wide wa;
            wa.set(a0, a1);
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                const f32x4 p = product(wa, xb[r]);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[t][r][j] = fmaf(p[j], s[r], acc[t][r][j]);
            }
        }
        // the next block's hidden states have landed: two blocks of tiles and one of rows were
        // asked for after them; then every wave is done with this block's
        wait_loads<steady ? 4 * TB + HL : 0>();
        if constexpr (KS == 1) barrier();
    };
    int i = 0;
    for (; (i + 1) * TB - 1 + S < ntiles; ++i) step(i, std::true_type{});
    for (; i < nb; ++i) step(i, std::false_type{});
    if constexpr (KS > 1) {
        f32x4 *part = reinterpret_cast<f32x4 *>(lds);
        __syncthreads();  // no wave reads its ring any more
        if (wave) {
#pragma unroll
            for (int r = 0; r < RB; ++r) part[((wave - 1) * RB + r) * 64 + lane] = acc[0][r];
        }
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int k = 0; k < KS - 1; ++k)
#pragma unroll
            for (int r = 0; r < RB; ++r) acc[0][r] += part[(k * RB + r) * 64 + lane];
    }
#pragma unroll
    for (int t = 0; t < TB; ++t) {
        const int tok = tok0 + 16 * t + 4 * g;
        f32x4 b;
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = P.bias && tok + j < P.N ? P.bias[tok + j] : 0.f;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int row = 16 * r + n;
            if (row < P.M && tok < P.N) store4<DT>(P, row, tok, acc[t][r] + b);
        }
    }
}

template <int RB, int TB, int KS, int DT>
__global__ __launch_bounds__(256, KS == 1 ? 2 : 1) void logits_stream_kernel(Fp8Problem P) {
    __shared__ __align__(128) char lds[StreamGeo<RB, TB, KS>::LDS];
    stream_body<RB, TB, KS, DT>(P, lds);
}

// Two workgroups fit a CU, so tokens per wave (64, 32 or 16) go by what gives the chip's 512
// places about one each, and below that K is split.  Measured (us), 64 / 32 / 16 tokens / K split:
// 64 rows of 128,256 tokens, d = 4096: 96 / 124 / 155 / 315;  65,536, 2048: 35 / 32 / 45 / 104;
// 32,003, 2048: 33 / 26 / 25 / 55;  16,384, 4096: 52 / 34 / 29 / 43;  8,192, 8192: 96 / 62 / 50 / 39;
// 4,096, 4096: 52 / 33 / 27 / 12.  One row: 128,256, 4096: 82 / 95 / 91 / 186;
// 8,192, 2048: 17 / 12 / 10 / 9.
template <int RB, int DT>
void launch_stream(const Fp8Problem &p, hipStream_t st) {
    const int tokens = p.N >= 98304 ? 64 : p.N >= 49152 ? 32 : p.N > 12288 ? 16 : 0;
    const dim3 wg(256);
    auto grid = [&](int per) { return dim3((unsigned)((p.N + per - 1) / per)); };
    if (tokens == 64)
        hipLaunchKernelGGL((logits_stream_kernel<RB, 4, 1, DT>), grid(256), wg, 0, st, p);
    else if (tokens == 32)
        hipLaunchKernelGGL((logits_stream_kernel<RB, 2, 1, DT>), grid(128), wg, 0, st, p);
    else if (tokens == 16)
        hipLaunchKernelGGL((logits_stream_kernel<RB, 1, 1, DT>), grid(64), wg, 0, st, p);
    else
        hipLaunchKernelGGL((logits_stream_kernel<RB, 1, 4, DT>), grid(16), wg, 0, st, p);
}

template <int DT>
hipError_t launch(const Fp8Problem &p, hipStream_t st) {
    if (p.M <= 16)
        launch_stream<1, DT>(p, st);
    else if (p.M <= 32)
        launch_stream<2, DT>(p, st);
    else if (p.M <= 64)
        launch_stream<4, DT>(p, st);
    else
        return launch_logits_tile(p, st);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_logits_fp8(const Fp8Problem &p, hipStream_t st) {
    return p.dtype == kBF16 ? launch<kBF16>(p, st) : launch<kF32>(p, st);
}

}  // namespace dcd
