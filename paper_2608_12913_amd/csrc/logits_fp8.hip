// Logits of a head in 8 bits:
//   z[r, v] = sum_b hs[r, b] ws[v / 128, b] sum_{k in block b} h[r, k] w[v, k] + bias[v]
// with e4m3 codes and fp32 scales per 128 columns (and, of the weights, 128 tokens).
//
// The codes are widened to bf16 in registers (exactly) and multiplied there.  The 8-bit matrix
// instructions of gfx950 would align the eight products of a group of columns before they add
// them, and drop what lies 13 bits below the largest one's power of two: measured, 2^-12
// of the magnitudes' sum, ten thousand times a rounding to fp32.
//
// A = weights (tokens), B = hidden states (rows), so a lane's four results belong to one row
// and the block's scale is one number per lane and row block.  Each block's product starts
// from zero and is added to the fp32 sum with one fused multiply-add per element.  A lane
// supplies columns 16 g .. and 64 + 16 g .. (g = lane / 16) of both operands: any order of
// the columns will do that is the same for both.
#include <type_traits>

#include "proposal.h"

namespace dcd {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// 32 columns of a block (a lane's 16 + 16) as four operands in bf16.
struct Wide {
    bf16x8 v[4];
    __device__ __forceinline__ void set(const u32x4 &x0, const u32x4 &x1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4 &x = i < 2 ? x0 : x1;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t c = x[2 * (i % 2) + j];
                const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, 1.f, false);
                const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, 1.f, true);
                v[i][4 * j] = lo[0], v[i][4 * j + 1] = lo[1], v[i][4 * j + 2] = hi[0], v[i][4 * j + 3] = hi[1];
            }
        }
    }
};

__device__ __forceinline__ f32x4 product(const Wide &a, const Wide &b) {
    f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}

__device__ __forceinline__ uint32_t to_bf16(float f) {  // round to nearest even, NaN stays NaN
    const uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (u >> 16) | 0x40u;
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

// Four logits of one row, tokens t .. t+3.
template <int DT>
__device__ __forceinline__ void store4(const Fp8Problem &P, int row, int t, f32x4 z, bool wide) {
    const size_t at = (size_t)row * P.stride + t;
    if constexpr (DT == kF32) {
        float *o = (float *)P.out + at;
        if (wide && t + 3 < P.N) {
            *reinterpret_cast<f32x4 *>(o) = z;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t + j < P.N) o[j] = z[j];
        }
    } else {
        uint16_t *o = (uint16_t *)P.out + at;
        uint32_t b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = to_bf16(z[j]);
        if (wide && t + 3 < P.N) {
            *reinterpret_cast<uint2 *>(o) = make_uint2(b[0] | b[1] << 16, b[2] | b[3] << 16);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t + j < P.N) o[j] = (uint16_t)b[j];
        }
    }
}

typedef __attribute__((address_space(3))) void *lds_ptr;

// Waits until at most N of this wave's vector memory operations are outstanding (they
// complete in issue order; the compiler does not track loads that write LDS).
template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N < 64, "vmcnt is 6 bits");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
}

// All waves of the workgroup; loads in flight stay so (__syncthreads() would wait for them).
__device__ __forceinline__ void barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A lane's two 16-byte pieces of a tile, at LDS address `at` and 64 columns on.  One block with
// its own wait: for plain loads the compiler would wait for every load to LDS in flight.
__device__ __forceinline__ void read_tile(u32x4 &a0, u32x4 &a1, uint32_t at) {
    asm volatile("ds_read_b128 %0, %2\n ds_read_b128 %1, %3\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(a0), "=&v"(a1)
                 : "v"(at), "v"(at ^ 64u)
                 : "memory");
}

__device__ __forceinline__ float read_float(uint32_t at) {
    float x;
    asm volatile("ds_read_b32 %0, %1\n s_waitcnt lgkmcnt(0)" : "=&v"(x) : "v"(at) : "memory");
    return x;
}

// The same of hidden states, with the row's scale.
__device__ __forceinline__ void read_rows(u32x4 &a0, u32x4 &a1, float &s, uint32_t at, uint32_t scale_at) {
    asm volatile("ds_read_b128 %0, %3\n ds_read_b128 %1, %4\n ds_read_b32 %2, %5\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(a0), "=&v"(a1), "=&v"(s)
                 : "v"(at), "v"(at ^ 64u), "v"(scale_at)
                 : "memory");
}

constexpr int TILE = 16 * kGroup;  // bytes of 16 rows x 128 columns

// Offset of a lane's first piece in such a tile in LDS.  A tile is 16 rows of 128 bytes; the
// 16-byte column c of row r lies at c ^ (r % 8), so that the 16 rows of a matrix operand fall
// into different banks.  (Its second piece, 64 columns on, lies at the address with bit 6
// flipped: tiles start at multiples of 128.)
__device__ __forceinline__ uint32_t piece_offset() {
    const int lane = threadIdx.x % 64, n = lane % 16, g = lane / 16;
    return (uint32_t)(n * kGroup + (g ^ n % 8) * 16);
}

// Half a tile (8 rows) from memory into LDS: lane l lands at byte 16 l, which holds column
// (l % 8) ^ (l / 8) of row l / 8.
template <int AUX>
__device__ __forceinline__ void load_half(const uint8_t *base, uint32_t off, char *to) {
    __builtin_amdgcn_global_load_lds(base + off, (lds_ptr)to, 16, 0, AUX);
}

__device__ __forceinline__ uint32_t lds_address(const char *p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}

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

// The weight stream: up to 64 rows, bound by HBM: 82 us for one row and 96 us for 64 rows of
// 128,256 tokens at d = 4096 (6.4 and 5.8 TB/s; each wave reading its matrix operands
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
__device__ __forceinline__ void stream_body(const Fp8Problem &P, int wide, char *lds) {
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
    const uint32_t col = (lane % 8 ^ lane / 8) * 16;
    uint32_t woff[2 * TB], hoff[HT];
#pragma unroll
    for (int q = 0; q < 2 * TB; ++q) woff[q] = (uint32_t)min(8 * q + lane / 8, P.N - 1 - base) * (uint32_t)P.K;
    const int half0 = KS == 1 ? wave * HT % (2 * RB) : 0;  // this wave's halves of the hidden-state tiles
#pragma unroll
    for (int q = 0; q < HT; ++q) hoff[q] = (uint32_t)min(8 * (half0 + q) + lane / 8, P.M - 1) * (uint32_t)P.K;
    // the scales it loads: lanes 0-15 those of 16 rows, lane 16 its tokens' (KS = 4: all rows')
    const float *wscale = P.ws + (size_t)(base / kGroup) * P.groups;
    const float *rscale = P.hs + (size_t)min(KS == 1 ? wave % RB * 16 + n : lane, P.M - 1) * P.groups;
    const float *scale = KS == 1 && lane >= 16 ? wscale : rscale;
    auto column = [&](int i) { return min((uint32_t)block(i) * kGroup + col, (uint32_t)P.K - 16); };
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
            if (row < P.M && tok < P.N) store4<DT>(P, row, tok, acc[t][r] + b, wide);
        }
    }
}

template <int RB, int TB, int KS, int DT>
__global__ __launch_bounds__(256, KS == 1 ? 2 : 1) void logits_stream_kernel(Fp8Problem P, int wide) {
    __shared__ __align__(128) char lds[StreamGeo<RB, TB, KS>::LDS];
    stream_body<RB, TB, KS, DT>(P, wide, lds);
}

// Two workgroups fit a CU, so tokens per wave (64, 32 or 16) go by what gives the chip's 512
// places about one each, and below that K is split.  Measured (us), 64 / 32 / 16 tokens / K split:
// 64 rows of 128,256 tokens, d = 4096: 96 / 124 / 155 / 315;  65,536, 2048: 35 / 32 / 45 / 104;
// 32,003, 2048: 33 / 26 / 25 / 55;  16,384, 4096: 52 / 34 / 29 / 43;  8,192, 8192: 96 / 62 / 50 / 39;
// 4,096, 4096: 52 / 33 / 27 / 12.  One row: 128,256, 4096: 82 / 95 / 91 / 186;
// 8,192, 2048: 17 / 12 / 10 / 9.
template <int RB, int DT>
void launch_stream(const Fp8Problem &p, int wide, hipStream_t st) {
    const int tokens = p.N >= 98304 ? 64 : p.N >= 49152 ? 32 : p.N > 12288 ? 16 : 0;
    const dim3 wg(256);
    auto grid = [&](int per) { return dim3((unsigned)((p.N + per - 1) / per)); };
    if (tokens == 64)
        hipLaunchKernelGGL((logits_stream_kernel<RB, 4, 1, DT>), grid(256), wg, 0, st, p, wide);
    else if (tokens == 32)
        hipLaunchKernelGGL((logits_stream_kernel<RB, 2, 1, DT>), grid(128), wg, 0, st, p, wide);
    else if (tokens == 16)
        hipLaunchKernelGGL((logits_stream_kernel<RB, 1, 1, DT>), grid(64), wg, 0, st, p, wide);
    else
        hipLaunchKernelGGL((logits_stream_kernel<RB, 1, 4, DT>), grid(16), wg, 0, st, p, wide);
}

// A wave owns 32 tokens x 32 rows.
template <int DT>
__global__ __launch_bounds__(256) void logits_rows_kernel(Fp8Problem P, int wide) {
    constexpr int RB = 2, TB = 2;
    const int lane = threadIdx.x % 64, n = lane % 16, g = lane / 16;
    const int tok0 = (blockIdx.x * 4 + threadIdx.x / 64) * 16 * TB, row0 = blockIdx.y * 16 * RB;
    if (tok0 >= P.N) return;
    const uint8_t *w[TB], *h[RB];
    const float *hs[RB];
#pragma unroll
    for (int t = 0; t < TB; ++t) w[t] = P.w + (size_t)min(tok0 + 16 * t + n, P.N - 1) * P.K;
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int row = min(row0 + 16 * r + n, P.M - 1);
        h[r] = P.h + (size_t)row * P.K;
        hs[r] = P.hs + (size_t)row * P.groups;
    }
    const float *ws = P.ws + (size_t)(tok0 / kGroup) * P.groups;
    f32x4 acc[TB][RB] = {};
    for (int b = 0; b < P.groups; ++b) {
        u32x4 a[TB][2], x[RB][2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = b * kGroup + 64 * s + 16 * g;
            const bool in = k < P.K;  // K is a multiple of 16
#pragma unroll
            for (int t = 0; t < TB; ++t) a[t][s] = in ? *(const u32x4 *)(w[t] + k) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int r = 0; r < RB; ++r) x[r][s] = in ? *(const u32x4 *)(h[r] + k) : u32x4{0, 0, 0, 0};
        }
        const float wsb = ws[b];
        Wide wa[TB], xb[RB];
#pragma unroll
        for (int t = 0; t < TB; ++t) wa[t].set(a[t][0], a[t][1]);
#pragma unroll
        for (int r = 0; r < RB; ++r) xb[r].set(x[r][0], x[r][1]);
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const float s = hs[r][b] * wsb;
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const f32x4 p = product(wa[t], xb[r]);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[t][r][j] = fmaf(p[j], s, acc[t][r][j]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < TB; ++t) {
        const int tok = tok0 + 16 * t + 4 * g;
        f32x4 b;
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = P.bias && tok + j < P.N ? P.bias[tok + j] : 0.f;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int row = row0 + 16 * r + n;
            if (row < P.M) store4<DT>(P, row, tok, acc[t][r] + b, wide);
        }
    }
}

template <int DT>
hipError_t launch(const Fp8Problem &p, hipStream_t st) {
    const int esz = DT == kF32 ? 4 : 2;
    // rows that start on a multiple of four elements take their stores four at a time
    const int wide = p.stride % 4 == 0 && (uintptr_t)p.out % (4 * esz) == 0;
    if (p.M <= 16)
        launch_stream<1, DT>(p, wide, st);
    else if (p.M <= 32)
        launch_stream<2, DT>(p, wide, st);
    else if (p.M <= 64)
        launch_stream<4, DT>(p, wide, st);
    else
        hipLaunchKernelGGL((logits_rows_kernel<DT>), dim3((unsigned)((p.N + 127) / 128), (unsigned)((p.M + 31) / 32)),
                           dim3(256), 0, st, p, wide);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_logits_fp8(const Fp8Problem &p, hipStream_t st) {
    return p.dtype == kBF16 ? launch<kBF16>(p, st) : launch<kF32>(p, st);
}

}  // namespace dcd
