// Logits of a head in 8 bits for more rows than the weight stream takes, bound by the matrix
// cores.
//
// Tile.  A workgroup owns 256 tokens x TR = 32 RB rows; its 8 waves form a 4 x 2 grid of 64
// tokens x 16 RB rows (4 x RB blocks of 16 x 16).  K is walked one block of 128 columns after
// the other.  Weights (a stage: the block's 256 tokens) and hidden states (a stage: half of
// each wave's rows) load straight into two rings in LDS while earlier ones are multiplied; the
// first four waves load the weights and their scales, the other four the hidden states and
// theirs, since a wave's loads complete in order and the weights come from further away.
//
// Two waves share a SIMD, one of each row half, and take turns: a stage of hidden states
// is a slot of LDS reads and a slot of products, and the second half of the waves runs one
// slot behind the first, so that one wave of a SIMD multiplies while the other reads.  Every
// slot ends with a workgroup barrier.
//
// The codes are widened to bf16 in registers, which is exact, and multiplied there, for logits of
// either type.  v_mfma_f32_16x16x128_f8f6f4 would multiply the codes themselves at twice the rate
// (2048 rows: 1.06 ms), but it aligns the eight products of a group of columns before it adds them
// and drops what lies 13 bits below the largest one's power of two (measured: at most 5 of the 7
// possible units): where large products cancel, a logit is lost in that.
//
// What bounds it, 2048 rows of 128,256 tokens at d = 4096: 1.79 ms in bf16 (fp32: 1.81), 1.2 PFLOP/s.
// Timing copies: without the widening 1.44 ms, without the stores 1.69.  Measured with the 8-bit
// instruction's shorter products, and not kept: deeper rings (nothing), workgroups that walk several
// tiles and ask for the next one's stages ahead (+10%: the choice of the tile costs more between the
// products than the wait it saves), workgroups set apart in time (-2%), non-temporal stores (+2%), stores
// straight from the registers (+3%, ragged rows +9%).
#include "logits_fp8.h"

namespace dcd {
namespace {

// Ends a slot: the wave's LDS reads have returned before it arrives, its loads stay in flight.
__device__ __forceinline__ void slot_end() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// `rows` rows of `bytes` bytes: reads past them give zeros.
struct Rows {
    const void *p;
    int n;
    Rows() = default;
    __device__ __forceinline__ Rows(const void *p_, int rows, uint32_t bytes) : p(p_) {
        const unsigned long long all = (unsigned long long)max(rows, 0) * bytes;
        n = (int)(all < 0x7fffffffull ? all : 0x7fffffffull);
    }
    __device__ __forceinline__ void load(uint32_t at, char *to) const {  // 16 bytes per lane
        __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, n, 0x00027000),
                                                 (lds_ptr)to, 16, at, 0, 0, 0);
    }
};
// The loads of one wave: weights (G = 0) or hidden states and their scales (G = 1).  Rows past
// the last one read as zeros, columns past the end of a row as its last ones (what is
// multiplied with them is zeroed).
template <int RB, int G>
struct Loader {
    using Q = TileGeo<RB>;
    static constexpr int L = G == 0 ? WL : Q::HL;
    Rows codes, scales;
    uint32_t off, soff, col, K;
    int lds_codes, lds_scale, nb, rot;

    __device__ __forceinline__ void init(const Fp8Problem &P, int tok0, int row0, int wv, int start) {
        const int lane = threadIdx.x % 64;
        col = (uint32_t)half_column(lane);
        K = (uint32_t)P.K;
        nb = P.groups;
        rot = start;
        if constexpr (G == 0) {
            const int t0 = tok0 + WT * wv;
            codes = Rows(P.w + (size_t)t0 * K, P.N - t0, K);
            off = (uint32_t)token_of(half_row(lane)) * K;
            lds_codes = wv * WT * kGroup;
        } else {
            codes = Rows(P.h + (size_t)row0 * K, P.M - row0, K);
            scales = Rows(P.hs + (size_t)row0 * P.groups, P.M - row0, (uint32_t)P.groups * 4);
            off = (uint32_t)(first_row(RB, wv) + half_row(lane)) * K;
            lds_codes = wv * 8 * Q::QB * kGroup;
            soff = (uint32_t)(wv * Q::SROWS + lane) * (uint32_t)P.groups * 4;
            lds_scale = wv * Q::SROWS * SB * 4;
        }
    }
    __device__ __forceinline__ int block(int b) const { return walk_block(b, nb, rot); }
    // Block b's stage (hidden states: part `par` of the rows) into `to`.
    struct Request {
        uint32_t at;
        char *to;
    };
    __device__ __forceinline__ Request request(int b, int par, char *to) const {
        Request r{off + load_column(block(b), col, K) + (G == 0 ? 0u : (uint32_t)(par * Q::HALF) * K),
                  to + lds_codes};
        asm volatile("" : "+v"(r.at));  // made here, not between the products that the loads are spread over
        return r;
    }
    __device__ __forceinline__ void load(const Request &r, int q) const {
        const uint32_t row = (uint32_t)(G == 0 ? token_of(8 * q) - token_of(0) : 8 * q);
        codes.load(r.at + row * K, r.to + q * 8 * kGroup);
    }
    __device__ __forceinline__ void load_all(const Request &r) const {
#pragma unroll
        for (int q = 0; q < L; ++q) load(r, q);
    }
    // scales of blocks b .. b + SB - 1 (a row's last ones run on into the next row's: not used)
    __device__ __forceinline__ void load_scales(int b, char *to) const {
        scales.load(soff + (uint32_t)block(b) * 4, to + lds_scale);
    }
};

// The operands of a slot, read in one asm block with its own wait (for plain loads the compiler
// would wait for the loads to LDS in flight).
#define DCD_RD(r0, r1, a, o) "ds_read_b128 %[" r0 "], %[" a "] offset:" o "\n ds_read_b128 %[" r1 "], %[" a "x] offset:" o "\n "
#define DCD_RA DCD_RD("a0", "a1", "w", "0") DCD_RD("a2", "a3", "w", "2048") DCD_RD("a4", "a5", "w", "4096") DCD_RD("a6", "a7", "w", "6144")
#define DCD_RB1 DCD_RD("b0", "b1", "h", "0") "ds_read_b32 %[s0], %[s]\n "
#define DCD_RB2 DCD_RB1 DCD_RD("b2", "b3", "h", "2048") "ds_read_b32 %[s1], %[s] offset:256\n "
#define DCD_RB3 DCD_RB2 DCD_RD("b4", "b5", "h", "4096") "ds_read_b32 %[s2], %[s] offset:512\n "
#define DCD_OA                                                                                          \
    [a0] "=&v"(a[0]), [a1] "=&v"(a[1]), [a2] "=&v"(a[2]), [a3] "=&v"(a[3]), [a4] "=&v"(a[4]),          \
        [a5] "=&v"(a[5]), [a6] "=&v"(a[6]), [a7] "=&v"(a[7])
#define DCD_OB1 [b0] "=&v"(b[0]), [b1] "=&v"(b[1]), [s0] "=&v"(s[0])
#define DCD_OB2 DCD_OB1, [b2] "=&v"(b[2]), [b3] "=&v"(b[3]), [s1] "=&v"(s[1])
#define DCD_OB3 DCD_OB2, [b4] "=&v"(b[4]), [b5] "=&v"(b[5]), [s2] "=&v"(s[2])
#define DCD_IB [h] "v"(h), [hx] "v"(h ^ 64u), [s] "v"(sc)
#define DCD_READ_ALL(n)                                                                       \
    asm volatile(DCD_RA DCD_RB##n "s_waitcnt lgkmcnt(0)"                                      \
                 : DCD_OA, DCD_OB##n                                                          \
                 : [w] "v"(w), [wx] "v"(w ^ 64u), DCD_IB                                      \
                 : "memory")
#define DCD_READ_ROWS(n) asm volatile(DCD_RB##n "s_waitcnt lgkmcnt(0)" : DCD_OB##n : DCD_IB : "memory")
static_assert(TILE == 2048 && 16 * SB * 4 == 256, "offsets of the reads");

template <int QB>
struct Operands {
    u32x4 a[2 * VB], b[2 * QB];
    float s[QB];

    __device__ __forceinline__ void read_all(uint32_t w, uint32_t h, uint32_t sc) {
        if constexpr (QB == 2) DCD_READ_ALL(2);
        if constexpr (QB == 3) DCD_READ_ALL(3);
    }
    __device__ __forceinline__ void read_rows(uint32_t h, uint32_t sc) {
        if constexpr (QB == 2) DCD_READ_ROWS(2);
        if constexpr (QB == 3) DCD_READ_ROWS(3);
    }
    // columns past the end of the rows count as zero
    __device__ __forceinline__ void zero_tail(int k, int K) {
        const int g = threadIdx.x % 64 / 16;
#pragma unroll
        for (int j = 0; j < QB; ++j) {
            if (k + 16 * g >= K) b[2 * j] = u32x4{0, 0, 0, 0};
            if (k + 64 + 16 * g >= K) b[2 * j + 1] = u32x4{0, 0, 0, 0};
        }
    }
};

// Products whose results are not added yet: a product's result is there two products later, so
// the matrix cores never wait for the additions.
struct Pending {
    f32x4 p[2];
    float s;
};

// One stage's products, added to row blocks R0 .. of the sums (and the last two of the stage
// before to row block RP), with the loads LO .. HI-1 of a stage spread over them.
template <int RB, int R0, int RP, class L>
__device__ __forceinline__ void multiply(const Operands<RB / 2> &o, const Wide (&wa)[VB], float ws,
                                         Pending &pend, f32x4 (&acc)[VB][RB], const L &ld, const typename L::Request &req,
                                         int lo, int hi) {
    constexpr int QB = RB / 2, N = VB * QB;
    f32x4 p[3];
    p[1] = pend.p[0];
    p[2] = pend.p[1];
    float s = 0.f, before = pend.s;
    Wide x[2];
    x[0].set(o.b[0], o.b[1]);
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int j = k / VB, v = k % VB;
        if (v == 0) s = o.s[j] * ws;
#pragma unroll
        for (int q = 0; q < 16; ++q)
            if (q >= lo && q < hi && (q - lo) * N / (hi > lo ? hi - lo : 1) == k) ld.load(req, q);
        if (v == 1 && j + 1 < QB) x[(j + 1) % 2].set(o.b[2 * j + 2], o.b[2 * j + 3]);
        p[k % 3] = product(wa[v], x[j % 2]);
        const int k2 = k - 2, row = k2 < 0 ? RP : R0 + k2 / VB, v2 = (k2 + VB) % VB;
        const float s2 = k2 < 0 || k2 / VB < j ? before : s;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[v2][row][i] = fmaf(p[(k + 1) % 3][i], s2, acc[v2][row][i]);
        if (v == 1) before = s;
        __builtin_amdgcn_sched_barrier(0);
    }
    pend.p[0] = p[(N - 2) % 3];
    pend.p[1] = p[(N - 1) % 3];
    pend.s = s;
    // the products belong to this slot: without a use here the compiler moves them past its end
    asm volatile("" : "+v"(pend.p[0]), "+v"(pend.p[1]), "+v"(pend.s));
#pragma unroll
    for (int j = 0; j < QB; ++j)
#pragma unroll
        for (int v = 0; v < VB; ++v) asm volatile("" : "+v"(acc[v][R0 + j]));
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
}

// A wave's work.  Stage q = 2 c + par of the hidden states holds block c of part `par` of the rows.
//
// Slots: the first half of the waves (G = 0) reads stage q in slot 2 q and multiplies it in slot
// 2 q + 1; the second half one slot later.  Every read of stage q has returned by the end of slot
// 2 q + 1, so from slot 2 q + 2 on it may be filled again; the weights of block c, which are read
// with its first stage and kept, from slot 4 c + 2.
//   G = 0 asks for weight block c + NW in slots 4 c + 2 and 4 c + 3, into the stage of block c, and
//     has waited for block c + 1 by the end of the latter.
//   G = 1 asks for hidden-state stage q + NH in slot 2 q + 2, its slot of the products of stage q,
//     into the stage of q, and has waited for stage q + 1 by the end of slot 2 q + 1; and at the
//     first block of every SB for the scales of the SB blocks after these.
// Requests past the end repeat the last block, so that the waits count the same loads (scales
// only make them stricter).
template <int RB, int G, int DT>
__device__ __forceinline__ void work(const Fp8Problem &P, char *lds, int tok0, int row0, int wv, int start) {
    using Q = TileGeo<RB>;
    constexpr int QB = Q::QB, NW = Q::NW, NH = Q::NH;
    static_assert(Q::HAHEAD < 2 * SB - 1, "scales have landed before they are read");
    const int lane = threadIdx.x % 64, n = lane % 16, g = lane / 16;
    char *hring = lds + NW * WSTAGE, *sring = lds + Q::SAT;
    Loader<RB, G> ld;
    ld.init(P, tok0, row0, wv, start);
    if constexpr (G == 0) {
#pragma unroll
        for (int c = 0; c < NW; ++c) ld.load_all(ld.request(c, 0, lds + c * WSTAGE));
    } else {
        ld.load_scales(0, sring);
#pragma unroll
        for (int q = 0; q < NH; ++q) ld.load_all(ld.request(q / 2, q % 2, hring + q * Q::HSTAGE));
    }
    if constexpr (G == 0) {
        const int t = WT * wv + lane;
        reinterpret_cast<float *>(lds + Q::BAT)[t] = P.bias && tok0 + t < P.N ? P.bias[tok0 + t] : 0.f;
    }
    wait_loads<0>();
    slot_end();
    const uint32_t w0 = lds_address(lds) + piece_offset() + wv * WT * kGroup;
    const uint32_t h0 = lds_address(hring) + piece_offset() + G * Q::HALF * kGroup;
    const uint32_t s0 = lds_address(sring) + (G * 16 * RB + n) * SB * 4;
    typedef const __attribute__((address_space(4))) float *scalar_ptr;  // read as scalars
    uint32_t wcur = 0, hcur = 0, scur = 0;
    auto next = [](uint32_t x, uint32_t stage, uint32_t ring) { return x + stage == ring ? 0u : x + stage; };
    const scalar_ptr ws = (scalar_ptr)(P.ws + (size_t)(min(tok0 + WT * wv, P.N - 1) / kGroup) * P.groups);
    float wsc = ws[ld.block(0)];
    f32x4 acc[VB][RB] = {};
    Operands<QB> o;
    Wide wa[VB];
    Pending pend = {};
    if constexpr (G == 1) slot_end();
    for (int c = 0; c < P.groups; ++c) {
        const int k = ld.block(c) * kGroup;
        const bool tail = k + kGroup > P.K;
        const uint32_t sc = s0 + scur + c % SB * 4;
        if constexpr (G == 1) {
            if (c % SB == 0 && c + SB < P.groups) ld.load_scales(c + SB, sring + (Q::SSTAGE - scur));
        }
        const float wsn = ws[ld.block(c + 1)];
#pragma unroll
        for (int par = 0; par < 2; ++par) {
            if (par == 0)
                o.read_all(w0 + wcur, h0 + hcur, sc);
            else
                o.read_rows(h0 + hcur, sc + QB * 16 * SB * 4);
            if (tail) o.zero_tail(k, P.K);
            if (par == 0) {
#pragma unroll
                for (int v = 0; v < VB; ++v) wa[v].set(o.a[2 * v], o.a[2 * v + 1]);
            }
            if constexpr (G == 1) wait_loads<Q::HAHEAD * Q::HL>();
            // G = 1: stage 2 c + par + NH
            const auto req = G == 0 ? ld.request(c + NW, 0, lds + wcur)
                                    : ld.request(c + (par + NH) / 2, (par + NH) % 2, hring + hcur);
            if constexpr (G == 0) {
                if (par == 1) {
#pragma unroll
                    for (int q = 0; q < WL / 2; ++q) ld.load(req, q);
                }
            }
            slot_end();
            constexpr int LO = G == 0 ? WL / 2 : 0, HI = G == 0 ? WL : Q::HL;
            if (par == 0)
                multiply<RB, 0, RB - 1>(o, wa, wsc, pend, acc, ld, req, G == 0 ? HI : LO, HI);
            else
                multiply<RB, QB, QB - 1>(o, wa, wsc, pend, acc, ld, req, LO, HI);
            if constexpr (G == 0) {
                if (par == 1) wait_loads<Q::WAHEAD * WL>();
            }
            slot_end();
            hcur = next(hcur, Q::HSTAGE, NH * Q::HSTAGE);
        }
        wcur = next(wcur, WSTAGE, NW * WSTAGE);
        wsc = wsn;
        if (c % SB == SB - 1) scur = Q::SSTAGE - scur;
    }
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[2 + v][RB - 1][i] = fmaf(pend.p[v][i], pend.s, acc[2 + v][RB - 1][i]);
    if constexpr (G == 0) slot_end();
    wait_loads<0>();  // what was asked for past the end
    slot_end();
    // The logits go through LDS, so that a store instruction writes 512 bytes in a row of two rows.
    // Blocks 2 i and 2 i + 1 hold tokens t .. t + 3 and t + 4 .. t + 7.
    constexpr int SIZE = DT == kBF16 ? 2 : 4, PASSES = SIZE / 2, PT = TT / PASSES;  // tokens per pass
    constexpr int EPL = 16 / SIZE, PITCH = 512 + 16;
    static_assert(Q::TR * PITCH <= Q::BAT, "the staged logits end before the bias");
    const int r0 = G * 16 * RB + n, half = lane / 32, slot = lane % 32;
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        if (wv * WT / PT == pass) {
            const int t0 = wv * WT + 8 * g;
#pragma unroll
            for (int i = 0; i < VB / 2; ++i) {
                const f32x4 *b = reinterpret_cast<const f32x4 *>(lds + Q::BAT) + (t0 + 32 * i) / 4;
#pragma unroll
                for (int r = 0; r < RB; ++r) {
                    char *to = lds + (r0 + 16 * r) * PITCH + (t0 + 32 * i - pass * PT) * SIZE;
                    const f32x4 x = acc[2 * i][r] + b[0], y = acc[2 * i + 1][r] + b[1];
                    if constexpr (DT == kBF16) {
                        *reinterpret_cast<u32x4 *>(to) = pack8(x, y);
                    } else {
                        *reinterpret_cast<f32x4 *>(to) = x;
                        *reinterpret_cast<f32x4 *>(to + 16) = y;
                    }
                }
            }
        }
        __syncthreads();
        const int tok = tok0 + pass * PT + slot * EPL, left = P.N - tok;
        for (int r = (wv + 4 * G) * 2 + half; r < Q::TR; r += 16) {
            if (row0 + r >= P.M || left <= 0) continue;
            const char *from = lds + r * PITCH + slot * 16;
            char *to = (char *)P.out + ((size_t)(row0 + r) * P.stride + tok) * SIZE;
            if (left >= EPL) {
                *reinterpret_cast<u32x4_any *>(to) = *reinterpret_cast<const u32x4 *>(from);
            } else {
                for (int j = 0; j < left; ++j) {
                    if constexpr (DT == kBF16)
                        reinterpret_cast<uint16_t *>(to)[j] = reinterpret_cast<const uint16_t *>(from)[j];
                    else
                        reinterpret_cast<float *>(to)[j] = reinterpret_cast<const float *>(from)[j];
                }
            }
        }
        if (pass + 1 < PASSES) __syncthreads();
    }
}

template <int RB, int DT>
__device__ __forceinline__ void tile_body(const Fp8Problem &P, int nrow, char *lds) {
    int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    asm("" : "+s"(wave));
    // workgroup id modulo 8 is its XCD: the row tiles of a token tile run back to back on one
    const int xcd = blockIdx.x % kXcds, at = blockIdx.x / kXcds;
    const int tok0 = (at / nrow * kXcds + xcd) * TT, row0 = at % nrow * TileGeo<RB>::TR;
    if (tok0 >= P.N) return;
    // From the first block and from a block of its own, us, 100 rows in bf16, d = 2048, 4096, 6144, 8192, 16384:
    // 65,536 tokens 42 and 42, 76 and 71, 105 and 102, 142 and 133, 256 and 252; 128,256 tokens, 4096: 150 and 140.
    // With more rows the weights come from the caches: 512 rows of 65,536, 8192 467 and 487, 1024 of 6144 685 and 721.
    const int start = walk_start(tok0 / TT, nrow, P.groups);
    if (wave < 4)
        work<RB, 0, DT>(P, lds, tok0, row0, wave, start);
    else
        work<RB, 1, DT>(P, lds, tok0, row0, wave - 4, start);
}

template <int RB, int DT>
__global__ __launch_bounds__(512, 2) void logits_tile_kernel(Fp8Problem P, int nrow) {
    __shared__ __align__(128) char lds[TileGeo<RB>::LDS];
    tile_body<RB, DT>(P, nrow, lds);
}

template <int RB, int DT>
hipError_t launch(const Fp8Problem &p, hipStream_t st) {
    const int nrow = (p.M + 32 * RB - 1) / (32 * RB), ntok = ((p.N + TT - 1) / TT + kXcds - 1) / kXcds * kXcds;
    hipLaunchKernelGGL((logits_tile_kernel<RB, DT>), dim3((unsigned)(ntok * nrow)), dim3(512), 0, st, p, nrow);
    return hipGetLastError();
}

}  // namespace

// Row blocks per wave: the shape of the least time, taken as rounds of one workgroup per CU times a
// round's time, which grows as 5 + 4 RB.  Measured (us), RB = 4 / 6 in bf16 (fp32 within 5%), d = 4096: 2048 rows
// of 128,256 tokens: 1860 / 1796;  320: 350 / 333;  256: 254 / 322;  160: 235 / 176;  96: 140 / 168;  of 32,003
// tokens, d = 2048: 512 rows 69 / 88;  285: 68 / 48;  160: 35 / 44.  (8 does not fit the registers.)
hipError_t launch_logits_tile(const Fp8Problem &p, hipStream_t st) {
    auto time = [&](int rb) {
        const long long tiles = ((long long)p.N + TT - 1) / TT * ((p.M + 32 * rb - 1) / (32 * rb));
        return (tiles + kCus - 1) / kCus * (5 + 4 * rb);
    };
    const bool large = time(6) < time(4), bf16 = p.dtype == kBF16;
    if (large) return bf16 ? launch<6, kBF16>(p, st) : launch<6, kF32>(p, st);
    return bf16 ? launch<4, kBF16>(p, st) : launch<4, kF32>(p, st);
}

}  // namespace dcd
