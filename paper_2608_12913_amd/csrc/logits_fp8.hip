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

// A wave owns 16 TB tokens x 16 RB rows.
template <int RB, int TB, int DT>
__global__ __launch_bounds__(256) void logits_stream_kernel(Fp8Problem P, int wide) {
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
    const dim3 grid((unsigned)((p.N + 127) / 128), (unsigned)((p.M + 31) / 32));
    hipLaunchKernelGGL((logits_stream_kernel<2, 2, DT>), grid, dim3(256), 0, st, p, wide);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_logits_fp8(const Fp8Problem &p, hipStream_t st) {
    return p.dtype == kBF16 ? launch<kBF16>(p, st) : launch<kF32>(p, st);
}

}  // namespace dcd
