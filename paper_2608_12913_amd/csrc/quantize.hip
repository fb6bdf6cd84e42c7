// Codes in 8 bits (e4m3) with one fp32 scale per group: 1 x 128 elements (hidden states) or
// 128 x 128 (weights).
//   s = fl32(max |x| / 448), at least 2^-126;   q = x / s rounded to e4m3, ties to even.
// A group that holds a NaN or an infinity gets the scale NaN and codes 0, so that every
// product with it is NaN.
//
// The quotient is rounded once.  A quotient rounded to fp32 first and to e4m3 then goes to
// the wrong code where the first rounding lands on a border (0.13% of the codes of bf16 data,
// whose quotients often lie near one).  So the fp32 quotient is rounded to odd: an
// inexact one with an even last bit moves to the odd neighbour on the side of the true
// quotient, which no border of e4m3 can be.
//
// Bound by memory: 3 bytes per bf16 element, 5 per fp32 one.  16 lanes hold a row's 128
// elements, 8 each, so the group's maximum is four lane exchanges away; a block of 128 x 128
// stays in registers between its maximum and its codes, so x is read once.  Weights of
// 128,256 x 4096 bf16: 286 to 294 us, 5.4 TB/s of reads and writes (a large copy: 4.9).  Hidden states
// of 64 x 4096 bf16 3.0 us, of 1,001 x 2000 fp32 4.1 us: a launch.
#include "proposal.h"

namespace dcd {
namespace {

constexpr int NT = 256;
constexpr int LG = 16;                // lanes per row of a group
constexpr int LE = kGroup / LG;       // elements per lane
constexpr int RP = NT / LG;           // rows per pass of a 128 x 128 block
constexpr float kE4m3Max = 448.f;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

template <int DT>
struct Lane {
    static constexpr int NV = DT == kBF16 ? 1 : 2;
    u32x4 v[NV];

    __device__ __forceinline__ void load(const void *x, size_t elem) {
        const u32x4 *p = reinterpret_cast<const u32x4 *>((const char *)x + elem * (DT == kBF16 ? 2 : 4));
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = __builtin_nontemporal_load(p + i);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = u32x4{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ uint32_t bits(int i) const {
        if constexpr (DT == kBF16) return i % 2 ? v[0][i / 2] & 0xffff0000u : v[0][i / 2] << 16;
        return v[i / 4][i % 4];
    }
    // the largest magnitude as a bit pattern: above 0x7f7fffff where one is not finite
    __device__ __forceinline__ uint32_t top() const {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < LE; ++i) t = max(t, bits(i) & 0x7fffffffu);
        return t;
    }
};

__device__ __forceinline__ uint32_t max16(uint32_t t) {
#pragma unroll
    for (int o = LG / 2; o > 0; o >>= 1) t = max(t, (uint32_t)__shfl_xor((int)t, o));
    return t;
}

// A group's scale and what its codes are computed with.
struct Scale {
    float s, up, inv;
    bool finite;
    __device__ __forceinline__ explicit Scale(uint32_t top) {
        finite = top <= 0x7f7fffffu;
        s = finite ? fmaxf(__uint_as_float(top) / kE4m3Max, 0x1p-126f) : __uint_as_float(0x7fc00000u);
        // small groups are scaled up first, so that no remainder below underflows
        up = s < 0x1p-60f ? 0x1p64f : 1.f;
        inv = 1.f / (s * up);
    }
    // x / s to within one unit of the last place, rounded to odd
    __device__ __forceinline__ float quotient(uint32_t xb) const {
        const float x = __uint_as_float(xb) * up, t = s * up;
        float d = x * inv;
        d = fmaf(fmaf(-d, t, x), inv, d);
        const float rest = fmaf(-d, t, x);
        const uint32_t db = __float_as_uint(d) | (xb & 0x80000000u);  // (-0 stays)
        const uint32_t away = (db ^ __float_as_uint(rest)) >> 31 ? 0xffffffffu : 1u;
        return __uint_as_float(rest != 0.f && !(db & 1u) ? db + away : db);
    }
};

template <int DT>
__device__ __forceinline__ u32x2 codes(const Lane<DT> &a, const Scale &s) {
    u32x2 o = {0u, 0u};
    if (s.finite) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int w = 0;
            w = __builtin_amdgcn_cvt_pk_fp8_f32(s.quotient(a.bits(4 * i)), s.quotient(a.bits(4 * i + 1)), w, false);
            w = __builtin_amdgcn_cvt_pk_fp8_f32(s.quotient(a.bits(4 * i + 2)), s.quotient(a.bits(4 * i + 3)), w, true);
            o[i] = (uint32_t)w;
        }
    }
    return o;
}

// 1 x 128: every 16 lanes take UN groups, one grid stride apart.
template <int DT, int UN>
__global__ __launch_bounds__(NT) void quantize_rows_kernel(QuantProblem P) {
    const int sub = threadIdx.x % LG;
    const long long ngroups = P.rows * P.groups, step = (long long)gridDim.x * (NT / LG);
    const long long g0 = (long long)blockIdx.x * (NT / LG) + threadIdx.x / LG;
    Lane<DT> a[UN];
    size_t at[UN];
    bool in[UN];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
        const long long g = g0 + i * step;
        const long long row = g / P.groups;
        const int col = (int)(g - row * P.groups) * kGroup + sub * LE;
        at[i] = (size_t)row * P.cols + col;
        in[i] = g < ngroups && col < P.cols;  // cols is a multiple of 16: all 8 elements or none
        if (in[i])
            a[i].load(P.x, at[i]);
        else
            a[i].zero();
    }
#pragma unroll
    for (int i = 0; i < UN; ++i) {
        const Scale s(max16(a[i].top()));
        if (in[i]) {
            *reinterpret_cast<u32x2 *>(P.q + at[i]) = codes(a[i], s);
            if (sub == 0) P.scale[g0 + i * step] = s.s;
        }
    }
}

// 128 x 128: a workgroup per block, held in registers between the maximum and the codes.
template <int DT>
__global__ __launch_bounds__(NT) void quantize_blocks_kernel(QuantProblem P) {
    __shared__ uint32_t tops[NT / 64];
    constexpr int NP = kGroup / RP;
    const int sub = threadIdx.x % LG, r = threadIdx.x / LG;
    const long long brow = blockIdx.x / P.groups;
    const int bcol = (int)(blockIdx.x - brow * P.groups);
    const int col = bcol * kGroup + sub * LE;
    Lane<DT> a[NP];
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const long long row = brow * kGroup + i * RP + r;
        if (row < P.rows && col < P.cols)
            a[i].load(P.x, (size_t)row * P.cols + col);
        else
            a[i].zero();
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) t = max(t, a[i].top());
    t = max16(t);
    t = max(t, (uint32_t)__shfl_xor((int)t, 16));
    t = max(t, (uint32_t)__shfl_xor((int)t, 32));
    if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = t;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) t = max(t, tops[i]);
    const Scale s(t);
    if (threadIdx.x == 0) P.scale[blockIdx.x] = s.s;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const long long row = brow * kGroup + i * RP + r;
        if (row < P.rows && col < P.cols)
            *reinterpret_cast<u32x2 *>(P.q + (size_t)row * P.cols + col) = codes(a[i], s);
    }
}

template <int DT>
hipError_t launch(const QuantProblem &p, hipStream_t st) {
    if (p.block_rows == 1) {
        const long long ngroups = p.rows * p.groups;
        // One group per 16 lanes, or four: for many groups of bf16, and for more fp32 ones than a launch
        // counts threads for.  One and four, us: bf16 rows of 4,096, 512 of them 3.4 and 5.0, 2,048: 8.2 and 8.6,
        // 4,096: 15.2 and 14.4, 16,384 of 8,192: 97 and 86; fp32, 8,192 of 4,096: 31 and 35, 65,536 of 8,192:
        // 464 and 510.
        constexpr int UN = 4;
        const bool many = ngroups > (DT == kBF16 ? 1LL << 16 : 1LL << 27);
        const long long per = NT / LG * (many ? UN : 1);
        const dim3 grid((unsigned)((ngroups + per - 1) / per));
        if (many)
            hipLaunchKernelGGL((quantize_rows_kernel<DT, UN>), grid, dim3(NT), 0, st, p);
        else
            hipLaunchKernelGGL((quantize_rows_kernel<DT, 1>), grid, dim3(NT), 0, st, p);
    } else {
        const long long blocks = (p.rows + kGroup - 1) / kGroup * p.groups;
        hipLaunchKernelGGL((quantize_blocks_kernel<DT>), dim3((unsigned)blocks), dim3(NT), 0, st, p);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const QuantProblem &p, hipStream_t st) {
    return p.dtype == kBF16 ? launch<kBF16>(p, st) : launch<kF32>(p, st);
}

}  // namespace dcd
