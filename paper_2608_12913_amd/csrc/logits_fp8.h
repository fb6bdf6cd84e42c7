// Device code that the kernels of the 8-bit logits share.
#pragma once

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

// Vectors at any element's address: rows of logits start where the stride puts them.
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

// Four logits of one row, tokens t .. t+3.
template <int DT>
__device__ __forceinline__ void store4(const Fp8Problem &P, int row, int t, f32x4 z) {
    const size_t at = (size_t)row * P.stride + t;
    if constexpr (DT == kF32) {
        float *o = (float *)P.out + at;
        if (t + 3 < P.N) {
            *reinterpret_cast<f32x4_any *>(o) = z;
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
        if (t + 3 < P.N) {
            *reinterpret_cast<u32x2_any *>(o) = u32x2{b[0] | b[1] << 16, b[2] | b[3] << 16};
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t + j < P.N) o[j] = (uint16_t)b[j];
        }
    }
}

// Eight logits as bf16.
__device__ __forceinline__ u32x4 pack8(f32x4 x, f32x4 y) {
    u32x4 o;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        o[j] = to_bf16(x[2 * j]) | to_bf16(x[2 * j + 1]) << 16;
        o[2 + j] = to_bf16(y[2 * j]) | to_bf16(y[2 * j + 1]) << 16;
    }
    return o;
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

__device__ __forceinline__ uint32_t piece_offset() { return (uint32_t)piece_at(threadIdx.x % 64); }

// Half a tile (8 rows) from memory into LDS.
template <int AUX>
__device__ __forceinline__ void load_half(const uint8_t *base, uint32_t off, char *to) {
    __builtin_amdgcn_global_load_lds(base + off, (lds_ptr)to, 16, 0, AUX);
}

__device__ __forceinline__ uint32_t lds_address(const char *p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}

}  // namespace
}  // namespace dcd
