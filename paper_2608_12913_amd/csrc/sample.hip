// Sampling of one token per row of logits, with each row's temperature T, top-k, top-p and
// min-p and a given uniform u.
//
// Order: logits descending, token id ascending on ties; -inf is never kept.  Weights
// w = exp((z - max z) / T).  All three rules keep a first part of that order:
//   n_k = top_k;  n_p = the smallest n whose weights sum to at least top_p of the first n_k's;
//   n_m = the number of weights of at least min_p.
// The token is the inverse CDF in token-id order over what is kept: the smallest one
// whose cumulative weight exceeds u times the total.
//
// Sums of weights are unsigned 64-bit fixed-point numbers, at a step small enough for the vocabulary
// (2^-45 of the largest weight at 128,256 tokens), of weights computed in 64 bits: they add
// up to the same whatever the order, so that sums in LDS atomics give the same bits in every
// call and a border between two tokens is where 64-bit arithmetic puts it.
#include "proposal.h"

namespace dcd {
namespace {

typedef unsigned long long u64;

constexpr int NT = 1024;             // threads of a row's workgroup
constexpr int NW = NT / 64;
constexpr int BITS = 11;             // of a key per search level
constexpr int BINS = 1 << BITS;
constexpr int MAXCHUNKS = 2048;      // pieces of a row for the draw
constexpr uint32_t kLowest = 0x00800000u;  // key of the lowest finite logit

// fp32 bits -> unsigned key of the same order; -0 counts as 0
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

template <int DT>
__device__ __forceinline__ float load(const void *row, int i) {
    if constexpr (DT == kBF16) return __uint_as_float((uint32_t)((const uint16_t *)row)[i] << 16);
    return ((const float *)row)[i];
}

// Weights of a row relative to its largest logit, in 64 bits and as fixed-point numbers.
struct Weights {
    double top, inv_T, one;  // one: 2^shift, the fixed-point weight of the largest logit
    __device__ __forceinline__ double exact(uint32_t key) const {
        return exp(((double)logit_of(key) - top) * inv_T);
    }
    __device__ __forceinline__ u64 fixed(uint32_t key) const { return (u64)rint(exact(key) * one); }
};

// The last kept element of the order.
struct Cut {
    uint32_t key, id;
    __device__ __forceinline__ bool keeps(uint32_t k, uint32_t i) const {
        return k > key || (k == key && i <= id);
    }
};

struct Shared {
    u64 mass[BINS];
    uint32_t count[BINS];
    u64 wmass[NW];
    uint32_t wcount[NW];
    u64 pick_mass;      // what lies above the bin that was found
    uint32_t pick_count;
    uint32_t pick_bin, bin_count;
    u64 total;
};

__device__ __forceinline__ u64 shfl_up64(u64 x, int o) {
    return (u64)__shfl_up((long long)x, o);
}

// Exclusive sums over the workgroup of (count, mass), in thread order.
__device__ __forceinline__ void block_scan(Shared &S, uint32_t &c, u64 &m) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t c0 = c;
    const u64 m0 = m;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t cc = __shfl_up(c, o);
        const u64 mm = shfl_up64(m, o);
        if (lane >= o) {
            c += cc;
            m += mm;
        }
    }
    __syncthreads();
    if (lane == 63) {
        S.wcount[wave] = c;
        S.wmass[wave] = m;
    }
    __syncthreads();
    c -= c0;
    m -= m0;
    for (int w = 0; w < wave; ++w) {
        c += S.wcount[w];
        m += S.wmass[w];
    }
}

__device__ __forceinline__ u64 block_sum(Shared &S, u64 m) {
    uint32_t c = 0;
    u64 mine = m;
    block_scan(S, c, m);
    if (threadIdx.x == NT - 1) S.total = m + mine;
    __syncthreads();
    return S.total;
}

// From the first bin in walking order (the highest if `down`): the bin where the running
// count (or mass) reaches `target`.  Returns the bin; above_* are advanced past the bins
// before it.
template <bool MASS, bool DOWN>
__device__ __forceinline__ uint32_t find_bin(Shared &S, u64 target, uint32_t &above_c, u64 &above_m) {
    constexpr int PER = BINS / NT;
    uint32_t c = 0;
    u64 m = 0;
    const int b0 = threadIdx.x * PER;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = DOWN ? BINS - 1 - (b0 + i) : b0 + i;
        c += S.count[b];
        m += S.mass[b];
    }
    block_scan(S, c, m);
    c += above_c;
    m += above_m;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = DOWN ? BINS - 1 - (b0 + i) : b0 + i;
        const uint32_t c1 = c + S.count[b];
        const u64 m1 = m + S.mass[b];
        if (MASS ? m < target && m1 >= target : c < target && c1 >= target) {
            S.pick_bin = b;
            S.pick_count = c;
            S.pick_mass = m;
            S.bin_count = S.count[b];
        }
        c = c1;
        m = m1;
    }
    __syncthreads();
    above_c = S.pick_count;
    above_m = S.pick_mass;
    return S.pick_bin;
}

__device__ __forceinline__ void clear_bins(Shared &S) {
    __syncthreads();
    for (int b = threadIdx.x; b < BINS; b += NT) {
        S.count[b] = 0;
        S.mass[b] = 0;
    }
    __syncthreads();
}

// The element of the order where the running count (or mass) reaches `target`, which the
// row's finite logits do reach; `kept` gets the mass up to and with it.
template <bool MASS, class ForEach>
__device__ Cut search(Shared &S, const ForEach &each, const Weights &W, u64 target, int idbits, u64 &kept) {
    uint32_t prefix = 0, above_c = 0;
    u64 above_m = 0;
    const int shifts[3] = {32 - BITS, 32 - 2 * BITS, 0};
    for (int l = 0; l < 3; ++l) {
        const int shift = shifts[l], bits = l < 2 ? BITS : 32 - 2 * BITS;
        clear_bins(S);
        each([&](uint32_t, uint32_t key) {
            if (key < kLowest || (l && key >> (shift + bits) != prefix)) return;
            const uint32_t b = key >> shift & ((1u << bits) - 1);
            atomicAdd(&S.count[b], 1u);
            const u64 w = W.fixed(key);
            if (w) atomicAdd(&S.mass[b], w);
        });
        __syncthreads();
        prefix = prefix << bits | find_bin<MASS, true>(S, target, above_c, above_m);
    }
    const uint32_t equal = S.bin_count;
    const u64 w = W.fixed(prefix);
    u64 m = MASS ? (target - above_m + w - 1) / (w ? w : 1) : target - above_c;
    m = m < 1 ? 1 : m > equal ? equal : m;
    kept = above_m + m * w;
    Cut cut{prefix, 0xffffffffu};
    if (m < equal) {  // the m-th of the equal logits in id order
        uint32_t idp = 0, c = 0;
        u64 none = 0;
        for (int hi = idbits; hi > 0;) {
            const int bits = hi < BITS ? hi : BITS, shift = hi - bits;
            clear_bins(S);
            each([&](uint32_t id, uint32_t key) {
                if (key == cut.key && (hi == idbits || id >> hi == idp))
                    atomicAdd(&S.count[id >> shift & ((1u << bits) - 1)], 1u);
            });
            __syncthreads();
            idp = idp << bits | find_bin<false, false>(S, m, c, none);
            hi = shift;
        }
        cut.id = idp;
    }
    return cut;
}

template <int DT>
__global__ __launch_bounds__(NT) void sample_row_kernel(SampleProblem P, int shift, int idbits) {
    __shared__ Shared S;
    __shared__ uint32_t top_key, bad;
    __shared__ u64 csum[MAXCHUNKS];
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const char *row = (const char *)P.logits + (size_t)r * P.stride * (DT == kBF16 ? 2 : 4);
    float *probs = P.probs ? P.probs + (size_t)r * P.V : nullptr;

    // the row's rules; one that is outside its range leaves the row without a target
    float T = P.temperature ? P.temperature[r] : 1.f;
    int k = P.top_k ? P.top_k[r] : 0;
    const float top_p = P.top_p ? P.top_p[r] : 1.f, min_p = P.min_p ? P.min_p[r] : 0.f;
    const float u = P.u[r];
    const bool rules_ok = T >= 0.f && T <= 3.4028235e38f && top_p >= 0.f && top_p <= 1.f && min_p >= 0.f &&
                          min_p <= 1.f && u >= 0.f && u < 1.f;
    if (T == 0.f) {
        T = 1.f;
        k = 1;
    }
    if (tid == 0) top_key = bad = 0;
    __syncthreads();

    // the largest logit; NaN and +inf leave the row without a target
    uint32_t top = 0, finite = 0;
    bool b = false;
    for (int i = tid; i < P.V; i += NT) {
        const float z = load<DT>(row, i);
        b |= !(z < INFINITY);
        const uint32_t key = key_of(z);
        top = max(top, key);
        finite += key >= kLowest;
    }
    atomicMax(&top_key, top);
    if (b) atomicOr(&bad, 1u);
    u64 nfinite = block_sum(S, finite);
    top = top_key;
    if (bad || !rules_ok || top < kLowest) {
        if (probs)
            for (int i = tid; i < P.V; i += NT) probs[i] = 0.f;
        if (tid == 0) {
            P.tokens[r] = -1;
            if (P.kept) P.kept[r] = 0;
            if (P.logprob) P.logprob[r] = __uint_as_float(0x7fc00000u);
        }
        return;
    }
    Weights W;
    W.top = (double)logit_of(top);
    W.inv_T = 1.0 / (double)T;
    W.one = (double)(1ull << shift);

    auto each = [&](auto f) {
        for (int i = tid; i < P.V; i += NT) f((uint32_t)i, key_of(load<DT>(row, i)));
    };
    Cut cut{kLowest, 0xffffffffu};
    u64 total = 0;
    bool have_total = false;
    if (k > 0 && (u64)k < nfinite) {
        cut = search<false>(S, each, W, (u64)k, idbits, total);
        have_total = true;
    }
    if (top_p < 1.f) {
        if (!have_total) {
            u64 m = 0;
            each([&](uint32_t, uint32_t key) {
                if (key >= kLowest) m += W.fixed(key);
            });
            total = block_sum(S, m);
        }
        u64 target = (u64)ceil((double)top_p * (double)total);
        target = target < 1 ? 1 : target > total ? total : target;
        cut = search<true>(S, each, W, target, idbits, total);
    }
    // kept weights per piece of the row, in token order
    const int chunk = max(256, (P.V + MAXCHUNKS - 1) / MAXCHUNKS);
    const int nchunks = (P.V + chunk - 1) / chunk;
    auto kept = [&](uint32_t i, uint32_t key, double &w) {
        if (key < kLowest || !cut.keeps(key, i)) return false;
        w = W.exact(key);
        return w >= (double)min_p;
    };
    u64 n = 0, sum = 0;
    for (int c = wave; c < nchunks; c += NW) {
        u64 m = 0;
        const int end = min(P.V, (c + 1) * chunk);
        for (int i = c * chunk + lane; i < end; i += 64) {
            double w;
            if (kept(i, key_of(load<DT>(row, i)), w)) {
                m += (u64)rint(w * W.one);
                ++n;
            }
        }
        sum += m;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m += (u64)__shfl_xor((long long)m, o);
        if (lane == 0) csum[c] = m;
    }
    total = block_sum(S, sum);
    n = block_sum(S, n);
    // the piece where the running weight exceeds u times the total, then the token in it
    const u64 target = (u64)((double)u * (double)total);  // exceeds: > floor
    u64 m = 0, c2[MAXCHUNKS / NT];
    uint32_t none = 0;
#pragma unroll
    for (int i = 0; i < MAXCHUNKS / NT; ++i) {
        const int c = tid * (MAXCHUNKS / NT) + i;
        c2[i] = c < nchunks ? csum[c] : 0;
        m += c2[i];
    }
    block_scan(S, none, m);
#pragma unroll
    for (int i = 0; i < MAXCHUNKS / NT; ++i) {
        if (m <= target && m + c2[i] > target) {
            S.pick_bin = tid * (MAXCHUNKS / NT) + i;
            S.pick_mass = m;
        }
        m += c2[i];
    }
    __syncthreads();
    if (wave == 0) {
        u64 at = S.pick_mass;
        const int c = S.pick_bin, end = min(P.V, (c + 1) * chunk);
        for (int i0 = c * chunk; i0 < end; i0 += 64) {
            const int i = i0 + lane;
            double w = 0;
            const uint32_t key = i < end ? key_of(load<DT>(row, i)) : 0;
            const u64 mine = kept(i, key, w) ? (u64)rint(w * W.one) : 0;
            u64 run = mine;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const u64 x = shfl_up64(run, o);
                if (lane >= o) run += x;
            }
            run += at;
            const u64 over = __ballot(run > target);
            if (over) {
                if (lane == __ffsll((long long)over) - 1) {
                    P.tokens[r] = i;
                    if (P.logprob)
                        P.logprob[r] =
                            (float)(((double)logit_of(key) - W.top) * W.inv_T - log((double)total / W.one));
                }
                break;
            }
            at = (u64)__shfl((long long)run, 63);
        }
    }
    if (P.kept && tid == 0) P.kept[r] = (int32_t)n;
    if (probs) {
        const double scale = W.one / (double)total;
        each([&](uint32_t i, uint32_t key) {
            double w;
            probs[i] = kept(i, key, w) ? (float)(w * scale) : 0.f;
        });
    }
}

int bits_of(uint32_t x) {
    int b = 0;
    while (b < 32 && x >> b) ++b;
    return b;
}

}  // namespace

size_t sample_workspace(const SampleProblem &) { return 256; }

hipError_t launch_sample(const SampleProblem &p, void *, hipStream_t st) {
    const int idbits = bits_of((uint32_t)(p.V - 1));
    // V weights of at most 2^shift stay below 2^62; a weight is a whole number in a double
    const int shift = idbits > 12 ? 62 - idbits : 50;
    if (p.dtype == kBF16)
        hipLaunchKernelGGL((sample_row_kernel<kBF16>), dim3(p.R), dim3(NT), 0, st, p, shift, idbits);
    else
        hipLaunchKernelGGL((sample_row_kernel<kF32>), dim3(p.R), dim3(NT), 0, st, p, shift, idbits);
    return hipGetLastError();
}

}  // namespace dcd
