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
//
// Two launches, or three.  scan_kernel reads the logits once, in slices of 2,048 or 8,192 spread over the chip:
// the largest logit of every 64, and where no top-k bounds the row the slice's weight and (top-p) a
// coarse histogram of it; it writes the zeros of the probabilities.  pick_kernel has a workgroup per
// row, which brackets the cutoff from these, reads again only the pieces that can hold kept
// tokens, sorts what lies inside the bracket and draws.  Rows without any rule are not cut: their
// dense probabilities are one more pass, spread over the chip (whole_kernel).  Where the bracket
// fails (too many tokens inside, a top-k larger than the number of pieces) the row's workgroup
// searches the logits themselves (search_row).
#include "proposal.h"

namespace dcd {
namespace {

typedef unsigned long long u64;

constexpr int NT = 1024;             // threads of a row's workgroup
constexpr int NW = NT / 64;
constexpr int BITS = 11;             // of a key per search level
constexpr int BINS = 1 << BITS;
constexpr int MAXCHUNKS = 2048;      // pieces of a row for the draw of search_row
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

// exp(x), x <= 0, in 64 bits: x = (64 k + j) ln 2 / 64 + r, exp(x) = 2^k 2^(j/64) exp(r) with the 64
// powers in a table and a polynomial of degree 5 for |r| <= ln 2 / 128 (Tang's table-driven
// method; the terms left out are 4e-17).  ln 2 / 64 = kLnHi + kLnLo, kLnHi with 32 bits, so that
// its product with k is exact.
constexpr double kLnHi = 0x1.62e42fee00000p-7, kLnLo = 0x1.a39ef35793c76p-39, kPerLn = 0x1.71547652b82fep+6;

__device__ __forceinline__ void fill_table(double *table) {  // by the first 64 threads
    if (threadIdx.x < 64) table[threadIdx.x] = exp2((double)threadIdx.x / 64.0);
}
__device__ __forceinline__ double exp_of(double x, const double *table) {
    x = fmax(x, -800.0);
    const double q = rint(x * kPerLn), r = fma(-q, kLnLo, fma(-q, kLnHi, x));
    const int k = (int)q;
    double e = fma(r, 1.0 / 120, 1.0 / 24);
    e = fma(r, e, 1.0 / 6);
    e = fma(r, e, 0.5);
    e = fma(r, e, 1.0);
    const double t = table[k & 63];
    return ldexp(fma(t * r, e, t), k >> 6);
}

// Weights of a row relative to its largest logit, in 64 bits and as fixed-point numbers.
struct Weights {
    double top, inv_T, one;  // one: 2^shift, the fixed-point weight of the largest logit
    const double *table;
    __device__ __forceinline__ double exact(uint32_t key) const {
        return exp_of(((double)logit_of(key) - top) * inv_T, table);
    }
    __device__ __forceinline__ u64 to_fixed(double w) const { return (u64)rint(w * one); }
    __device__ __forceinline__ u64 fixed(uint32_t key) const { return to_fixed(exact(key)); }
};

// A row's rules; one that is outside its range leaves the row without a target.
struct Rules {
    float T, p, m, u;
    int k;       // 0: off
    bool ok;
    bool whole;  // no rule: every finite logit is kept
    __device__ __forceinline__ Rules(const SampleProblem &P, int r) {
        T = P.temperature ? P.temperature[r] : 1.f;
        p = P.top_p ? P.top_p[r] : 1.f;
        m = P.min_p ? P.min_p[r] : 0.f;
        u = P.u[r];
        k = P.top_k ? P.top_k[r] : 0;
        ok = T >= 0.f && T <= 3.4028235e38f && p >= 0.f && p <= 1.f && m >= 0.f && m <= 1.f && u >= 0.f && u < 1.f;
        if (T == 0.f) {
            T = 1.f;
            k = 1;
        }
        if (k < 0 || k >= P.V) k = 0;
        whole = ok && k == 0 && p == 1.f && m == 0.f;
    }
    __device__ __forceinline__ bool weighs() const { return ok && k == 0 && (whole || p < 1.f); }  // all of the row
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

// A row without a token.
__device__ __forceinline__ void no_token(const SampleProblem &P, int r) {
    P.tokens[r] = -1;
    if (P.kept) P.kept[r] = 0;
    if (P.logprob) P.logprob[r] = __uint_as_float(0x7fc00000u);
}

// One row by its workgroup alone, from the logits: any size, any rules.
struct SearchLds {
    Shared s;
    u64 csum[MAXCHUNKS];
    uint32_t top_key, bad;
};

template <int DT>
__device__ void search_row(const SampleProblem &P, int r, const Rules &rules, int shift, int idbits, SearchLds &lds,
                           const double *table) {
    Shared &S = lds.s;
    u64 *csum = lds.csum;
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const char *row = (const char *)P.logits + (size_t)r * P.stride * (DT == kBF16 ? 2 : 4);
    float *probs = P.probs ? P.probs + (size_t)r * P.V : nullptr;
    const int k = rules.k;
    const float top_p = rules.p, min_p = rules.m, u = rules.u;
    if (tid == 0) lds.top_key = lds.bad = 0;
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
    atomicMax(&lds.top_key, top);
    if (b) atomicOr(&lds.bad, 1u);
    u64 nfinite = block_sum(S, finite);
    top = lds.top_key;
    if (lds.bad || !rules.ok || top < kLowest) {
        if (probs)
            for (int i = tid; i < P.V; i += NT) probs[i] = 0.f;
        if (tid == 0) no_token(P, r);
        return;
    }
    const Weights W{(double)logit_of(top), 1.0 / (double)rules.T, (double)(1ull << shift), table};

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

template <int DT>
__global__ __launch_bounds__(NT) void search_kernel(SampleProblem P, int shift, int idbits) {
    __shared__ SearchLds lds;
    __shared__ double table[64];
    fill_table(table);
    search_row<DT>(P, blockIdx.x, Rules(P, blockIdx.x), shift, idbits, lds, table);
}

// ---------------------------------------------------------------------------
// The two launches.

constexpr int ST = 256;         // threads of a slice's workgroup
constexpr int PIECE = 64;       // logits per recorded maximum
constexpr int UNIT = 256;       // logits read again together
constexpr int HB = 256;         // histogram bins, 1/16 of a temperature wide, below the slice's largest logit
constexpr int SLICE = 8192;     // logits per slice (of a dense row's second pass, too)
constexpr int MAXV = 1 << 20;   // largest vocabulary of this path
constexpr int MAXLIST = 8192;   // tokens inside a row's bracket
constexpr int MAXSLICES = MAXV / SLICE > 512 ? MAXV / SLICE : 512;
constexpr float kBinLimit = 4194304.f;  // |bin numbers| up to here are exact in fp32

struct SliceStat {
    uint32_t top, bad, finite, unused;
    double mass;  // weight relative to the slice's largest logit
};

struct Scan {
    int slice, slices, pieces, units;  // logits per slice; slices, pieces and units of a row
    SliceStat *stat;                   // [R][slices]
    uint32_t *tops;                    // [R][pieces]: key of each piece's largest logit
    float *hist;                       // [R][slices][HB]
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

// Four logits from i on; -inf past the vocabulary.
template <int DT>
__device__ __forceinline__ f32x4 load4(const void *row, int i, int V) {
    f32x4 z = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (i + 3 < V) {
        if constexpr (DT == kBF16) {
            const u32x2 x = *reinterpret_cast<const u32x2_any *>((const uint16_t *)row + i);
            z = f32x4{__uint_as_float(x[0] << 16), __uint_as_float(x[0] & 0xffff0000u), __uint_as_float(x[1] << 16),
                      __uint_as_float(x[1] & 0xffff0000u)};
        } else {
            z = *reinterpret_cast<const f32x4_any *>((const float *)row + i);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < V) z[j] = load<DT>(row, i + j);
    }
    return z;
}

template <int DT>
__device__ __forceinline__ const char *row_of(const SampleProblem &P, int r) {
    return (const char *)P.logits + (size_t)r * P.stride * (DT == kBF16 ? 2 : 4);
}

// Bin number of a logit: the same in both launches, and monotone.
__device__ __forceinline__ float bin_of(float z, float per) { return floorf(z * per); }

// One slice: EPT logits per thread, held in registers between the maximum and the weights.
template <int DT, int EPT>
__global__ __launch_bounds__(ST) void scan_kernel(SampleProblem P, Scan L) {
    __shared__ double table[64], wmass[ST / 64];
    __shared__ float hist[HB];
    __shared__ uint32_t wtop[ST / 64], wbad[ST / 64], wfinite[ST / 64];
    const int s = blockIdx.x % L.slices, r = blockIdx.x / L.slices;
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const char *row = row_of<DT>(P, r);
    const int at = s * (ST * EPT) + tid * 4;
    f32x4 z[EPT / 4];
#pragma unroll
    for (int i = 0; i < EPT / 4; ++i) z[i] = load4<DT>(row, at + i * ST * 4, P.V);
    const Rules rules(P, r);
    if (P.probs && !rules.whole) {
        float *probs = P.probs + (size_t)r * P.V;
#pragma unroll
        for (int i = 0; i < EPT / 4; ++i) {
            const int e = at + i * ST * 4;
            if (e + 3 < P.V) {
                __builtin_nontemporal_store(f32x4{0.f, 0.f, 0.f, 0.f}, reinterpret_cast<f32x4_any *>(probs + e));
            } else {
                for (int j = e; j < P.V; ++j) probs[j] = 0.f;
            }
        }
    }
    const bool weighs = rules.weighs();
    if (weighs) {
        fill_table(table);
        hist[tid] = 0.f;
    }
    uint32_t top = 0, bad = 0, finite = 0;
    uint32_t *tops = L.tops + (size_t)r * L.pieces;
#pragma unroll
    for (int i = 0; i < EPT / 4; ++i) {
        uint32_t t = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bad |= !(z[i][j] < INFINITY);
            const uint32_t key = key_of(z[i][j]);
            t = max(t, key);
            finite += key >= kLowest;
        }
#pragma unroll
        for (int o = 1; o < PIECE / 4; o <<= 1) t = max(t, (uint32_t)__shfl_xor((int)t, o));
        if (lane % (PIECE / 4) == 0) tops[(at + i * ST * 4) / PIECE] = t;
        top = max(top, t);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        top = max(top, (uint32_t)__shfl_xor((int)top, o));
        bad |= (uint32_t)__shfl_xor((int)bad, o);
        finite += (uint32_t)__shfl_xor((int)finite, o);
    }
    if (lane == 0) {
        wtop[wave] = top;
        wbad[wave] = bad;
        wfinite[wave] = finite;
    }
    __syncthreads();
    bad = finite = 0;
#pragma unroll
    for (int w = 0; w < ST / 64; ++w) {
        top = max(top, wtop[w]);
        bad |= wbad[w];
        finite += wfinite[w];
    }
    SliceStat st{top, bad, finite, 0, 0.0};
    if (weighs && finite && !bad) {
        const Weights W{(double)logit_of(top), 1.0 / (double)rules.T, 1.0, table};
        const float per = 16.f / rules.T, first = bin_of(logit_of(top), per);
        double m = 0.0;
#pragma unroll
        for (int i = 0; i < EPT / 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t key = key_of(z[i][j]);
                if (key < kLowest) continue;
                const double w = W.exact(key);
                m += w;
                if (rules.p < 1.f) atomicAdd(&hist[(int)fminf(first - bin_of(z[i][j], per), HB - 1.f)], (float)w);
            }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) m += __shfl_xor(m, o);
        if (lane == 0) wmass[wave] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < ST / 64; ++w) st.mass += wmass[w];
        if (rules.p < 1.f) L.hist[((size_t)r * L.slices + s) * HB + tid] = hist[tid];
    }
    if (tid == 0) L.stat[(size_t)r * L.slices + s] = st;
}

// What a row's workgroup keeps in LDS.
struct PickLds {
    double table[64];
    union {
        u64 list[MAXLIST];               // (key, ~id) of the tokens inside the bracket
        uint32_t tops[2 * MAXLIST];      // before: the pieces' maxima
        SearchLds search;                // instead: the search of the logits themselves
    };
    u64 unit[MAXV / UNIT];               // kept weight per unit
    uint16_t todo[MAXV / UNIT];          // units that may hold kept tokens
    float bins[HB], scale[MAXSLICES];
    int below[MAXSLICES];                // bins from the row's first to the slice's first
    u64 wmass[NW];
    uint32_t wcount[NW];
    u64 total, at, sure_mass;
    uint32_t top, bad, finite, ntodo, nlist, nsure, pick, lo_bin, hi_bin;
};
static_assert(sizeof(PickLds) <= 160 * 1024 && MAXV / PIECE <= 2 * MAXLIST, "LDS of a row");

// Exclusive sums over the workgroup of (count, mass), in thread order.
__device__ __forceinline__ void block_scan(PickLds &S, uint32_t &c, u64 &m) {
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
__device__ __forceinline__ u64 block_sum(PickLds &S, u64 m) {
    uint32_t c = 0;
    const u64 mine = m;
    block_scan(S, c, m);
    if (threadIdx.x == NT - 1) S.total = m + mine;
    __syncthreads();
    return S.total;
}

// A row's largest logit and whether it has a target; with `weigh` the fixed-point weight of each slice
// in the thread of its number (the others: 0).
__device__ __forceinline__ bool gather_stats(PickLds &S, const Scan &L, int r, const Rules &rules, int shift, Weights &W,
                                             u64 &mine) {
    const int tid = threadIdx.x;
    if (tid == 0) S.top = S.bad = S.finite = 0;
    fill_table(S.table);
    __syncthreads();
    SliceStat st{0, 0, 0, 0, 0.0};
    if (tid < L.slices) st = L.stat[(size_t)r * L.slices + tid];
    if (tid < L.slices) {
        atomicMax(&S.top, st.top);
        if (st.bad) atomicOr(&S.bad, 1u);
        atomicAdd(&S.finite, st.finite);
    }
    __syncthreads();
    W = Weights{(double)logit_of(S.top), 1.0 / (double)rules.T, (double)(1ull << shift), S.table};
    mine = 0;
    if (S.bad || !rules.ok || S.top < kLowest) return false;
    if (rules.weighs() && st.finite) {
        const double scale = W.exact(st.top);
        mine = W.to_fixed(st.mass * scale);
        if (rules.p < 1.f) {
            const float per = 16.f / rules.T, d = bin_of((float)W.top, per) - bin_of(logit_of(st.top), per);
            S.scale[tid] = (float)scale;
            S.below[tid] = (int)fminf(d, (float)HB);
        }
    } else if (tid < L.slices) {
        S.scale[tid] = 0.f;
        S.below[tid] = HB;
    }
    return true;
}

__device__ __forceinline__ float log_of(const Weights &W, uint32_t key, u64 total) {
    return (float)(((double)logit_of(key) - W.top) * W.inv_T - log((double)total / W.one));
}

// The draw of a row without rules: the slice where the running weight exceeds the target, then
// the token in it.
template <int DT>
__device__ __forceinline__ void whole_draw(const SampleProblem &P, const Scan &L, int r, const Rules &rules,
                                           const Weights &W, u64 mine, PickLds &S) {
    const int tid = threadIdx.x;
    const u64 total = block_sum(S, mine);
    const u64 target = (u64)((double)rules.u * (double)total);  // exceeds: > floor
    uint32_t none = 0;
    u64 m = mine;
    block_scan(S, none, m);
    if (m <= target && m + mine > target) {
        S.pick = tid;
        S.at = m;
    }
    __syncthreads();
    const int per = L.slice / NT, e0 = (int)S.pick * L.slice + tid * per;
    const char *row = row_of<DT>(P, r);
    const u64 at = S.at;
    m = 0;
    // the slice's last token (of any weight, if there is one), should rounding leave the target above them all
    constexpr uint32_t kWeighs = 0x80000000u;
    uint32_t last = 0;
    for (int j = 0; j < per; ++j) {
        const uint32_t key = e0 + j < P.V ? key_of(load<DT>(row, e0 + j)) : 0;
        if (key < kLowest) continue;
        const u64 w = W.fixed(key);
        m += w;
        last = max(last, (uint32_t)(e0 + j) | (w ? kWeighs : 0u));
    }
    __syncthreads();
    if (tid == 0) S.pick = 0;
    __syncthreads();
    atomicMax(&S.pick, last);
    const u64 own = m;
    block_scan(S, none, m);
    m += at;
    if (tid == 0) S.ntodo = S.pick & ~kWeighs;
    __syncthreads();
    if (m <= target && m + own > target) {
        for (int j = 0; j < per; ++j) {
            const uint32_t key = e0 + j < P.V ? key_of(load<DT>(row, e0 + j)) : 0;
            if (key >= kLowest) m += W.fixed(key);
            if (m > target) {
                S.ntodo = e0 + j;
                break;
            }
        }
    }
    __syncthreads();
    if (tid == 0) {
        const int token = (int)S.ntodo;
        P.tokens[r] = token;
        if (P.logprob) P.logprob[r] = log_of(W, key_of(load<DT>(row, token)), total);
        if (P.kept) P.kept[r] = (int32_t)S.finite;
    }
}

// Descending order of n numbers in LDS (n a power of two, at least 128).  Pairs up to 64 apart stay
// within a wave.
__device__ __forceinline__ void sort_list(u64 *list, int n) {
    for (int k = 2; k <= n; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int t = threadIdx.x; t < n / 2; t += NT) {
                const int i = 2 * j * (t / j) + t % j;
                const u64 a = list[i], b = list[i + j];
                if ((a < b) == ((i & k) == 0)) {
                    list[i] = b;
                    list[i + j] = a;
                }
            }
            if (j > 64 || (j == 1 && k >= 128)) {
                __syncthreads();
            } else {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_wave_barrier();
            }
        }
    __syncthreads();
}

// A row's token.
template <int DT>
__device__ void pick_row(const SampleProblem &P, const Scan &L, int r, int shift, int idbits, PickLds &S) {
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const Rules rules(P, r);
    const char *row = row_of<DT>(P, r);
    Weights W;
    u64 mine;
    if (!gather_stats(S, L, r, rules, shift, W, mine)) {
        if (tid == 0) no_token(P, r);
        return;
    }
    if (rules.whole) {
        whole_draw<DT>(P, L, r, rules, W, mine, S);
        return;
    }
    auto search = [&] {
        __syncthreads();
        search_row<DT>(P, r, rules, shift, idbits, S.search, S.table);
    };
    // The bracket: tokens that are surely kept by top-k and top-p, and the ones that may be.  By
    // logit (key >= least) or by histogram bin (from hi_bin on sure, from lo_bin on possible; min-p is
    // decided token by token).
    const int k = min(rules.k, (int)S.finite);
    const bool bins = rules.k == 0 && rules.p < 1.f, all_sure = rules.k == 0 && !bins;
    uint32_t least = kLowest;
    float per = 0.f, lo = 0.f, hi = 0.f;
    u64 total = 0;
    const uint32_t *tops = L.tops + (size_t)r * L.pieces;
    if (tid == 0) S.ntodo = S.nlist = S.nsure = S.sure_mass = 0;
    if (bins) {
        total = block_sum(S, mine);
        per = 16.f / rules.T;
        const float first = bin_of((float)W.top, per);
        if (!(fabsf(first) < kBinLimit)) return search();
        // the row's histogram, in units of its largest weight, and its running sum
        float h = 0.f;
        if (tid < HB)
            for (int s = 0; s < L.slices; ++s) {
                const int b = tid - S.below[s];
                if (b >= 0 && b < HB - 1) h += L.hist[((size_t)r * L.slices + s) * HB + b] * S.scale[s];
            }
        if (tid < HB) S.bins[tid] = h;
        __syncthreads();
        for (int o = 1; o < HB; o <<= 1) {
            const float x = tid >= o && tid < HB ? S.bins[tid - o] : 0.f;
            __syncthreads();
            if (tid < HB) S.bins[tid] += x;
            __syncthreads();
        }
        if (tid == 0) S.lo_bin = S.hi_bin = HB;
        __syncthreads();
        // the sums in fp32 are good to far better than a thousandth
        const float goal = (float)((double)rules.p * ((double)total / W.one));
        if (tid < HB - 1) {
            if (S.bins[tid] * 1.001f >= goal) atomicMin(&S.hi_bin, (uint32_t)tid);
            if (S.bins[tid] * 0.999f >= goal) atomicMin(&S.lo_bin, (uint32_t)tid);
        }
        __syncthreads();
        if (S.lo_bin >= HB - 1) return search();
        lo = first - (float)S.lo_bin;
        hi = first - (float)S.hi_bin;
    } else if (all_sure) {
        // the logit of weight min_p, a little lower
        const double z = W.top + (double)rules.T * log((double)rules.m);
        const float f = (float)(z - fabs(z) * 1e-6 - 1e-30);
        least = f >= -3.4028235e38f ? max(key_of(f), kLowest) : kLowest;
    } else if (k <= L.pieces) {
        // at least k tokens reach the k-th largest of the pieces' maxima; its upper 16 bits do
        for (int i = tid; i < L.pieces; i += NT) S.tops[i] = tops[i];
        __syncthreads();
        uint32_t prefix = 0;
        for (int bit = 30; bit >= 16; bit -= 2) {
            u64 counts = 0;
            for (int i = tid; i - tid < L.pieces; i += NT) {
                const uint32_t key = i < L.pieces ? S.tops[i] : 0;
#pragma unroll
                for (int c = 1; c < 4; ++c)
                    counts += (u64)__popcll(__ballot(i < L.pieces && key >= (prefix | (uint32_t)c << bit))) << (21 * (c - 1));
            }
            __syncthreads();
            if (lane == 0) S.wmass[wave] = counts;
            __syncthreads();
            counts = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w) counts += S.wmass[w];
            for (int c = 3; c > 0; --c)
                if ((int)(counts >> (21 * (c - 1)) & 0x1fffff) >= k) {
                    prefix |= (uint32_t)c << bit;
                    break;
                }
        }
        least = max(prefix, kLowest);
    }
    auto possible = [&](uint32_t key) { return key >= least && (!bins || bin_of(logit_of(key), per) >= lo); };
    auto sure = [&](uint32_t key) { return all_sure || (bins && bin_of(logit_of(key), per) > hi); };
    // units that hold possible tokens
    __syncthreads();
    for (int i = tid; i < L.units; i += NT) {
        uint32_t t = 0;
#pragma unroll
        for (int j = 0; j < UNIT / PIECE; ++j) t = max(t, tops[i * (UNIT / PIECE) + j]);
        S.unit[i] = 0;
        if (possible(t)) S.todo[atomicAdd(&S.ntodo, 1u)] = (uint16_t)i;
    }
    __syncthreads();
    const int ntodo = (int)S.ntodo;
    for (int q = wave; q < ntodo; q += NW) {
        const int unit = S.todo[q], e = unit * UNIT + lane * 4;
        const f32x4 z = load4<DT>(row, e, P.V);
        u64 m = 0;
        uint32_t n = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t key = key_of(z[j]);
            const bool in = key >= kLowest && possible(key), is_sure = in && sure(key);
            if (is_sure) {
                const double w = W.exact(key);
                if (w >= (double)rules.m) {
                    m += W.to_fixed(w);
                    ++n;
                }
            }
            const u64 vote = __ballot(in && !is_sure);
            if (vote) {
                uint32_t base = 0;
                if (lane == 0) base = atomicAdd(&S.nlist, (uint32_t)__popcll(vote));
                base = __shfl((int)base, 0) + __popcll(vote & ((1ull << lane) - 1));
                if (in && !is_sure && base < MAXLIST) S.list[base] = (u64)key << 32 | (uint32_t)~(e + j);
            }
        }
        if (__ballot(n > 0)) {
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                m += (u64)__shfl_xor((long long)m, o);
                n += (uint32_t)__shfl_xor((int)n, o);
            }
            if (lane == 0) {
                S.unit[unit] = m;
                atomicAdd(&S.sure_mass, m);
                atomicAdd(&S.nsure, n);
            }
        }
    }
    __syncthreads();
    const int nlist = (int)S.nlist;
    if (nlist > MAXLIST || (rules.k && nlist < k) || (bins && !nlist)) return search();
    const u64 sure_mass = S.sure_mass;
    int n = 0;  // kept tokens of the list
    if (nlist) {
        int size = 128;
        while (size < nlist) size <<= 1;
        for (int i = nlist + tid; i < size; i += NT) S.list[i] = 0;
        __syncthreads();
        sort_list(S.list, size);
        const int each = (size + NT - 1) / NT;
        const int limit = rules.k ? k : nlist;
        u64 m = 0;
        for (int i = tid * each; i < min((tid + 1) * each, limit); ++i) m += W.fixed((uint32_t)(S.list[i] >> 32));
        const u64 own = m;
        uint32_t none = 0;
        block_scan(S, none, m);
        if (rules.k && rules.p < 1.f) total = block_sum(S, own);
        n = limit;
        if (rules.p < 1.f) {
            u64 goal = (u64)ceil((double)rules.p * (double)total);
            goal = goal < 1 ? 1 : goal > total ? total : goal;
            if (tid == 0) S.pick = 0xffffffffu;
            __syncthreads();
            m += sure_mass;
            if (m < goal && m + own >= goal)
                for (int i = tid * each; i < min((tid + 1) * each, limit); ++i) {
                    m += W.fixed((uint32_t)(S.list[i] >> 32));
                    if (m >= goal) {
                        S.pick = i + 1;
                        break;
                    }
                }
            __syncthreads();
            if (S.pick == 0xffffffffu) {
                if (sure_mass < goal) return search();
                n = 0;
            } else {
                n = (int)S.pick;
            }
        }
        if (rules.m > 0.f) {
            uint32_t c = 0;
            for (int i = tid * each; i < min((tid + 1) * each, n); ++i)
                c += W.exact((uint32_t)(S.list[i] >> 32)) >= (double)rules.m;
            n = (int)block_sum(S, c);
        }
        for (int i = tid; i < n; i += NT) {
            const u64 x = S.list[i];
            atomicAdd(&S.unit[(uint32_t)~x / UNIT], W.fixed((uint32_t)(x >> 32)));
        }
        __syncthreads();
    }
    const Cut cut = n ? Cut{(uint32_t)(S.list[n - 1] >> 32), (uint32_t)~S.list[n - 1]} : Cut{0xffffffffu, 0u};
    // the unit where the running weight exceeds the target, then the token in it
    const int each = (L.units + NT - 1) / NT;
    u64 m = 0;
    for (int i = tid * each; i < min((tid + 1) * each, L.units); ++i) m += S.unit[i];
    const u64 own = m;
    uint32_t none = 0;
    const u64 all = block_sum(S, own);
    const u64 target = (u64)((double)rules.u * (double)all);  // exceeds: > floor
    block_scan(S, none, m);
    if (m <= target && m + own > target)
        for (int i = tid * each;; ++i) {
            if (m + S.unit[i] > target) {
                S.pick = i;
                S.at = m;
                break;
            }
            m += S.unit[i];
        }
    __syncthreads();
    const double scale = W.one / (double)all;
    if (wave == 0) {
        const int e = (int)S.pick * UNIT + lane * 4;
        const f32x4 z = load4<DT>(row, e, P.V);
        u64 w[4], run = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t key = key_of(z[j]);
            w[j] = 0;
            if (key >= kLowest && possible(key)) {
                const double x = W.exact(key);
                if (x >= (double)rules.m && (sure(key) || cut.keeps(key, e + j))) w[j] = W.to_fixed(x);
            }
            run += w[j];
        }
        const u64 own4 = run;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const u64 x = shfl_up64(run, o);
            if (lane >= o) run += x;
        }
        run += S.at;
        const u64 over = __ballot(run > target);
        if (lane == __ffsll((long long)over) - 1) {
            run -= own4;
            int token = -1;
            float logit = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                run += w[j];
                if (token < 0 && run > target) {
                    token = e + j;
                    logit = z[j];
                }
            }
            P.tokens[r] = token;
            if (P.logprob) P.logprob[r] = log_of(W, key_of(logit), all);
            if (P.kept) P.kept[r] = (int32_t)(S.nsure + n);
        }
    }
    if (!P.probs) return;
    float *probs = P.probs + (size_t)r * P.V;
    for (int i = tid; i < n; i += NT) {
        const u64 x = S.list[i];
        probs[(uint32_t)~x] = (float)(W.exact((uint32_t)(x >> 32)) * scale);
    }
    if (S.nsure == 0) return;
    for (int q = wave; q < ntodo; q += NW) {
        const int e = S.todo[q] * UNIT + lane * 4;
        const f32x4 z = load4<DT>(row, e, P.V);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t key = key_of(z[j]);
            if (key < kLowest || !possible(key) || !sure(key)) continue;
            const double w = W.exact(key);
            if (w >= (double)rules.m) probs[e + j] = (float)(w * scale);
        }
    }
}

template <int DT>
__global__ __launch_bounds__(NT) void pick_kernel(SampleProblem P, Scan L, int shift, int idbits) {
    __shared__ PickLds S;
    pick_row<DT>(P, L, blockIdx.x, shift, idbits, S);
}

// The dense probabilities of the rows without rules, a slice of SLICE tokens per workgroup.
template <int DT>
__global__ __launch_bounds__(ST) void whole_kernel(SampleProblem P, Scan L, int shift) {
    __shared__ double table[64];
    __shared__ uint32_t top_key, bad;
    __shared__ u64 wmass[ST / 64];
    const int per = (P.V + SLICE - 1) / SLICE, r = blockIdx.x / per, s = blockIdx.x % per, tid = threadIdx.x;
    const Rules rules(P, r);
    if (!rules.whole) return;
    const char *row = row_of<DT>(P, r);
    f32x4 z[SLICE / ST / 4];
#pragma unroll
    for (int i = 0; i < SLICE / ST / 4; ++i) z[i] = load4<DT>(row, s * SLICE + (i * ST + tid) * 4, P.V);
    fill_table(table);
    if (tid == 0) top_key = bad = 0;
    __syncthreads();
    const SliceStat *stat = L.stat + (size_t)r * L.slices;
    uint32_t top = 0, b = 0;
    for (int i = tid; i < L.slices; i += ST) {
        top = max(top, stat[i].top);
        b |= stat[i].bad;
    }
    atomicMax(&top_key, top);
    if (b) atomicOr(&bad, 1u);
    __syncthreads();
    const Weights W{(double)logit_of(top_key), 1.0 / (double)rules.T, (double)(1ull << shift), table};
    const bool ok = !bad && top_key >= kLowest;
    u64 total = 0;
    for (int i = tid; i < L.slices; i += ST)
        if (ok && stat[i].finite) total += W.to_fixed(stat[i].mass * W.exact(stat[i].top));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += (u64)__shfl_xor((long long)total, o);
    if (tid % 64 == 0) wmass[tid / 64] = total;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < ST / 64; ++w) total += wmass[w];
    const double scale = ok ? W.one / (double)total : 0.0;
    float *probs = P.probs + (size_t)r * P.V;
#pragma unroll
    for (int i = 0; i < SLICE / ST / 4; ++i) {
        const int e = s * SLICE + (i * ST + tid) * 4;
        f32x4 q;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t key = key_of(z[i][j]);
            q[j] = ok && key >= kLowest ? (float)(W.exact(key) * scale) : 0.f;
        }
        if (e + 3 < P.V) {
            __builtin_nontemporal_store(q, reinterpret_cast<f32x4_any *>(probs + e));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e + j < P.V) probs[e + j] = q[j];
        }
    }
}

int bits_of(uint32_t x) {
    int b = 0;
    while (b < 32 && x >> b) ++b;
    return b;
}

// Slices of 8,192 logits, or of 2,048 where the rows are too few to fill the chip with those.
Scan layout(const SampleProblem &p, char *ws, size_t &bytes) {
    Scan L{};
    const int large = (p.V + SLICE - 1) / SLICE;
    L.slice = (long long)p.R * large < 2 * kCus && p.V <= 2048 * MAXSLICES ? 2048 : SLICE;
    L.slices = (p.V + L.slice - 1) / L.slice;
    L.pieces = L.slices * L.slice / PIECE;
    L.units = L.slices * L.slice / UNIT;
    size_t off = 0;
    auto take = [&](size_t n) {
        char *at = ws ? ws + off : nullptr;
        off += (n + 255) / 256 * 256;
        return at;
    };
    const size_t R = (size_t)p.R;
    L.stat = (SliceStat *)take(R * L.slices * sizeof(SliceStat));
    L.tops = (uint32_t *)take(R * L.pieces * 4);
    L.hist = (float *)take(R * L.slices * HB * 4);
    bytes = off ? off : 256;
    return L;
}

template <int DT>
hipError_t launch(const SampleProblem &p, char *ws, hipStream_t st) {
    const int idbits = bits_of((uint32_t)(p.V - 1));
    // V weights of at most 2^shift stay below 2^62; a weight is a whole number in a double
    const int shift = idbits > 12 ? 62 - idbits : 50;
    if (p.V > MAXV) {
        hipLaunchKernelGGL((search_kernel<DT>), dim3(p.R), dim3(NT), 0, st, p, shift, idbits);
        return hipGetLastError();
    }
    size_t bytes;
    const Scan L = layout(p, ws, bytes);
    const dim3 scan((unsigned)(p.R * L.slices));
    if (L.slice == SLICE)
        hipLaunchKernelGGL((scan_kernel<DT, SLICE / ST>), scan, dim3(ST), 0, st, p, L);
    else
        hipLaunchKernelGGL((scan_kernel<DT, 2048 / ST>), scan, dim3(ST), 0, st, p, L);
    hipLaunchKernelGGL((pick_kernel<DT>), dim3((unsigned)p.R), dim3(NT), 0, st, p, L, shift, idbits);
    if (p.probs) {
        const dim3 whole((unsigned)(p.R * ((p.V + SLICE - 1) / SLICE)));
        hipLaunchKernelGGL((whole_kernel<DT>), whole, dim3(ST), 0, st, p, L, shift);
    }
    return hipGetLastError();
}

}  // namespace

size_t sample_workspace(const SampleProblem &p) {
    if (p.V > MAXV) return 256;
    size_t bytes;
    layout(p, nullptr, bytes);
    return bytes;
}

hipError_t launch_sample(const SampleProblem &p, void *ws, hipStream_t st) {
    return p.dtype == kBF16 ? launch<kBF16>(p, (char *)ws, st) : launch<kF32>(p, (char *)ws, st);
}

}  // namespace dcd
