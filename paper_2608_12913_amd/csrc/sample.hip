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
// call.  A token under half a step weighs nothing and is never drawn.  Slices of tokens are rounded as a
// whole where they are summed before the largest weight is known, which moves a sum by about half a
// step per token (2^-29 of the largest weight at 128,256 tokens).
//
// Two launches, or three.  scan_kernel reads the logits once, in slices of 2,048 or 8,192 spread over
// the chip: the largest logit of every 64 (of fewer in short vocabularies) and, where no top-k bounds
// the row, a histogram of the slice's weight; it writes the zeros of the probabilities.  pick_kernel
// has a workgroup per row, which brackets the cutoff from these to a few hundred tokens, reads again
// only the pieces that can hold one, puts what lies inside the bracket in order, and draws.  What lies
// surely above the bracket (rows without top-k) is spread over the chip once more for its dense
// probabilities (spread_kernel).  Where the bracket fails (too many tokens inside, a top-k larger
// than the number of pieces) the row's workgroup searches the logits themselves (search_row), as it
// does for vocabularies under 4 or above 2^20 tokens.
//
// What bounds it, rows of 128,256 fp32 logits without dense probabilities, us (of which a streaming
// read needs 0.1, 10 and 77):
//                         1 row   128 rows   1,024 rows
//   argmax                 19.4     33         130
//   top-k 50               20.4     34         132    memory, and 20 us of a row's dependent steps
//   min-p 0.05             22.5     41         159
//   no rule                11.9     41         198    a 64-bit exponential per logit
//   top-p 0.9              31.3     58         235    the same, and the slices' histograms
//   top-p 0.9, flat        104      130        430    a bracket of thousands: order, second reading
// A row by one workgroup from the logits alone, with a radix search of all of them per level, took
// 301 us (1 row, top-k and top-p) and 2,156 us (1,024 rows of mixed rules, 345 now).
#include "proposal.h"

namespace dcd {
namespace {

typedef unsigned long long u64;

// Threads of a row's workgroup.  256 or 1,024 instead: one row of top-p 42 or 37 us (32 with 512), of a
// flat nucleus 187 or 101 (117), 512 rows of top-k 64 or 87 (66), of a flat nucleus 295 or 291 (251).
constexpr int NT = 512;
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

// 2^(y / 128), y <= 0, in 64 bits: y = 128 k + j + f, 2^k 2^(j/128) 2^(f/128) with the 128 powers in a
// table and a polynomial of degree 4 for |f| <= 1/2 (the table-driven method of Tang; the terms
// left out are 1e-15).
constexpr int POWERS = 1 << 7;
constexpr double kLn = 0.693147180559945309417 / POWERS;

__device__ __forceinline__ void fill_table(double *table) {  // by the first POWERS threads
    if (threadIdx.x < POWERS) table[threadIdx.x] = exp2((double)threadIdx.x / POWERS);
}
__device__ __forceinline__ double power_of(double y, const double *table) {
    y = fmax(y, -160000.0);  // (2^-1250 is 0)
    const double q = rint(y), f = y - q;
    const int k = (int)q;
    double e = fma(f, kLn * kLn * kLn * kLn / 24, kLn * kLn * kLn / 6);
    e = fma(f, e, kLn * kLn / 2);
    e = fma(f, e, kLn);
    const double t = table[k & (POWERS - 1)];
    return ldexp(fma(t * f, e, t), k >> 7);
}

// Weights of a row relative to its largest logit, in 64 bits and as fixed-point numbers of at most
// 2^50.
struct Weights {
    double top, per, one;  // per: 128 / (T ln 2); one: the fixed-point weight of the largest logit
    const double *table;
    __device__ __forceinline__ Weights(uint32_t top_key, float T, int shift, const double *table_)
        : top((double)logit_of(top_key)), per(1.0 / kLn / (double)T), one((double)(1ull << shift)), table(table_) {}
    __device__ __forceinline__ double of(float z) const { return power_of(((double)z - top) * per, table); }
    __device__ __forceinline__ double exact(uint32_t key) const { return of(logit_of(key)); }
    __device__ __forceinline__ u64 to_fixed(double w) const {  // w <= 1: rounded by the sum with 2^52
        return (u64)__double_as_longlong(fma(w, one, 0x1p52)) - 0x4330000000000000ull;
    }
    __device__ __forceinline__ u64 fixed(uint32_t key) const { return to_fixed(exact(key)); }
    __device__ __forceinline__ double log_weight(uint32_t key) const { return ((double)logit_of(key) - top) * per * kLn; }
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
    __device__ __forceinline__ bool weighs() const { return ok && k == 0; }  // all of the row
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
__device__ __forceinline__ Cut search(Shared &S, const ForEach &each, const Weights &W, u64 target, int idbits, u64 &kept) {
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
__device__ __forceinline__ void search_row(const SampleProblem &P, int r, const Rules &rules, int shift, int idbits, SearchLds &lds,
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
    const Weights W(top, rules.T, shift, table);

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
                m += W.to_fixed(w);
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
            const u64 mine = kept(i, key, w) ? W.to_fixed(w) : 0;
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
                            (float)(W.log_weight(key) - log((double)total / W.one));
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
    __shared__ double table[POWERS];
    fill_table(table);
    search_row<DT>(P, blockIdx.x, Rules(P, blockIdx.x), shift, idbits, lds, table);
}

// ---------------------------------------------------------------------------
// The launches.

constexpr int ST = 256;         // threads of a slice's workgroup
// Logits per recorded maximum: 4 or 16 where a row still has no more than MANY of those, else 64.  A top-k
// needs at least k maxima, and its bracket is the narrower the more there are, but each is also looked
// at: 16 rows of 32,003 with top-k 50 take 19.8 us with pieces of 16, 24.8 with 4, 20.7 with 64 (which a
// top-k above 501 cannot use, and then the logits are searched: 11 rows of 3,779 took 114 us, 25 with 4).
constexpr int PIECE = 64;
constexpr int MANY = 2048;
constexpr int UNIT = 256;       // logits of a wave's load: the draw goes slice, unit, token
constexpr int HB = 256;         // histogram bins, 1/16 of a temperature wide, below the slice's largest logit
constexpr int SLICE = 8192;     // logits per slice (of a dense row's second pass, too)
constexpr int MAXV = 1 << 20;   // largest vocabulary of this path
constexpr int MAXLIST = 4096;   // tokens inside a row's bracket
constexpr int MAXTODO = 4096;   // pieces that may hold one, by number (more: every piece of the row)
constexpr int MAXCOUNTED = 512;  // up to so many are put in order by counting (240: 5.7 us, sorted in pairs 9)
constexpr int kHistShift = 50;  // 8,192 weights of a slice stay below 2^63
constexpr int MAXSLICES = MAXV / SLICE > 512 ? MAXV / SLICE : 512;
constexpr float kBinLimit = 4194304.f;  // |bin numbers| up to here are exact in fp32

struct SliceStat {
    uint32_t top, bad, finite, unused;
    u64 mass;  // rows without top-k: the slice's weight, relative to its largest logit, at 2^kHistShift
};

// What pick_kernel leaves for a row's dense probabilities.
struct Spread {
    double scale;    // of a weight
    uint32_t top;    // key of the row's largest logit
    uint32_t least;  // every token from this key on is kept (0xffffffff: none)
};

struct Scan {
    int slice, slices, bits, pieces;  // logits per slice, 2^bits per piece; slices and pieces of a row
    SliceStat *stat;                   // [R][slices]
    uint16_t *tops;                    // [R][pieces]: upper half of the key of each piece's largest logit
    u64 *hist;                         // [R][slices][HB]: weights at 2^kHistShift (the last bin stays 0)
    Spread *spread;                    // [R]
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

// Four logits from i on; -inf past the vocabulary (of at least four: where they would pass its end, the
// last four are loaded and moved).
template <int DT>
__device__ __forceinline__ f32x4 load4(const void *row, int i, int V) {
    const int at = min(i, V - 4), d = i - at;
    f32x4 z;
    if constexpr (DT == kBF16) {
        const u32x2 x = *reinterpret_cast<const u32x2_any *>((const uint16_t *)row + at);
        z = f32x4{__uint_as_float(x[0] << 16), __uint_as_float(x[0] & 0xffff0000u), __uint_as_float(x[1] << 16),
                  __uint_as_float(x[1] & 0xffff0000u)};
    } else {
        z = *reinterpret_cast<const f32x4_any *>((const float *)row + at);
    }
    if (d) {
        const float none = -INFINITY, z1 = z[1], z2 = z[2], z3 = z[3];
        z[0] = d == 1 ? z1 : d == 2 ? z2 : d == 3 ? z3 : none;
        z[1] = d == 1 ? z2 : d == 2 ? z3 : none;
        z[2] = d == 1 ? z3 : none;
        z[3] = none;
    }
    return z;
}

template <int DT>
__device__ __forceinline__ const char *row_of(const SampleProblem &P, int r) {
    return (const char *)P.logits + (size_t)r * P.stride * (DT == kBF16 ? 2 : 4);
}

// Bin number of a logit: the same in both launches, and monotone.
__device__ __forceinline__ float bin_of(float z, float per) { return floorf(z * per); }

// Sums along a wave in registers: row shifts within 16 lanes, then broadcasts of a row's last lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 shifted(u64 x) {
    const int lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xf, false);
    return (u64)(uint32_t)hi << 32 | (uint32_t)lo;
}
__device__ __forceinline__ u64 wave_scan(u64 x) {  // inclusive
    x += shifted<0x111, 0xf>(x);
    x += shifted<0x112, 0xf>(x);
    x += shifted<0x114, 0xf>(x);
    x += shifted<0x118, 0xf>(x);
    x += shifted<0x142, 0xa>(x);
    x += shifted<0x143, 0xc>(x);
    return x;
}
__device__ __forceinline__ u64 last_lane(u64 x) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, 63);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), 63);
    return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 wave_sum(u64 x) { return last_lane(wave_scan(x)); }

// One slice: EPT logits per thread, held in registers between the maximum and the weights.
template <int DT, int EPT>
__global__ __launch_bounds__(ST) void scan_kernel(SampleProblem P, Scan L) {
    __shared__ double table[POWERS];
    __shared__ u64 hist[HB], wmass[ST / 64];
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
        hist[tid] = 0;
    }
    uint32_t top = 0, bad = 0, finite = 0;
    uint16_t *tops = L.tops + (size_t)r * L.pieces;
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
        const int e = at + i * ST * 4;
        for (int o = 1; o < 1 << (L.bits - 2); o <<= 1) t = max(t, (uint32_t)__shfl_xor((int)t, o));
        if ((e & ((1 << L.bits) - 1)) == 0 && e >> L.bits < L.pieces) tops[e >> L.bits] = (uint16_t)(t >> 16);
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
    SliceStat st{top, bad, finite, 0, 0};
    if (weighs && finite && !bad) {
        const Weights W(top, rules.T, kHistShift, table);
        u64 m = 0;
        const float per = 16.f / rules.T, first = bin_of(logit_of(top), per);
        // with min-p alone, only the bins above its bound are read (4: for the roundings on the way to it)
        const float most = rules.p == 1.f && !rules.whole ? fminf(4.f - 16.f * logf(rules.m), HB - 1.f) : INFINITY;
#pragma unroll
        for (int i = 0; i < EPT / 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float bin = first - bin_of(z[i][j], per);
                if (z[i][j] == -INFINITY || bin >= most) continue;
                const u64 w = W.to_fixed(W.of(z[i][j]));
                m += w;
                if (!rules.whole && w && bin < HB - 1.f) atomicAdd(&hist[(int)bin], w);
            }
        m = wave_sum(m);
        if (lane == 0) wmass[wave] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < ST / 64; ++w) st.mass += wmass[w];
        if (!rules.whole) L.hist[((size_t)r * L.slices + s) * HB + tid] = hist[tid];
    }
    if (tid == 0) L.stat[(size_t)r * L.slices + s] = st;
}

// What a row's workgroup keeps in LDS.
struct PickLds {
    double table[POWERS];
    union {
        u64 list[MAXLIST + MAXCOUNTED];  // (key, ~id) of the tokens inside the bracket; the last ones: in order
        SearchLds search;                // instead: the search of the logits themselves
    };
    uint16_t todo[MAXTODO];      // pieces that may hold tokens of the bracket
    double scale[MAXSLICES];     // a slice's largest weight
    int below[MAXSLICES];        // bins from the row's first to the slice's first
    u64 kept[MAXSLICES];         // kept weight per slice
    u64 unit[SLICE / UNIT];      // and per unit of a slice
    u64 wave[2][NW];        // of BlockScan
    u64 reach[8];                // three counts of pieces' maxima for each pair of bits
    u64 at;
    uint32_t top[NW], bad[NW], finite[NW];
    uint32_t ntodo, nlist, pick, lo_bin, hi_bin;
};
static_assert(sizeof(PickLds) <= 64 * 1024, "two rows and more share a CU");

// Exclusive sums over the workgroup in thread order, and the total.  Calls take the two buffers in
// turns, so that one barrier each is enough: a buffer is written again only after the barrier of the
// call in between, which everybody reaches with the earlier one read.
struct BlockScan {
    PickLds &S;
    int turn = 0;
    __device__ __forceinline__ u64 operator()(u64 x, u64 &total) {
        const int wave = threadIdx.x / 64;
        const u64 in = wave_scan(x);
        if (threadIdx.x % 64 == 63) S.wave[turn][wave] = in;
        __syncthreads();
        u64 before = 0;
        total = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const u64 y = S.wave[turn][w];
            before += w < wave ? y : 0;
            total += y;
        }
        turn ^= 1;
        return before + in - x;
    }
    __device__ __forceinline__ u64 sum(u64 x) {
        u64 total;
        (*this)(x, total);
        return total;
    }
};

__device__ __forceinline__ float log_of(const Weights &W, uint32_t key, u64 total) {
    return (float)(W.log_weight(key) - log((double)total / W.one));
}

// Descending order of n numbers of list[], into list[MAXLIST ..] (few: each by counting the larger ones)
// or in place.  Returns where.
__device__ __forceinline__ u64 *sort_list(u64 *list, int n) {
    const int tid = threadIdx.x;
    if (n <= MAXCOUNTED) {
        // each number against the list or a share of it; its place is kept in list[MAXLIST / 2 ..]
        int size = 64;
        while (size < n) size <<= 1;
        const int shares = size < NT ? NT / size : 1, len = size / shares;
        uint32_t *place = reinterpret_cast<uint32_t *>(list + MAXLIST / 2);
        for (int e = tid; e < size; e += NT) {
            place[e] = 0;
            if (e >= n) list[e] = 0;
        }
        __syncthreads();
        for (int e = tid % size; e < size; e += NT) {
            const int first = size < NT ? tid / size * len : 0;
            const u64 x = list[e];
            uint32_t larger = 0;
            for (int i = first; i < first + len; i += 4) {
#pragma unroll
                for (int j = 0; j < 4; ++j) larger += list[i + j] > x;
            }
            if (e < n) atomicAdd(&place[e], larger);
        }
        __syncthreads();
        for (int e = tid; e < n; e += NT) list[MAXLIST + place[e]] = list[e];
        __syncthreads();
        return list + MAXLIST;
    }
    int size = 2 * MAXCOUNTED;
    while (size < n) size <<= 1;
    for (int i = n + tid; i < size; i += NT) list[i] = 0;
    __syncthreads();
    // pairs up to 64 apart stay within a wave
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int t = tid; t < size / 2; t += NT) {
                const int i = 2 * (t & -j) + (t & (j - 1));
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
    return list;
}

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// The smallest key whose bin is at least b (above every logit's: none).  A wave tries 64 keys around
// the quotient, which is off by its rounding; where that does not decide (quotients that underflow)
// it halves the range of all keys.
__device__ __forceinline__ uint32_t first_key(float b, float per) {
    constexpr uint32_t kNone = 0xff800000u;
    const uint32_t from = min(max(key_of(b / per), kLowest + 32u), kNone - 64u) - 32u;
    const u64 votes = __ballot(bin_of(logit_of(from + threadIdx.x % 64), per) >= b);
    if (votes && !(votes & 1)) return from + (uint32_t)__ffsll((long long)votes) - 1;
    uint32_t lo = kLowest, hi = kNone;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (bin_of(logit_of(mid), per) >= b)
            hi = mid;
        else
            lo = mid + 1;
    }
    return lo;
}

// A row's token; false (for every thread) where the bracket fails.
template <int DT>
__device__ __forceinline__ bool pick_row(const SampleProblem &P, const Scan &L, int r, int shift, PickLds &S) {
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const char *row = row_of<DT>(P, r);
    BlockScan scan{S};
    // everything that is read at an address known from the start: one trip to memory
    constexpr int SPT = (MAXSLICES + NT - 1) / NT;  // slices per thread
    SliceStat st[SPT];
#pragma unroll
    for (int i = 0; i < SPT; ++i) {
        st[i] = SliceStat{0, 0, 0, 0, 0};
        if (tid + i * NT < L.slices) st[i] = L.stat[(size_t)r * L.slices + tid + i * NT];
    }
    constexpr int GROUP = 2048 / NT;  // pieces of a group
    constexpr int MOST = MAXV / PIECE / GROUP / NT;  // groups per thread
    static_assert(MANY <= GROUP * MOST * NT, "pieces");
    struct alignas(GROUP * 2) Group {
        uint32_t two[GROUP / 2];
        __device__ __forceinline__ uint32_t operator[](int j) const { return two[j / 2] >> (j % 2 * 16) & 0xffffu; }
    };
    const int groups = L.pieces / GROUP;
    Group tops[MOST];
    const Group *all_tops = reinterpret_cast<const Group *>(L.tops + (size_t)r * L.pieces);
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        tops[i] = Group{};
        if (tid + i * NT < groups) tops[i] = all_tops[tid + i * NT];
    }
    const Rules rules(P, r);
    fill_table(S.table);
    // the row's largest logit
    uint32_t top = 0, finite = 0, bad = 0;
#pragma unroll
    for (int i = 0; i < SPT; ++i) {
        top = max(top, st[i].top);
        finite += st[i].finite;
        bad |= st[i].bad;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    finite = (uint32_t)wave_sum(finite);
    const u64 bads = __ballot(bad != 0);
    if (lane == 0) {
        S.top[wave] = top;
        S.finite[wave] = finite;
        S.bad[wave] = bads != 0;
    }
    if (tid == 0) {
        S.ntodo = S.nlist = 0;
        S.lo_bin = S.hi_bin = HB;
    }
    if (tid < SLICE / UNIT) S.unit[tid] = 0;
    if (tid < 8) S.reach[tid] = 0;
    __syncthreads();
    bad = top = finite = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        top = max(top, S.top[w]);
        bad |= S.bad[w];
        finite += S.finite[w];
    }
    Spread spread{0.0, top, 0xffffffffu};
    if (bad || !rules.ok || top < kLowest) {
        if (tid == 0) {
            L.spread[r] = spread;
            no_token(P, r);
        }
        return true;
    }
    const Weights W(top, rules.T, shift, S.table);
    const float per = 16.f / rules.T, first = bin_of((float)W.top, per);
    if (rules.k == 0) {
#pragma unroll
        for (int i = 0; i < SPT; ++i) {
            const int s = tid + i * NT;
            if (s >= L.slices) break;
            const double w = st[i].finite ? W.exact(st[i].top) : 0.0;
            // a slice whose largest weight is under half a step has no token to draw: it weighs nothing
            S.scale[s] = W.to_fixed(w) ? w : 0.0;
            S.below[s] = st[i].finite ? (int)fminf(first - bin_of(logit_of(st[i].top), per), (float)HB) : HB;
            S.kept[s] = 0;
        }
    } else {
        for (int s = tid; s < L.slices; s += NT) S.kept[s] = 0;
    }
    // The bracket: tokens with key >= high are surely kept, those with key >= low may be.
    const int k = min(rules.k, (int)finite);
    uint32_t low = kLowest, high = 0xffffffffu;
    u64 total = 0, goal = 0, sure_mass = 0;
    bool bounded = false;  // the bracket ends where min-p does: top-p need not cut inside it
    const double to_one = W.one / (double)(1ull << kHistShift);
    auto to_row = [&](u64 x, int s) {  // a slice's weight in the row's fixed point
        return (u64)rint((double)x * S.scale[s] * to_one);
    };
    if (rules.whole) {
        high = kLowest;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < SPT; ++i)
            if (tid + i * NT < L.slices) S.kept[tid + i * NT] = to_row(st[i].mass, tid + i * NT);
    } else if (rules.k == 0) {
        if (!(fabsf(first) < kBinLimit)) return false;
        __syncthreads();
        const u64 *hist = L.hist + (size_t)r * L.slices * HB;
        int lo_bin = HB, hi_bin = HB;
        u64 before = 0;
        if (rules.p < 1.f) {
            u64 mine = 0;
#pragma unroll
            for (int i = 0; i < SPT; ++i)
                if (tid + i * NT < L.slices) mine += to_row(st[i].mass, tid + i * NT);
            total = scan.sum(mine);
            // the row's histogram, a bin of a share of the slices per thread, and its running sum
            constexpr int AHEAD = 8;
            const int bin = tid % HB;
            double weight = 0.0;
#pragma unroll 1
            for (int s0 = tid / HB * AHEAD; s0 < L.slices; s0 += NT / HB * AHEAD) {
                u64 x[AHEAD];
                int b[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int s = min(s0 + i, L.slices - 1);
                    b[i] = s0 + i < L.slices ? bin - S.below[s] : -1;
                    x[i] = hist[(size_t)s * HB + min(max(b[i], 0), HB - 1)];
                }
#pragma unroll
                for (int i = 0; i < AHEAD; ++i)
                    if (b[i] >= 0 && b[i] < HB - 1) weight += (double)x[i] * S.scale[min(s0 + i, L.slices - 1)];
            }
            double *part = reinterpret_cast<double *>(S.list);
            part[tid] = weight;
            __syncthreads();
            for (int t = tid + HB; t < NT; t += HB) weight += part[t];
            const u64 h = tid < HB ? (u64)rint(weight * to_one) : 0;
            u64 all;
            before = scan(h, all);
            const u64 run = before + h;
            goal = (u64)ceil((double)rules.p * (double)total);
            goal = goal < 1 ? 1 : goal > total ? total : goal;
            // (slices and bins were rounded apart: a billionth is far more than that)
            if (tid < HB - 1) {
                if ((double)run >= (double)goal * (1.0 - 1e-9)) atomicMin(&S.hi_bin, (uint32_t)tid);
                if ((double)run >= (double)goal * (1.0 + 1e-9)) atomicMin(&S.lo_bin, (uint32_t)tid);
            }
            __syncthreads();
            hi_bin = (int)S.hi_bin;
            lo_bin = (int)S.lo_bin;
        }
        if (rules.m > 0.f) {  // the bins around the logit of weight min_p
            const double z = W.top + (double)rules.T * log((double)rules.m), d = fabs(z) * 1e-6 + 1e-30;
            const float above = first - bin_of((float)(z + d), per), under = first - bin_of((float)(z - d), per);
            hi_bin = min(hi_bin, (int)fmaxf(fminf(above, (float)HB), 0.f));
            if (under < (float)lo_bin) {
                lo_bin = (int)fmaxf(under, 0.f);
                bounded = true;
            }
        }
        if (lo_bin >= HB - 1) return false;
        low = first_key(first - (float)lo_bin, per);
        high = first_key(first - (float)hi_bin + 1.f, per);
        if (tid == hi_bin) S.at = before;
        // the sure weight per slice: its bins before the row's hi_bin
#pragma unroll 1
        for (int s0 = wave; s0 < L.slices; s0 += NW * 4) {
            u64 x[4][HB / 64];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < HB / 64; ++j) {
                    x[i][j] = 0;
                    if (64 * j < hi_bin) x[i][j] = hist[(size_t)min(s0 + i * NW, L.slices - 1) * HB + lane + 64 * j];
                }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = s0 + i * NW;
                if (s >= L.slices) break;
                const int most = min(hi_bin - S.below[s], HB - 1);
                u64 sum = 0;
#pragma unroll
                for (int j = 0; j < HB / 64; ++j) sum += lane + 64 * j < most ? x[i][j] : 0;
                sum = wave_sum(sum);
                if (lane == 0) S.kept[s] = to_row(sum, s);
            }
        }
        __syncthreads();
        sure_mass = S.at;
    } else if (k <= L.pieces) {
        // at least k tokens reach the k-th largest of the pieces' maxima; its upper 16 bits do
        uint32_t prefix = 0;
#pragma unroll 1
        for (int bit = 14; bit >= 0; bit -= 2) {
            uint32_t reach[3] = {0, 0, 0};
#pragma unroll
            for (int i = 0; i < MOST; ++i)
                if (i * NT < groups) {
#pragma unroll
                    for (int j = 0; j < GROUP; ++j)
#pragma unroll
                        for (int c = 0; c < 3; ++c)
                            reach[c] += (uint32_t)__popcll(__ballot(tops[i][j] >= (prefix | (uint32_t)(c + 1) << bit)));
                }
            if (lane == 0) atomicAdd(&S.reach[bit / 2], (u64)reach[0] | (u64)reach[1] << 21 | (u64)reach[2] << 42);
            __syncthreads();
            const u64 counts = S.reach[bit / 2];
            const int c = ((int)(counts & 0x1fffff) >= k) + ((int)(counts >> 21 & 0x1fffff) >= k) + ((int)(counts >> 42) >= k);
            prefix |= (uint32_t)c << bit;
        }
        prefix <<= 16;
        low = max(prefix, kLowest);
    }
    // pieces that hold tokens of the bracket, and these
    uint32_t nsure = finite;
    int nlist = 0, n = 0;  // n: kept tokens of the list
    const u64 *list = S.list;
    if (!rules.whole) {
        const uint32_t least = low >> 16;
#pragma unroll
        for (int i = 0; i < MOST; ++i)
            if (i * NT < groups) {
                uint32_t mine = 0;
#pragma unroll
                for (int j = 0; j < GROUP; ++j) mine += tops[i][j] >= least;
                const uint32_t run = (uint32_t)wave_scan(mine);
                uint32_t at = 0;
                if (lane == 63 && run) at = atomicAdd(&S.ntodo, run);
                at = (uint32_t)__builtin_amdgcn_readlane((int)at, 63) + run - mine;
#pragma unroll
                for (int j = 0; j < GROUP; ++j)
                    if (tops[i][j] >= least) {
                        if (at < MAXTODO) S.todo[at] = (uint16_t)(GROUP * (tid + i * NT) + j);
                        ++at;
                    }
            }
        __syncthreads();
        const bool every = S.ntodo > MAXTODO;
        const int ntodo = every ? L.pieces : (int)S.ntodo;
        // the bracket as logits (nothing is >= NaN; -0 equals 0)
        const float from = logit_of(low), to = logit_of(high);
        const int lane_bits = L.bits - 2, per_wave = 64 >> lane_bits, sub = lane >> lane_bits;
        const int at0 = (lane & ((1 << lane_bits) - 1)) * 4;
        constexpr int AHEAD = 4;  // loads in flight per lane, twice
        struct Batch {
            int e[AHEAD];
            f32x4 z[AHEAD];
        };
        auto fetch = [&](int q0, Batch &b) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int q = (q0 + i * NW) * per_wave + sub;
                const int piece = every ? q : (int)S.todo[min(q, MAXTODO - 1)];
                b.e[i] = q < ntodo ? (piece << L.bits) + at0 : P.V + 3;  // (load4: -inf)
                b.z[i] = load4<DT>(row, b.e[i], P.V);
            }
        };
        uint32_t sure = 0;
        auto take = [&](const Batch &b) {
            u64 votes[AHEAD][4];
            uint32_t listed = 0;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bool above = b.z[i][j] >= to;
                    sure += above;
                    votes[i][j] = __ballot(b.z[i][j] >= from && !above);
                    listed += (uint32_t)__popcll(votes[i][j]);
                }
            if (!listed) return;
            uint32_t base = 0;
            if (lane == 0) base = atomicAdd(&S.nlist, listed);
            base = (uint32_t)__builtin_amdgcn_readfirstlane((int)base);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t at = base + __popcll(votes[i][j] & ((1ull << lane) - 1));
                    if ((votes[i][j] >> lane & 1) && at < MAXLIST)
                        S.list[at] = (u64)key_of(b.z[i][j]) << 32 | (uint32_t)~(b.e[i] + j);
                    base += (uint32_t)__popcll(votes[i][j]);
                }
        };
        Batch one, two;
        fetch(wave, one);
        for (int q0 = wave; q0 * per_wave < ntodo; q0 += 2 * NW * AHEAD) {
            fetch(q0 + NW * AHEAD, two);
            take(one);
            fetch(q0 + 2 * NW * AHEAD, one);
            take(two);
        }
        nsure = (uint32_t)scan.sum(sure);
        nlist = (int)S.nlist;
        if (nlist > MAXLIST || (rules.k && nlist < k)) return false;
        if (nlist == 0 && rules.p < 1.f && !bounded) return false;
    }
    if (nlist) {
        list = sort_list(S.list, nlist);
        const int limit = rules.k ? k : nlist, each = (limit + NT - 1) / NT;
        u64 own = 0, sum;
        for (int i = tid * each; i < min((tid + 1) * each, limit); ++i) own += W.fixed((uint32_t)(list[i] >> 32));
        u64 m = scan(own, sum);
        n = limit;
        if (rules.p < 1.f) {
            if (rules.k) {
                goal = (u64)ceil((double)rules.p * (double)sum);
                goal = goal < 1 ? 1 : goal > sum ? sum : goal;
            }
            if (sure_mass + sum >= goal) {
                if (sure_mass >= goal) return false;
                m += sure_mass;
                if (m < goal && m + own >= goal)
                    for (int i = tid * each; i < min((tid + 1) * each, limit); ++i) {
                        m += W.fixed((uint32_t)(list[i] >> 32));
                        if (m >= goal) {
                            S.pick = i + 1;
                            break;
                        }
                    }
                __syncthreads();
                n = (int)S.pick;
            } else if (!bounded) {
                return false;
            }
        }
        if (rules.m > 0.f) {
            u64 c = 0;
            for (int i = tid * each; i < min((tid + 1) * each, n); ++i)
                c += W.exact((uint32_t)(list[i] >> 32)) >= (double)rules.m;
            n = (int)scan.sum(c);
        }
        for (int i = tid; i < n; i += NT) {
            const u64 x = list[i];
            atomicAdd(&S.kept[(uint32_t)~x / (uint32_t)L.slice], W.fixed((uint32_t)(x >> 32)));
        }
    }
    __syncthreads();
    const Cut cut = n ? Cut{(uint32_t)(list[n - 1] >> 32), (uint32_t)~list[n - 1]} : Cut{0xffffffffu, 0u};
    // the slice where the running weight exceeds the target
    u64 own = 0, all;
#pragma unroll
    for (int i = 0; i < SPT; ++i)
        if (tid * SPT + i < L.slices) own += S.kept[tid * SPT + i];
    u64 m = scan(own, all);
    u64 target = (u64)((double)rules.u * (double)all);  // exceeds: > floor
    if (m <= target && m + own > target) {
#pragma unroll
        for (int i = 0; i < SPT; ++i) {
            const u64 x = S.kept[tid * SPT + i];
            if (m <= target && m + x > target) {
                S.pick = tid * SPT + i;
                S.at = m;
            }
            m += x;
        }
    }
    __syncthreads();
    // the unit in it, then the token
    const int e0 = (int)S.pick * L.slice, units = L.slice / UNIT;
    target -= S.at;
    auto weight = [&](uint32_t key, int e) -> u64 {  // of a kept token
        if (key < low || !(key >= high || cut.keeps(key, e))) return 0;
        return W.fixed(key);
    };
    if (high == 0xffffffffu) {  // every kept token is in the list
        for (int i = tid; i < n; i += NT) {
            const u64 x = list[i];
            const int e = (int)(uint32_t)~x - e0;
            if (e < 0 || e >= L.slice) continue;
            atomicAdd(&S.unit[e / UNIT], W.fixed((uint32_t)(x >> 32)));
        }
    } else {
        f32x4 z = load4<DT>(row, e0 + wave * UNIT + lane * 4, P.V);
#pragma unroll 1
        for (int i = wave; i < units; i += NW) {
            const f32x4 next = load4<DT>(row, e0 + min(i + NW, units - 1) * UNIT + lane * 4, P.V);
            const int e = e0 + i * UNIT + lane * 4;
            u64 w = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) w += weight(key_of(z[j]), e + j);
            w = wave_sum(w);
            if (lane == 0) S.unit[i] = w;
            z = next;
        }
    }
    __syncthreads();
    if (wave == 0) {
        const u64 w = lane < units ? S.unit[lane] : 0, run = wave_scan(w), whole = last_lane(run);
        // (a slice that was picked weighs something, but it was rounded apart from its tokens: the target may
        // lie above them all)
        if (target >= whole) target = whole - 1;
        const int u = __ffsll((long long)__ballot(run > target)) - 1;
        target -= u ? (u64)__shfl((long long)run, u - 1) : 0;
        const int e = e0 + u * UNIT + lane * 4;
        const f32x4 x = load4<DT>(row, e, P.V);
        u64 v[4], mine = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = weight(key_of(x[j]), e + j);
            mine += v[j];
        }
        u64 at = wave_scan(mine);
        const u64 here = __ballot(at > target);
        int token = -1;
        float logit = 0.f;
        if (lane == __ffsll((long long)here) - 1) {
            at -= mine;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                at += v[j];
                if (token < 0 && at > target) {
                    token = e + j;
                    logit = x[j];
                }
            }
        }
        if (token >= 0) {
            P.tokens[r] = token;
            if (P.logprob) P.logprob[r] = log_of(W, key_of(logit), all);
            if (P.kept) P.kept[r] = (int32_t)(nsure + n);
        }
    }
    const double scale = W.one / (double)all;
    if (tid == 0) L.spread[r] = Spread{scale, top, high};
    if (!P.probs) return true;
    float *probs = P.probs + (size_t)r * P.V;
    for (int i = tid; i < n; i += NT) {
        const u64 x = list[i];
        probs[(uint32_t)~x] = (float)(W.exact((uint32_t)(x >> 32)) * scale);
    }
    return true;
}

template <int DT>
__global__ __launch_bounds__(NT) void pick_kernel(SampleProblem P, Scan L, int shift, int idbits) {
    __shared__ PickLds S;
    const int r = blockIdx.x;
    if (pick_row<DT>(P, L, r, shift, S)) return;
    __syncthreads();
    if (threadIdx.x == 0) L.spread[r] = Spread{0.0, 0u, 0xffffffffu};
    search_row<DT>(P, r, Rules(P, r), shift, idbits, S.search, S.table);
}

// The probabilities of what is surely kept, a slice of SLICE tokens per workgroup (rows without rules:
// of every token).
template <int DT>
__global__ __launch_bounds__(ST) void spread_kernel(SampleProblem P, Scan L) {
    __shared__ double table[POWERS];
    const int per = (P.V + SLICE - 1) / SLICE, r = blockIdx.x / per, s = blockIdx.x % per, tid = threadIdx.x;
    const Spread spread = L.spread[r];
    const Rules rules(P, r);
    if (!rules.whole && (spread.least == 0xffffffffu || spread.least > spread.top)) return;
    const char *row = row_of<DT>(P, r);
    f32x4 z[SLICE / ST / 4];
#pragma unroll
    for (int i = 0; i < SLICE / ST / 4; ++i) z[i] = load4<DT>(row, s * SLICE + (i * ST + tid) * 4, P.V);
    fill_table(table);
    __syncthreads();
    const Weights W(spread.top, rules.T, 0, table);
    const float least = logit_of(spread.least);  // (none: a NaN)
    float *probs = P.probs + (size_t)r * P.V;
#pragma unroll
    for (int i = 0; i < SLICE / ST / 4; ++i) {
        const int e = s * SLICE + (i * ST + tid) * 4;
        f32x4 q;
        bool in[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            in[j] = z[i][j] >= least;
            q[j] = in[j] ? (float)(W.of(z[i][j]) * spread.scale) : 0.f;
        }
        if (rules.whole && e + 3 < P.V) {
            __builtin_nontemporal_store(q, reinterpret_cast<f32x4_any *>(probs + e));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e + j < P.V && (rules.whole || in[j])) probs[e + j] = q[j];
        }
    }
}

int bits_of(uint32_t x) {
    int b = 0;
    while (b < 32 && x >> b) ++b;
    return b;
}

// Slices of 8,192 logits, or of 2,048 where the rows are too few to fill the chip with those.  8,192 and
// 2,048, us, no rule / min-p / top-p: 1 row of 128,256 21 and 12 / 26 and 23 / 34 and 32; 24 rows 23 and 16 /
// 27 and 26 / 39 and 39; 64 rows 29 and 25 / 31 and 34 / 42 and 47; 128 rows of 32,003 23 and 18 / 27 and 25 /
// 35 and 33.
int most_rows_of_short_slices(int V) { return 2 * kCus / ((V + SLICE - 1) / SLICE); }
static_assert(MAXV <= 2048 * MAXSLICES, "short slices of the longest row");

Scan layout(const SampleProblem &p, char *ws, size_t &bytes) {
    Scan L{};
    L.slice = p.R <= most_rows_of_short_slices(p.V) ? 2048 : SLICE;
    L.slices = (p.V + L.slice - 1) / L.slice;
    L.bits = p.V <= 4 * MANY ? 2 : p.V <= 16 * MANY ? 4 : 6;
    L.pieces = (p.V + (8 << L.bits) - 1) / (8 << L.bits) * 8;  // (a slice is a multiple of that)
    size_t off = 0;
    auto take = [&](size_t n) {
        char *at = ws ? ws + off : nullptr;
        off += (n + 255) / 256 * 256;
        return at;
    };
    const size_t R = (size_t)p.R;
    L.stat = (SliceStat *)take(R * L.slices * sizeof(SliceStat));
    L.tops = (uint16_t *)take(R * L.pieces * 2);
    L.hist = (u64 *)take(R * L.slices * HB * sizeof(u64));
    L.spread = (Spread *)take(R * sizeof(Spread));
    bytes = off ? off : 256;
    return L;
}

template <int DT>
hipError_t launch(const SampleProblem &p, char *ws, hipStream_t st) {
    const int idbits = bits_of((uint32_t)(p.V - 1));
    // V weights of at most 2^shift stay below 2^62; a weight is a whole number in a double
    const int shift = idbits > 12 ? 62 - idbits : 50;
    if (p.V > MAXV || p.V < 4) {
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
        const dim3 spread((unsigned)(p.R * ((p.V + SLICE - 1) / SLICE)));
        hipLaunchKernelGGL((spread_kernel<DT>), spread, dim3(ST), 0, st, p, L);
    }
    return hipGetLastError();
}

}  // namespace

size_t sample_workspace(const SampleProblem &p) {
    if (p.V > MAXV || p.V < 4) return 256;
    // Short slices need more per row, so that fewer rows can need more: what any number of rows up to
    // this one needs.
    SampleProblem fewer = p;
    fewer.R = min(p.R, most_rows_of_short_slices(p.V));
    size_t bytes, most;
    layout(p, nullptr, bytes);
    layout(fewer, nullptr, most);
    return max(bytes, most);
}

hipError_t launch_sample(const SampleProblem &p, void *ws, hipStream_t st) {
    return p.dtype == kBF16 ? launch<kBF16>(p, (char *)ws, st) : launch<kF32>(p, (char *)ws, st);
}

}  // namespace dcd
