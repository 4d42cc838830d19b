// A token for each row of logits (include/fireq_sample.h).
//
// min-p, top-k and top-p all keep a first run of the tokens in one order (larger logit first, lower index first among equals), so
// what is kept is comp >= tau for one number: comp = (ordered bits of the logit, inverted index).  Two kernels find it without sorting:
//     parts   a row is cut into parts of up to 8192 logits.  Each finds its largest logit, takes e = exp((x - largest) / T) as a whole number of
//             2^-36 (sums of whole numbers do not depend on their order; a token below 2^-37 of its part's best has no mass) and, where the row is
//             filtered at all, counts numbers and masses in FQS_BINS equal steps of x / T.  The steps lie on one grid for all parts.
//     row     one workgroup per row adds the parts' bins and finds the bin in which the kept run ends.  Only that bin's tokens are looked at
//             one by one: a radix selection by number or by mass over comp, in LDS (or over the row again, where they are too many).  The token: the
//             part, and in it the index, at which the kept mass in index order passes u times its sum.
#include "fq_common.h"
#include "fq_kernels.h"

namespace {

typedef unsigned long long fqs_u64;

constexpr int FQS_BINS = 512, FQS_LIST = 4096, FQS_T1 = 256, FQS_T2 = 512, FQS_MOST_PARTS = 256;
constexpr float FQS_UNIT = 0x1p36f;                       // masses in 2^-36 of the largest
constexpr float FQS_SPAN = 26.0f;                         // nats that the bins cover: e^-26 is below 2^-37
constexpr fqs_u64 FQS_MASS = (1ull << 50) - 1;            // a part's bin: number of tokens << 50 | mass (8192 * 2^36 at most)

struct fqs_plan { int per, parts; };                      // chunks of 8 logits of a part; parts of a row
__host__ __device__ inline fqs_plan fqs_choose(int B, int V) {
    const int chunks = (V + 7 + 7) / 8;                   // (a row may begin inside a chunk)
    int per = FQS_T1;                                     // at least one chunk a thread, at most four
    while (per < 4 * FQS_T1 && (long long)B * ((chunks + per - 1) / per) > 1024) per += FQS_T1;
    if ((chunks + per - 1) / per > FQS_MOST_PARTS) per = 4 * FQS_T1;
    return {per, (chunks + per - 1) / per};
}

struct fqs_work {
    float* top;                                           // [B][parts] largest logit of a part; NaN: one that is NaN or +infinity
    fqs_u64* total;                                       // [B][parts] mass of all its tokens
    fqs_u64* bins;                                        // [B][parts][FQS_BINS]
    fqs_plan plan;
};

// A row's parameters as the kernels take them.
struct fqs_row {
    float c, steps;                                       // log2 e / T, bins per unit of x
    double T;
    int k;                                                // 0: off
    float p, low;                                         // 1: off, 0: off
    bool bad, filtered;
};
__device__ __forceinline__ fqs_row fqs_parameters(const fq_sample_args& a, int b) {
    fqs_row r;
    const float T = a.temperature ? a.temperature[b] : 1.0f, u = a.u[b];
    r.k = a.top_k ? a.top_k[b] : 0;
    r.p = a.top_p ? a.top_p[b] : 1.0f;
    r.low = a.min_p ? a.min_p[b] : 0.0f;
    r.bad = !(T >= 0.0f && T <= 3.402823466e38f) || u != u || r.p != r.p || r.low != r.low;
    if (r.k < 0 || r.k >= a.V) r.k = 0;
    if (T == 0.0f) r.k = 1;
    const float t = T == 0.0f ? 1.0f : fminf(fmaxf(T, 0x1p-100f), 0x1p100f);   // (beyond, one token or all alike)
    r.T = t;
    r.c = 1.44269504088896340736f / t;
    r.steps = (float)FQS_BINS / FQS_SPAN / t;
    r.low = fminf(r.low, 1.0f);
    r.filtered = r.k > 0 || r.p < 1.0f || r.low > 0.0f;
    return r;
}
// The grid line below x; x in bins from a line `top` (not below x's): top - line, dropped from FQS_BINS on.
__device__ __forceinline__ float fqs_line(float x, float steps) { return floorf(fminf(x * steps, 0x1p100f)); }
__device__ __forceinline__ fqs_u64 fqs_mass(float x, float top, float c) {
    return (fqs_u64)(unsigned long long)rintf(__builtin_amdgcn_exp2f((x - top) * c) * FQS_UNIT);
}

// Bits that order as the numbers do (-0 as 0), 16 of bf16 and 32 of FP32, above the inverted index.
template <bool WIDE>
__device__ __forceinline__ fqs_u64 fqs_key(float x) {
    const unsigned b = __float_as_uint(x + 0.0f), o = b & 0x80000000u ? ~b : b | 0x80000000u;
    return WIDE ? o : o >> 16;
}
template <bool WIDE>
__device__ __forceinline__ fqs_u64 fqs_comp(float x, int i) { return fqs_key<WIDE>(x) << 20 | (fqs_u64)(0xFFFFF - i); }

// Eight logits of chunk c (tokens 8 c - skew ..): -infinity outside the row.
template <bool WIDE>
__device__ __forceinline__ void fqs_load(const fq_sample_args& a, int b, int skew, int c, float (&x)[8]) {
    const int i0 = 8 * c - skew;
    const char* row = static_cast<const char*>(a.logits) + (long long)b * a.ld * (WIDE ? 4 : 2);
    if (i0 >= 0 && i0 + 8 <= a.V) {
        if constexpr (WIDE) {
            const fq_v4f* p = reinterpret_cast<const fq_v4f*>(row + (long long)i0 * 4);
            const fq_v4f lo = p[0], hi = p[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = lo[e]; x[4 + e] = hi[e]; }
        } else {
            const fq_v4i w = *reinterpret_cast<const fq_v4i*>(row + (long long)i0 * 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[2 * e] = fq_bf16_lo(w[e]); x[2 * e + 1] = fq_bf16_hi(w[e]); }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = i0 + e;
            x[e] = -__builtin_inff();
            if (i >= 0 && i < a.V) {
                if constexpr (WIDE) x[e] = reinterpret_cast<const float*>(row)[i];
                else x[e] = __uint_as_float((unsigned)reinterpret_cast<const uint16_t*>(row)[i] << 16);
            }
        }
    }
}
// Tokens of chunk 0 that lie before the row: chunks begin at multiples of 16 bytes.
template <bool WIDE>
__device__ __forceinline__ int fqs_skew(const fq_sample_args& a, int b) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.logits) + (uintptr_t)((long long)b * a.ld * (WIDE ? 4 : 2));
    return (int)((p & 15) / (WIDE ? 4 : 2));
}

__device__ __forceinline__ float fqs_wave_max(float v) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = fmaxf(v, __shfl_xor(v, d, 64));
    return v;
}
__device__ __forceinline__ fqs_u64 fqs_wave_sum(fqs_u64 v) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
    return v;
}

template <bool WIDE>
__global__ __launch_bounds__(FQS_T1) void fqs_parts_kernel(fq_sample_args a, fqs_work w) {
    __shared__ fqs_u64 bins[FQS_BINS];
    __shared__ float wave_top[FQS_T1 / 64];
    __shared__ fqs_u64 wave_sum[FQS_T1 / 64];
    __shared__ int wave_bad[FQS_T1 / 64];
    const int part = blockIdx.x, b = blockIdx.y, t = threadIdx.x, wave = t >> 6;
    const fqs_row r = fqs_parameters(a, b);
    const size_t at = (size_t)b * w.plan.parts + part;
    if (r.bad) {
        if (t == 0) w.top[at] = __builtin_nanf("");
        return;
    }
    const int skew = fqs_skew<WIDE>(a, b), mine = w.plan.per / FQS_T1;
    float x[4][8], top = -__builtin_inff();
    int bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i < mine) {
            fqs_load<WIDE>(a, b, skew, part * w.plan.per + i * FQS_T1 + t, x[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = -__builtin_inff();
        }
    }
    if (r.filtered)
        for (int i = t; i < FQS_BINS; i += FQS_T1) bins[i] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bad |= !(x[i][e] < __builtin_inff()) ? 1 : 0;
            top = fmaxf(top, x[i][e]);
        }
    top = fqs_wave_max(top);
    bad = __any(bad) ? 1 : 0;
    if ((t & 63) == 0) {
        wave_top[wave] = top;
        wave_bad[wave] = bad;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FQS_T1 / 64; ++i) {
        top = fmaxf(top, wave_top[i]);
        bad |= wave_bad[i];
    }
    const bool none = bad || !(top > -__builtin_inff());  // nothing to count
    fqs_u64 sum = 0;
    if (!none) {
        const float line = fqs_line(top, r.steps);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const fqs_u64 m = fqs_mass(x[i][e], top, r.c);
                sum += m;
                if (r.filtered) {
                    const float d = line - fqs_line(x[i][e], r.steps);
                    if (d < (float)FQS_BINS) atomicAdd(&bins[(int)d], (1ull << 50) + m);
                }
            }
    }
    sum = fqs_wave_sum(sum);
    if ((t & 63) == 0) wave_sum[wave] = sum;
    __syncthreads();
    if (t == 0) {
        for (int i = 1; i < FQS_T1 / 64; ++i) sum += wave_sum[i];
        w.top[at] = bad ? __builtin_nanf("") : top;
        w.total[at] = sum;
    }
    if (r.filtered)
        for (int i = t; i < FQS_BINS; i += FQS_T1) w.bins[at * FQS_BINS + i] = bins[i];
}

// Inclusive sums over the workgroup's threads, in their order; `all`: the sum.  (scratch: one number a wave)
__device__ __forceinline__ fqs_u64 fqs_scan(fqs_u64 v, fqs_u64* scratch, fqs_u64& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const fqs_u64 o = __shfl_up(v, d, 64);
        if (lane >= d) v += o;
    }
    __syncthreads();
    if (lane == 63) scratch[wave] = v;
    __syncthreads();
    fqs_u64 before = 0;
    all = 0;
#pragma unroll
    for (int i = 0; i < FQS_T2 / 64; ++i) {
        if (i < wave) before += scratch[i];
        all += scratch[i];
    }
    return v + before;
}

struct fqs_shared {
    fqs_u64 scan[FQS_T2 / 64], reach[FQS_T2 / 64];
    fqs_u64 part_mass[FQS_MOST_PARTS];                    // kept mass of each part
    float top[FQS_MOST_PARTS];
    float factor[FQS_MOST_PARTS];                         // of a part's masses
    int shift[FQS_MOST_PARTS];                            // of its bins
    fqs_u64 mass[FQS_BINS];                               // inclusive sums
    fqs_u64 digit[2][256];
    fqs_u64 list[FQS_LIST];                               // comps of one bin
    int some[FQS_MOST_PARTS];                             // parts that have tokens in it
    fqs_u64 found_before, found_own;
    int n, parts, found;
};

template <bool WIDE>
struct fqs_finder {
    const fq_sample_args& a;
    const fqs_work& w;
    const fqs_row& r;
    fqs_shared& sh;
    int b, skew, t;
    float top, line;

    // the first index whose value in `cum` (inclusive, of n) reaches `want`, in sh.found (n: none), and what lies before it
    __device__ __forceinline__ void first_reaching(fqs_u64 own, fqs_u64 cum, int n, fqs_u64 want) {
        __syncthreads();
        if (t == 0) { sh.found = n; sh.found_before = 0; }
        __syncthreads();
        if (t < n && cum >= want && cum - own < want) {
            sh.found = t;
            sh.found_before = cum - own;
        }
        __syncthreads();
    }
    template <class F>
    __device__ __forceinline__ void each_logit(F f) {     // of the whole row
        for (int c = t; c < (a.V + skew + 7) / 8; c += FQS_T2) {
            float x[8];
            fqs_load<WIDE>(a, b, skew, c, x);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (x[e] > -__builtin_inff()) f(x[e], 8 * c - skew + e);
        }
    }
    __device__ __forceinline__ bool in_bin(float x, int bin) { return line - fqs_line(x, r.steps) == (float)bin; }
    __device__ __forceinline__ float value_of(fqs_u64 comp) {
        const unsigned k = (unsigned)(comp >> 20), o = WIDE ? k : k << 16;
        return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : WIDE ? ~o : ~o & 0xFFFF0000u);
    }
    // a part's numbers in the row's bin i (0 before its first)
    __device__ __forceinline__ fqs_u64 bin_of(int p, int i) {
        const int q = i - sh.shift[p];
        const fqs_u64 v = w.bins[((size_t)b * w.plan.parts + p) * FQS_BINS + (q < 0 ? 0 : q)];
        return q < 0 ? 0ull : v;
    }
    // the tokens of a bin into the list; only those parts are read that have some, four chunks of a thread at a time
    __device__ __forceinline__ void gather(int bin) {
        __syncthreads();
        if (t == 0) sh.n = sh.parts = 0;
        __syncthreads();
        if (t < w.plan.parts && bin_of(t, bin) != 0) sh.some[atomicAdd(&sh.parts, 1)] = t;
        __syncthreads();
        const int chunks = (a.V + skew + 7) / 8, all = sh.parts * w.plan.per;
        for (int i0 = t; i0 < all; i0 += 4 * FQS_T2) {
            float x[4][8];
            int c[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * FQS_T2, p = i < all ? i / w.plan.per : 0;
                c[u] = i < all ? sh.some[p] * w.plan.per + (i - p * w.plan.per) : chunks;
                if (c[u] < chunks) fqs_load<WIDE>(a, b, skew, c[u], x[u]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c[u] < chunks)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (x[u][e] > -__builtin_inff() && in_bin(x[u][e], bin)) {
                            const int at = atomicAdd(&sh.n, 1);
                            if (at < FQS_LIST) sh.list[at] = fqs_comp<WIDE>(x[u][e], 8 * c[u] - skew + e);
                        }
        }
        __syncthreads();
    }
    template <class F>
    __device__ __forceinline__ void each_in_bin(int bin, F f) {
        if (sh.n <= FQS_LIST)
            for (int i = t; i < sh.n; i += FQS_T2) f(sh.list[i]);
        else
            each_logit([&](float x, int i) __attribute__((always_inline)) { if (in_bin(x, bin)) f(fqs_comp<WIDE>(x, i)); });
    }
    __device__ __forceinline__ fqs_u64 mass_of(fqs_u64 comp) { return fqs_mass(value_of(comp), top, r.c); }
    // The least comp of the bin's best tokens: of the first `want`, or (BY_MASS) of the first whose mass reaches `want`.  Eight bits at a time from the
    // highest in which the bin's comps differ: sums for each digit, then the first wave finds the digit in which the run ends, while the others clear
    // the sums of the next eight.
    template <bool BY_MASS>
    __device__ __forceinline__ fqs_u64 select(int bin, fqs_u64 want) {
        const int lane = t & 63, wave = t >> 6;
        fqs_u64 lo = ~0ull, hi = 0ull;
        each_in_bin(bin, [&](fqs_u64 c) __attribute__((always_inline)) { lo = c < lo ? c : lo; hi = c > hi ? c : hi; });
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const fqs_u64 l = __shfl_xor(lo, d, 64), h = __shfl_xor(hi, d, 64);
            lo = l < lo ? l : lo;
            hi = h > hi ? h : hi;
        }
        __syncthreads();
        if (lane == 0) { sh.scan[wave] = lo; sh.reach[wave] = hi; }
        for (int i = t; i < 256; i += FQS_T2) sh.digit[0][i] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < FQS_T2 / 64; ++i) {
            lo = sh.scan[i] < lo ? sh.scan[i] : lo;
            hi = sh.reach[i] > hi ? sh.reach[i] : hi;
        }
        if (lo >= hi) return lo;                          // one token
        int above = 64 - __builtin_clzll(lo ^ hi);        // bits below are still open
        fqs_u64 prefix = hi >> above << above;            // (comps have 52 bits)
        const bool listed = sh.n <= FQS_LIST;             // (their number then fits beside their mass)
        for (int buf = 0; above > 0; buf ^= 1) {
            const int width = above < 8 ? above : 8, shift = above - width;
            each_in_bin(bin, [&](fqs_u64 c) __attribute__((always_inline)) {
                if ((c ^ prefix) >> above == 0) atomicAdd(&sh.digit[buf][255 - (int)(c >> shift & ((1u << width) - 1u))], BY_MASS ? (listed ? 1ull << 50 : 0ull) + mass_of(c) : 1ull);
            });
            __syncthreads();
            if (wave == 0) {
                fqs_u64 v[4], own = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = sh.digit[buf][4 * lane + i];
                    own += BY_MASS && listed ? v[i] & FQS_MASS : v[i];
                }
                fqs_u64 cum = own;
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const fqs_u64 o = __shfl_up(cum, d, 64);
                    if (lane >= d) cum += o;
                }
                const unsigned long long reached = __ballot(cum >= want);
                if (reached == 0ull) {
                    if (lane == 0) sh.found = 256;
                } else if (lane == __ffsll((long long)reached) - 1) {
                    fqs_u64 before = cum - own;
                    int i = 0;
                    for (; i < 3; ++i) {
                        const fqs_u64 x = BY_MASS && listed ? v[i] & FQS_MASS : v[i];
                        if (before + x >= want) break;
                        before += x;
                    }
                    sh.found = 4 * lane + i;
                    sh.found_before = before;
                    sh.found_own = i == 0 ? v[0] : i == 1 ? v[1] : i == 2 ? v[2] : v[3];
                }
            } else {
                for (int i = t - 64; i < 256; i += FQS_T2 - 64) sh.digit[buf ^ 1][i] = 0;
            }
            __syncthreads();
            const int found = sh.found;
            if (found >= 256) return prefix;              // (all of them do not reach it: rounding)
            want -= sh.found_before;
            prefix |= (fqs_u64)(255 - found) << shift;
            // one token, or as many as are wanted: whatever its lower bits
            if (BY_MASS ? listed && sh.found_own >> 50 == 1ull : sh.found_own == want) return prefix;
            above = shift;
        }
        return prefix;
    }
    // mass of the bin's tokens from `least` on
    __device__ __forceinline__ fqs_u64 kept_in_bin(int bin, fqs_u64 least) {
        fqs_u64 m = 0, all;
        each_in_bin(bin, [&](fqs_u64 c) __attribute__((always_inline)) { if (c >= least) m += mass_of(c); });
        fqs_scan(m, sh.scan, all);
        return all;
    }
};

template <bool WIDE>
__global__ __launch_bounds__(FQS_T2) void fqs_row_kernel(fq_sample_args a, fqs_work w) {
    __shared__ fqs_shared sh;
    const int b = blockIdx.x, t = threadIdx.x, parts = w.plan.parts;
    const fqs_row r = fqs_parameters(a, b);
    // largest logit, then each part's factor and shift
    float top = -__builtin_inff();
    int bad = r.bad ? 1 : 0;
    if (t < parts) {
        const float x = w.top[(size_t)b * parts + t];
        sh.top[t] = x;
        bad |= x != x ? 1 : 0;
        top = x;
    }
    top = fqs_wave_max(top);
    if ((t & 63) == 0) sh.scan[t >> 6] = __float_as_uint(top);
    bad = __syncthreads_or(bad);
#pragma unroll
    for (int i = 0; i < FQS_T2 / 64; ++i) top = fmaxf(top, __uint_as_float((unsigned)sh.scan[i]));
    __syncthreads();
    if (bad || !(top > -__builtin_inff())) {
        if (t == 0) {
            a.token[b] = -1;
            if (a.logprob) a.logprob[b] = __builtin_nanf("");
        }
        return;
    }
    const float line = fqs_line(top, r.steps);
    fqs_u64 part_total = 0;
    if (t < parts) {
        const float x = sh.top[t], f = x > -__builtin_inff() ? __builtin_amdgcn_exp2f((x - top) * r.c) : 0.0f;
        const float d = x > -__builtin_inff() ? line - fqs_line(x, r.steps) : (float)FQS_BINS;
        sh.factor[t] = f;
        sh.shift[t] = d < (float)FQS_BINS ? (int)d : FQS_BINS;
        part_total = (fqs_u64)rint((double)w.total[(size_t)b * parts + t] * (double)f);
    }
    fqs_u64 total;
    fqs_scan(part_total, sh.scan, total);                 // (its barriers also publish factors and shifts)
    const int skew = fqs_skew<WIDE>(a, b);
    fqs_finder<WIDE> find = {a, w, r, sh, b, skew, t, top, line};
    fqs_u64 least = 0, kept;                              // kept tokens: comp >= least
    if (t < parts) sh.part_mass[t] = part_total;
    if (r.filtered) {
        unsigned count = 0;
        fqs_u64 mass = 0;
        static_assert(FQS_BINS == FQS_T2, "a bin a thread");
        for (int p0 = 0; p0 < parts; p0 += 8) {           // (eight requested at a time)
            fqs_u64 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = p0 + u < parts ? find.bin_of(p0 + u, t) : 0ull;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                count += (unsigned)(v[u] >> 50);
                mass += (fqs_u64)rint((double)(v[u] & FQS_MASS) * (double)sh.factor[p0 + u < parts ? p0 + u : 0]);
            }
        }
        fqs_u64 all;
        const fqs_u64 counts = fqs_scan(count, sh.scan, all), masses = fqs_scan(mass, sh.scan, all);
        sh.mass[t] = masses;
        int bin = FQS_BINS;                               // the bin in which the kept run ends (FQS_BINS: behind all)
        fqs_u64 run = all;                                // its mass
        // min-p: from a value on
        if (r.low > 0.0f) {
            const double from = (double)top + r.T * log((double)r.low);
            float x = (float)from;
            if ((double)x < from) x = x < 0.0f ? __uint_as_float(__float_as_uint(x) - 1u) : x == 0.0f ? 0x1p-149f : __uint_as_float(__float_as_uint(x) + 1u);
            const unsigned bits = __float_as_uint(x + 0.0f), o = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
            least = (WIDE ? (fqs_u64)o : ((fqs_u64)o + 0xFFFF) >> 16) << 20;
            const float d = line - fqs_line(x, r.steps);
            bin = d < (float)FQS_BINS ? (int)d : FQS_BINS;
        }
        bool ranked = false;
        fqs_u64 rank_left = 0;
        if (r.k > 0) {
            find.first_reaching(count, counts, FQS_BINS, (fqs_u64)r.k);
            if (sh.found <= bin && sh.found < FQS_BINS) {
                bin = sh.found;
                ranked = true;
                rank_left = (fqs_u64)r.k - sh.found_before;
            }
        }
        if (bin < FQS_BINS) {
            find.gather(bin);
            if (ranked && sh.n > 0) {
                const fqs_u64 x = find.template select<false>(bin, rank_left);
                least = x > least ? x : least;
            }
            run = (bin > 0 ? sh.mass[bin - 1] : 0) + find.kept_in_bin(bin, least);
        }
        if (r.p < 1.0f) {
            fqs_u64 want = (fqs_u64)ceil((double)run * (double)r.p);
            want = want < 1 ? 1 : want;
            if (r.p <= 0.0f) want = 1;
            const fqs_u64 before_bin = bin < FQS_BINS ? (bin > 0 ? sh.mass[bin - 1] : 0) : all;
            if (bin < FQS_BINS && want > before_bin) {
                if (sh.n > 0) {
                    const fqs_u64 x = find.template select<true>(bin, want - before_bin);
                    least = x > least ? x : least;
                }
            } else {
                find.first_reaching(mass, masses, FQS_BINS, want);
                const int at = sh.found;
                const fqs_u64 left = want - sh.found_before;
                if (at < FQS_BINS) {
                    bin = at;
                    find.gather(bin);
                    const fqs_u64 x = find.template select<true>(bin, left);
                    least = x > least ? x : least;
                }
            }
        }
        // kept mass of each part: its bins before that one, and the kept of that one
        __syncthreads();
        const int lane = t & 63;
        for (int p = t >> 6; p < parts; p += FQS_T2 / 64) {
            fqs_u64 v[FQS_BINS / 64], m = 0;
#pragma unroll
            for (int i = 0; i < FQS_BINS / 64; ++i) v[i] = lane + 64 * i < bin ? find.bin_of(p, lane + 64 * i) : 0ull;
#pragma unroll
            for (int i = 0; i < FQS_BINS / 64; ++i) m += (fqs_u64)rint((double)(v[i] & FQS_MASS) * (double)sh.factor[p]);
            m = fqs_wave_sum(m);
            if (lane == 0) sh.part_mass[p] = m;
        }
        __syncthreads();
        if (bin < FQS_BINS)
            find.each_in_bin(bin, [&](fqs_u64 c) __attribute__((always_inline)) {
                if (c >= least) atomicAdd(&sh.part_mass[((int)(0xFFFFF - (c & 0xFFFFF)) + skew) / 8 / w.plan.per], find.mass_of(c));
            });
    }
    __syncthreads();
    // the part, then the token, at which the mass in index order passes u times the whole
    const fqs_u64 own = t < parts ? sh.part_mass[t] : 0, cum = fqs_scan(own, sh.scan, kept);
    const float u = fminf(fmaxf(a.u[b], 0.0f), 0x1.fffffep-1f);
    const fqs_u64 target = (fqs_u64)((double)u * (double)kept);
    find.first_reaching(own, cum, parts, target + 1);
    const int part = sh.found < parts ? sh.found : parts - 1;
    const double left = (double)(target - sh.found_before);   // in the row's unit
    const double scale = 1.0 / (double)sh.factor[part];
    const float part_top = sh.top[part];
    constexpr int MINE = 4 * FQS_T1 / FQS_T2;             // chunks of a thread, one behind the other
    static_assert(MINE * FQS_T2 == 4 * FQS_T1, "a part's chunks");
    float x[MINE][8];
    fqs_u64 m = 0;
    const int c0 = part * w.plan.per + MINE * t;
#pragma unroll
    for (int u = 0; u < MINE; ++u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] = -__builtin_inff();
        if (MINE * t + u < w.plan.per) fqs_load<WIDE>(a, b, skew, c0 + u, x[u]);
    }
#pragma unroll
    for (int u = 0; u < MINE; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (x[u][e] > -__builtin_inff() && fqs_comp<WIDE>(x[u][e], 8 * (c0 + u) - skew + e) >= least) m += fqs_mass(x[u][e], part_top, r.c);
    fqs_u64 in_part, run = fqs_scan(m, sh.scan, in_part) - m;
    // (the part's own sum and the bins' may differ by rounding: the last token with a mass then)
    double want = left * scale;
    if (!(want < (double)in_part)) want = in_part > 0 ? (double)(in_part - 1) : 0.0;
    if ((double)run <= want && want < (double)(run + m)) {
        int token = -1;
        float value = 0.f;
#pragma unroll
        for (int u = 0; u < MINE; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = 8 * (c0 + u) - skew + e;
                if (token >= 0 || !(x[u][e] > -__builtin_inff()) || fqs_comp<WIDE>(x[u][e], i) < least) continue;
                run += fqs_mass(x[u][e], part_top, r.c);
                if ((double)run > want) {
                    token = i;
                    value = x[u][e];
                }
            }
        a.token[b] = token;
        if (a.logprob) a.logprob[b] = (float)(((double)value - (double)top) / r.T - log((double)total * 0x1p-36));
    }
}

}  // namespace

size_t fq_sample_scratch_bytes(int B, int V) {
    const size_t rows = (size_t)B * fqs_choose(B, V).parts;
    return rows * (8 * FQS_BINS + 8) + (rows * 4 + 15) / 16 * 16;
}

void fq_launch_sample(const fq_sample_args& a, void* scratch, hipStream_t stream) {
    fqs_work w;
    w.plan = fqs_choose(a.B, a.V);
    const size_t rows = (size_t)a.B * w.plan.parts;
    w.bins = static_cast<fqs_u64*>(scratch);
    w.total = w.bins + rows * FQS_BINS;
    w.top = reinterpret_cast<float*>(w.total + rows);
    const dim3 grid((unsigned)w.plan.parts, (unsigned)a.B);
    if (a.wide) {
        hipLaunchKernelGGL(fqs_parts_kernel<true>, grid, dim3(FQS_T1), 0, stream, a, w);
        hipLaunchKernelGGL(fqs_row_kernel<true>, dim3((unsigned)a.B), dim3(FQS_T2), 0, stream, a, w);
    } else {
        hipLaunchKernelGGL(fqs_parts_kernel<false>, grid, dim3(FQS_T1), 0, stream, a, w);
        hipLaunchKernelGGL(fqs_row_kernel<false>, dim3((unsigned)a.B), dim3(FQS_T2), 0, stream, a, w);
    }
}
