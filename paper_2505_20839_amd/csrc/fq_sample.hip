// A token for each row of logits (include/fireq_sample.h).
//
// min-p, top-k and top-p all keep a first run of the tokens in one order (larger logit first, lower index first among equals), so
// what is kept is comp >= least for one number: comp = (ordered bits of the logit, inverted index).  It is found without sorting: of rows
// of up to 32761 logits by a workgroup each (fqs_row_kernel), of longer ones by three kernels:
//     parts    a row is cut into parts of up to 8192 logits.  Each finds its largest logit, takes e = exp((x - largest) / T) in whole numbers of
//              2^-32 (fq_mass.h; their sums do not depend on their order, and a token below 2^-33 of its part's best has no mass) and, where the row is
//              filtered at all, counts numbers and masses in FQS_BINS equal steps of x / T.  The steps lie on one grid for all parts.
//     borders  a workgroup per row adds the parts' bins and finds the bin in which min-p or top-k end, and those in which top-p may.
//     draw     the parts again: the tokens of those bins into a list.  The row's last workgroup selects among them, by number and then by mass, eight
//              bits of comp at a time (over the row again, where they are too many for its LDS), and finds the part, and in it the index, at which the
//              kept mass in index order passes u times its sum.
// 64 x 131072 of any filters 42 us in a graph (FP32 45; one row 35 and 33): 12, 9 and 23 under a profiler, where reading the logits once takes 3.4; what
// is left are steps that wait for each other (67 % of the last kernel's time).  One workgroup a row behind the parts' took 56 (512 rows: 140 and not 178).
#include <type_traits>

#include "fq_common.h"
#include "fq_kernels.h"
#include "fq_mass.h"

namespace {

typedef unsigned long long fqs_u64;

constexpr int FQS_BINS = 512, FQS_LIST = 4096, FQS_ROW_LIST = 2048, FQS_T1 = 256, FQS_MOST_PARTS = 256;
constexpr float FQS_SPAN = 23.0f;                         // nats that the bins cover: e^-23 is below 2^-33
constexpr fqs_u64 FQS_MASS = (1ull << 50) - 1;            // a part's bin: number of tokens << 50 | mass (8192 * 2^32 at most)

struct fqs_plan { int per, parts; };                      // chunks of 8 logits of a part; parts of a row
__host__ __device__ inline fqs_plan fqs_choose(int B, int V) {
    const int chunks = (V + 7 + 7) / 8;                   // (a row may begin inside a chunk)
    int per = FQS_T1;                                     // at least one chunk a thread, at most four
    while (per < 4 * FQS_T1 && (long long)B * ((chunks + per - 1) / per) > 1024) per += FQS_T1;
    if ((chunks + per - 1) / per > FQS_MOST_PARTS) per = 4 * FQS_T1;
    return {per, (chunks + per - 1) / per};
}

// What `borders` finds of a row, and what its workgroups in `draw` count.
struct fqs_border {
    float top, line;                                      // largest logit, the grid line below it (NaN: nothing can be drawn)
    fqs_u64 total, run, before, least;                    // masses: of all tokens; of the bins kept whole; of those before `low`.  min-p's comp
    fqs_u64 rank_left;                                    // top-k: tokens to keep of bin `end` (0: all)
    int end, low, high;                                   // bins: where min-p or top-k end, and from which to which top-p may (FQS_BINS: nowhere)
    int listed, arrived;                                  // in `draw`: tokens in the list, workgroups that are through
};
struct fqs_work {
    float* top;                                           // [B][parts] largest logit of a part; NaN: one that is NaN or +infinity
    fqs_u64* total;                                       // [B][parts] mass of all its tokens
    fqs_u64* sure;                                        // [B][parts] and of those in bins before the list's, in the row's unit
    fqs_u64* bins;                                        // [B][parts][FQS_BINS]
    fqs_u64* list;                                        // [B][FQS_LIST] comps
    fqs_border* border;                                   // [B]
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
// The grid line below x, -infinity for -infinity alone; x in bins from a line `top` (not below x's): top - line, dropped from FQS_BINS on.
__device__ __forceinline__ float fqs_line(float x, float steps) {
    const float y = floorf(__builtin_amdgcn_fmed3f(x * steps, -0x1p100f, 0x1p100f));
    return x > -__builtin_inff() ? y : x;
}
__device__ __forceinline__ fqs_u64 fqs_mass(float x, float top, float c) {
    return fqs_units(__builtin_amdgcn_exp2f((x - top) * c));
}

// Bits that order as the numbers do (-0 as 0), 16 of bf16 and 32 of FP32, above the inverted index.
template <bool WIDE>
__device__ __forceinline__ fqs_u64 fqs_key(float x) {
    const unsigned b = __float_as_uint(x + 0.0f), o = b & 0x80000000u ? ~b : b | 0x80000000u;
    return WIDE ? o : o >> 16;
}
template <bool WIDE>
__device__ __forceinline__ fqs_u64 fqs_comp(float x, int i) { return fqs_key<WIDE>(x) << 20 | (fqs_u64)(0xFFFFF - i); }

template <bool WIDE>
__device__ __forceinline__ float fqs_value(fqs_u64 comp) {
    const unsigned k = (unsigned)(comp >> 20), o = WIDE ? k : k << 16;
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : WIDE ? ~o : ~o & 0xFFFF0000u);
}

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
// The same, kept as they came.
template <bool WIDE>
struct fqs_pack {
    fq_v4i w[WIDE ? 2 : 1];
    __device__ __forceinline__ float operator[](int e) const {
        if constexpr (WIDE) { const int v = w[e >> 2][e & 3]; return __int_as_float(v); }
        const int v = w[0][(e >> 1) & 3];
        return e & 1 ? fq_bf16_hi(v) : fq_bf16_lo(v);
    }
    __device__ __forceinline__ float most() const {
        const fqs_pack& x = *this;
        return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    }
};
template <bool WIDE>
__device__ __forceinline__ fqs_pack<WIDE> fqs_load_pack(const fq_sample_args& a, int b, int skew, int c) {
    const int i0 = 8 * c - skew;
    const char* row = static_cast<const char*>(a.logits) + (long long)b * a.ld * (WIDE ? 4 : 2);
    fqs_pack<WIDE> x;
    if (i0 >= 0 && i0 + 8 <= a.V) {
        const fq_v4i* p = reinterpret_cast<const fq_v4i*>(row + (long long)i0 * (WIDE ? 4 : 2));
        x.w[0] = p[0];
        if constexpr (WIDE) x.w[1] = p[1];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = i0 + e;
            const bool in = i >= 0 && i < a.V;
            if constexpr (WIDE) {
                x.w[e >> 2][e & 3] = in ? reinterpret_cast<const int*>(row)[i] : (int)0xFF800000u;
            } else {
                const unsigned v = in ? reinterpret_cast<const uint16_t*>(row)[i] : 0xFF80u;
                if (e & 1) x.w[0][e >> 1] |= (int)(v << 16);
                else x.w[0][e >> 1] = (int)v;
            }
        }
    }
    return x;
}
// Tokens of chunk 0 that lie before the row: chunks begin at multiples of 16 bytes.
template <bool WIDE>
__device__ __forceinline__ int fqs_skew(const fq_sample_args& a, int b) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.logits) + (uintptr_t)((long long)b * a.ld * (WIDE ? 4 : 2));
    return (int)((p & 15) / (WIDE ? 4 : 2));
}

// Lanes' values moved within a wave: 1, 2, 4 and 8 up in a row of sixteen, then a row's last to the next row, and the first half's last to the second.  Lanes
// without a source keep `old`.
template <int STEP>
__device__ __forceinline__ int fqs_moved(int old, int v) {
    constexpr int CTRL = STEP == 16 ? 0x142 : STEP == 32 ? 0x143 : 0x110 + STEP, ROWS = STEP == 16 ? 0xA : STEP == 32 ? 0xC : 0xF;
    return __builtin_amdgcn_update_dpp(old, v, CTRL, ROWS, 0xF, false);
}
template <int STEP>
__device__ __forceinline__ float fqs_max_step(float v) { return fmaxf(v, __int_as_float(fqs_moved<STEP>(__float_as_int(v), __float_as_int(v)))); }
template <int STEP>
__device__ __forceinline__ fqs_u64 fqs_sum_step(fqs_u64 v) {
    return v + ((fqs_u64)(unsigned)fqs_moved<STEP>(0, (int)(v >> 32)) << 32 | (unsigned)fqs_moved<STEP>(0, (int)(unsigned)v));
}
template <int STEP>
__device__ __forceinline__ unsigned fqs_sum_step(unsigned v) { return v + (unsigned)fqs_moved<STEP>(0, (int)v); }
__device__ __forceinline__ float fqs_wave_max(float v) {
    v = fqs_max_step<32>(fqs_max_step<16>(fqs_max_step<8>(fqs_max_step<4>(fqs_max_step<2>(fqs_max_step<1>(v))))));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
// Inclusive sums over a wave's lanes.
template <class T>
__device__ __forceinline__ T fqs_wave_scan(T v) { return fqs_sum_step<32>(fqs_sum_step<16>(fqs_sum_step<8>(fqs_sum_step<4>(fqs_sum_step<2>(fqs_sum_step<1>(v)))))); }
__device__ __forceinline__ fqs_u64 fqs_last_lane(fqs_u64 v) {
    return (fqs_u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, 63);
}
__device__ __forceinline__ fqs_u64 fqs_wave_sum(fqs_u64 v) { return fqs_last_lane(fqs_wave_scan(v)); }

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

// Inclusive sums over a workgroup of THREADS threads, in their order; `all`: the sum.  (scratch: one number a wave)
template <int THREADS>
__device__ __forceinline__ fqs_u64 fqs_scan(fqs_u64 v, fqs_u64* scratch, fqs_u64& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = fqs_wave_scan(v);
    __syncthreads();
    if (lane == 63) scratch[wave] = v;
    __syncthreads();
    fqs_u64 before = 0;
    all = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
        if (i < wave) before += scratch[i];
        all += scratch[i];
    }
    return v + before;
}

__device__ __forceinline__ fqs_u64 fqs_scaled(fqs_u64 mass, float factor) { return (fqs_u64)rint((double)mass * (double)factor); }
// A part's masses in the row's unit, and its bins' distance from the row's.
__device__ __forceinline__ float fqs_factor(float part_top, float top, float c) { return part_top > -__builtin_inff() ? __builtin_amdgcn_exp2f((part_top - top) * c) : 0.0f; }
__device__ __forceinline__ int fqs_shift(float part_top, float line, float steps) {
    const float d = part_top > -__builtin_inff() ? line - fqs_line(part_top, steps) : (float)FQS_BINS;
    return d < (float)FQS_BINS ? (int)d : FQS_BINS;
}

// min-p: the least number that is kept, and the least comp.
__device__ __forceinline__ float fqs_lowest(const fqs_row& r, float top) {
    const double from = (double)top + r.T * log((double)r.low);
    const float x = (float)from;
    return (double)x >= from ? x : x < 0.0f ? __uint_as_float(__float_as_uint(x) - 1u) : x == 0.0f ? 0x1p-149f : __uint_as_float(__float_as_uint(x) + 1u);
}
__device__ __forceinline__ fqs_u64 fqs_least_of(float x, bool wide) {
    const unsigned bits = __float_as_uint(x + 0.0f), k = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    // (the ordered bits of a bf16 number end in sixteen zeros, or, below 0, in sixteen ones)
    return (wide ? (fqs_u64)k : k < 0x80000000u ? (fqs_u64)(k >> 16) : ((fqs_u64)k + 0xFFFF) >> 16) << 20;
}

// What the borders of a row leave in LDS.
struct fqs_bin_ends {
    fqs_u64 counts[16], masses[16];                       // of waves
    fqs_u64 ends[3][2], at_end[2];                        // of three borders: bin, what lies before it; masses before and up to `end`
};
// The borders in o, whose top, line and total are there, from the number and mass of bin t of a thread (0 behind the bins).  whole: the mass of all tokens
// (0: that of the bins).
__device__ __forceinline__ void fqs_find_borders(fqs_border& o, const fqs_row& r, bool wide, unsigned count, fqs_u64 mass, fqs_u64 whole, float line, fqs_bin_ends& sh) {
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    fqs_u64 counts = fqs_wave_scan(count), masses = fqs_wave_scan(mass), all = 0;
    if (lane == 63) { sh.counts[wave] = counts; sh.masses[wave] = masses; }
    __syncthreads();
    {
        fqs_u64 c = 0, m = 0;
#pragma unroll
        for (int i = 0; i < FQS_BINS / 64; ++i) {
            if (i < wave) { c += sh.counts[i]; m += sh.masses[i]; }
            all += sh.masses[i];
        }
        counts += c;
        masses += m;
        if (whole > 0) all = whole;
    }
    // where min-p ends: at a value
    int end = FQS_BINS;
    if (r.low > 0.0f) {
        const float x = fqs_lowest(r, o.top);
        o.least = fqs_least_of(x, wide);
        const float d = line - fqs_line(x, r.steps);
        end = d < (float)FQS_BINS ? (int)d : FQS_BINS;
    }
    // ... and top-k: the first border of the two
    if (t < 3) { sh.ends[t][0] = FQS_BINS; sh.ends[t][1] = all; }
    __syncthreads();
    const fqs_u64 k = (fqs_u64)r.k;
    if (k > 0 && counts >= k && counts - count < k && t <= end) {
        sh.ends[0][0] = t;
        sh.ends[0][1] = counts - count;
    }
    __syncthreads();
    if (sh.ends[0][0] < FQS_BINS) {
        end = (int)sh.ends[0][0];
        o.rank_left = k - sh.ends[0][1];
    }
    if (t == end) { sh.at_end[0] = masses - mass; sh.at_end[1] = masses; }
    __syncthreads();
    // what is kept of that bin lies between nothing and all, and so lie top-p's borders
    const fqs_u64 least_run = end < FQS_BINS ? sh.at_end[0] : all, most_run = end < FQS_BINS ? sh.at_end[1] : all;
    o.end = end;
    o.run = least_run;
    if (r.p < 1.0f) {
        const float p = fmaxf(r.p, 0.0f);
        const fqs_u64 lo = (fqs_u64)ceil((double)least_run * (double)p), hi = (fqs_u64)ceil((double)most_run * (double)p);
        const fqs_u64 first = lo < 1 ? 1 : lo, last = hi < 1 ? 1 : hi;
        if (masses >= first && masses - mass < first) { sh.ends[1][0] = t; sh.ends[1][1] = masses - mass; }
        if (masses >= last && masses - mass < last) sh.ends[2][0] = t;
        __syncthreads();
        o.low = (int)sh.ends[1][0];
        o.high = (int)sh.ends[2][0];
        o.before = sh.ends[1][1];
        if (o.high > end) o.high = end;
        if (o.low > o.high) o.low = o.high;           // (where only the end's bin is left)
    }
}

// A bin a thread.
__global__ __launch_bounds__(FQS_BINS) void fqs_borders_kernel(fq_sample_args a, fqs_work w) {
    constexpr int WAVES = FQS_BINS / 64;
    __shared__ fqs_u64 scan[WAVES];
    __shared__ float tops[WAVES], factor[FQS_MOST_PARTS];
    __shared__ int shift[FQS_MOST_PARTS];
    __shared__ fqs_bin_ends found;
    const int b = blockIdx.x, t = threadIdx.x, parts = w.plan.parts;
    const fqs_row r = fqs_parameters(a, b);
    fqs_border* const out = w.border + b;
    float top = -__builtin_inff(), mine = top;
    fqs_u64 part_total = 0;
    int bad = r.bad ? 1 : 0;
    if (t < parts) {
        mine = w.top[(size_t)b * parts + t];
        part_total = w.total[(size_t)b * parts + t];
        bad |= mine != mine ? 1 : 0;
    }
    top = fqs_wave_max(mine);
    if ((t & 63) == 0) tops[t >> 6] = top;
    bad = __syncthreads_or(bad);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) top = fmaxf(top, tops[i]);
    if (bad || !(top > -__builtin_inff())) {
        if (t == 0) {
            out->top = out->line = __builtin_nanf("");
            out->listed = out->arrived = 0;
        }
        return;
    }
    const float line = fqs_line(top, r.steps);
    if (t < parts) {
        factor[t] = fqs_factor(mine, top, r.c);
        shift[t] = fqs_shift(mine, line, r.steps);
        part_total = fqs_scaled(part_total, factor[t]);
    }
    fqs_u64 total;
    fqs_scan<FQS_BINS>(part_total, scan, total);          // (its barriers also publish factors and shifts)
    fqs_border o = {top, line, total, total, 0, 0, 0, FQS_BINS, FQS_BINS, FQS_BINS, 0, 0};
    if (r.filtered) {
        unsigned count = 0;
        fqs_u64 mass = 0;
        for (int p0 = 0; p0 < parts; p0 += 16) {          // (sixteen requested at a time)
            fqs_u64 v[16];
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                const int p = p0 + u < parts ? p0 + u : 0, q = t - shift[p];
                v[u] = w.bins[((size_t)b * parts + p) * FQS_BINS + (q < 0 ? 0 : q)];
                v[u] = q < 0 || p0 + u >= parts ? 0ull : v[u];
            }
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                count += (unsigned)(v[u] >> 50);
                mass += fqs_scaled(v[u] & FQS_MASS, factor[p0 + u < parts ? p0 + u : 0]);
            }
        }
        fqs_find_borders(o, r, a.wide, count, mass, 0, line, found);
    }
    if (t == 0) *out = o;
}

template <int LIST>
struct fqs_shared {
    static constexpr int ROOM = LIST;
    fqs_u64 scan[16], reach[16];                          // of waves
    fqs_u64 digit[2][256];
    fqs_u64 list[LIST];                                   // comps
    fqs_u64 found_before, found_own;
    int found, last;
};

// A workgroup of THREADS threads over the listed tokens of a row, or, where they are more than the list holds, over all: tokens(f) gives f each of the
// thread's share, as a logit and an index.
template <bool WIDE, int THREADS, class SHARED, class TOKENS>
struct fqs_finder {
    const fqs_row& r;
    SHARED& sh;
    const TOKENS& tokens;
    int t, n;                                             // n: tokens listed (or more than the list holds)
    float top, line;

    __device__ __forceinline__ int bin(float x) const {   // (-infinity lies in none)
        const float d = line - fqs_line(x, r.steps);
        return d < (float)FQS_BINS ? (int)d : FQS_BINS;
    }
    __device__ __forceinline__ fqs_u64 mass_of(fqs_u64 comp) const { return fqs_mass(fqs_value<WIDE>(comp), top, r.c); }
    // the tokens of bins lo .. hi
    template <class F>
    __device__ __forceinline__ void each(int lo, int hi, F f) const {
        if (n <= SHARED::ROOM) {
            for (int i = t; i < n; i += THREADS) {
                const int q = bin(fqs_value<WIDE>(sh.list[i]));
                if (q >= lo && q <= hi) f(sh.list[i]);
            }
            return;
        }
        tokens([&](float x, int i) __attribute__((always_inline)) {
            const int q = bin(x);
            if (q < FQS_BINS && q >= lo && q <= hi) f(fqs_comp<WIDE>(x, i));
        });
    }
    // The least comp of the best tokens of bins lo .. hi: of the first `want`, or (BY_MASS) of the first whose mass reaches `want`.  Eight bits at a
    // time from the highest in which their comps differ: sums for each digit, then the first wave finds the digit in which the run ends, while the
    // others clear the sums of the next eight.
    template <bool BY_MASS>
    __device__ __forceinline__ fqs_u64 select(int lo_bin, int hi_bin, fqs_u64 want) {
        const int lane = t & 63, wave = t >> 6;
        if (n <= 64) {                                    // each lane of a wave against every token
            __syncthreads();
            if (wave == 0) {
                const fqs_u64 own = lane < n ? sh.list[lane] : 0ull;
                const int q = lane < n ? bin(fqs_value<WIDE>(own)) : FQS_BINS;
                const bool in = q >= lo_bin && q <= hi_bin && q < FQS_BINS;
                const unsigned weight = in ? (BY_MASS ? (unsigned)mass_of(own) : 1u) : 0u;
                fqs_u64 before = 0, least = in ? own : ~0ull;
                for (int i = 0; i < n; ++i) {
                    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)own, i), hi = (unsigned)__builtin_amdgcn_readlane((int)(own >> 32), i);
                    const unsigned m = (unsigned)__builtin_amdgcn_readlane((int)weight, i);
                    before += ((fqs_u64)hi << 32 | lo) > own ? m : 0u;
                }
                least = in && before < want ? least : ~0ull;   // the worst of those that are kept
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const fqs_u64 l = __shfl_xor(least, d, 64);
                    least = l < least ? l : least;
                }
                if (lane == 0) sh.found_before = least == ~0ull ? 0ull : least;
            }
            __syncthreads();
            return sh.found_before;
        }
        fqs_u64 lo = ~0ull, hi = 0ull;
        each(lo_bin, hi_bin, [&](fqs_u64 c) __attribute__((always_inline)) { lo = c < lo ? c : lo; hi = c > hi ? c : hi; });
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const fqs_u64 l = __shfl_xor(lo, d, 64), h = __shfl_xor(hi, d, 64);
            lo = l < lo ? l : lo;
            hi = h > hi ? h : hi;
        }
        __syncthreads();
        if (lane == 0) { sh.scan[wave] = lo; sh.reach[wave] = hi; }
        if (t < 256) sh.digit[0][t] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) {
            lo = sh.scan[i] < lo ? sh.scan[i] : lo;
            hi = sh.reach[i] > hi ? sh.reach[i] : hi;
        }
        if (lo >= hi) return lo == hi ? lo : 0;           // one token, or none
        int above = 64 - __builtin_clzll(lo ^ hi);        // bits below are still open
        fqs_u64 prefix = hi >> above << above;            // (comps have 52 bits)
        const bool listed = n <= SHARED::ROOM;                // (their number then fits beside their mass)
        for (int buf = 0; above > 0; buf ^= 1) {
            const int width = above < 8 ? above : 8, shift = above - width;
            each(lo_bin, hi_bin, [&](fqs_u64 c) __attribute__((always_inline)) {
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
                const fqs_u64 cum = fqs_wave_scan(own);
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
                for (int i = t - 64; i < 256; i += THREADS - 64) sh.digit[buf ^ 1][i] = 0;
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
    // What is kept of a row whose borders are o: comp >= the answer.
    __device__ __forceinline__ fqs_u64 least(const fqs_border& o) {
        fqs_u64 l = o.least, run = o.run;
        const bool by_mass = o.low < FQS_BINS;
        if (o.end < FQS_BINS) {
            if (o.rank_left > 0) {
                const fqs_u64 x = select<false>(o.end, o.end, o.rank_left);
                l = x > l ? x : l;
            }
            if (by_mass) run += kept_in(o.end, o.end, l);
        }
        if (by_mass) {
            fqs_u64 want = (fqs_u64)ceil((double)run * (double)fmaxf(r.p, 0.0f));
            want = want < 1 ? 1 : want;
            const fqs_u64 x = select<true>(o.low, o.high, want > o.before ? want - o.before : 1);
            l = x > l ? x : l;
        }
        return l;
    }
    // The same where all that may be kept is listed.
    __device__ __forceinline__ fqs_u64 least_of_listed(fqs_u64 l) {
        if (r.k > 0) {
            const fqs_u64 x = select<false>(0, FQS_BINS - 1, (fqs_u64)r.k);
            l = x > l ? x : l;
        }
        if (r.p < 1.0f) {
            const fqs_u64 want = (fqs_u64)ceil((double)kept_in(0, FQS_BINS - 1, l) * (double)fmaxf(r.p, 0.0f)), x = select<true>(0, FQS_BINS - 1, want < 1 ? 1 : want);
            l = x > l ? x : l;
        }
        return l;
    }
    // The same of at most 256, by 1024 threads: four waves for 64 of them each compare these with a quarter of all, which gives every token the number and
    // the mass of those before it, and with these all filters.  (before, rank: zeros)
    __device__ __forceinline__ fqs_u64 least_of_few(fqs_u64 l, fqs_u64* before, unsigned* rank) {
        static_assert(THREADS == 1024, "sixteen waves");
        const int lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), groups = n <= 64 ? 1 : n <= 128 ? 2 : 4, quarter = 16 * groups;
        const int own_at = 64 * (wave & (groups - 1)), other_at = wave / groups * quarter;
        __syncthreads();
        if (other_at < n && own_at < n) {
            const int i = own_at + lane, j = other_at + lane;
            const fqs_u64 own = i < n ? sh.list[i] : 0ull, other = j < n ? sh.list[j] : 0ull;
            const unsigned weight = j < n ? (unsigned)mass_of(other) : 0u;
            fqs_u64 m = 0;
            unsigned k = 0;
            const int last = n - other_at < quarter ? n - other_at : quarter;
#pragma unroll 4
            for (int u = 0; u < last; ++u) {
                const fqs_u64 x = (fqs_u64)(unsigned)__builtin_amdgcn_readlane((int)(other >> 32), u) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)other, u);
                const unsigned w = (unsigned)__builtin_amdgcn_readlane((int)weight, u);
                const bool ahead = x > own;
                m += ahead ? w : 0u;
                k += ahead ? 1u : 0u;
            }
            if (i < n) {
                atomicAdd(&before[i], m);
                atomicAdd(&rank[i], k);
            }
        }
        __syncthreads();
        const fqs_u64 own = t < n ? sh.list[t] : 0ull, ahead = t < n ? before[t] : 0ull;
        bool kept = t < n && (r.k == 0 || rank[t] < (unsigned)r.k) && own >= l;
        if (r.p < 1.0f) {
            fqs_u64 run;
            fqs_scan<THREADS>(kept ? mass_of(own) : 0ull, sh.scan, run);
            const fqs_u64 want = (fqs_u64)ceil((double)run * (double)fmaxf(r.p, 0.0f));
            kept = kept && ahead < (want < 1 ? 1 : want);
        }
        fqs_u64 least = kept ? own : ~0ull;
        if (wave < 4) {
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const fqs_u64 o = __shfl_xor(least, d, 64);
                least = o < least ? o : least;
            }
            if (lane == 0) sh.reach[wave] = least;
        }
        __syncthreads();
        least = sh.reach[0];
#pragma unroll
        for (int i = 1; i < 4; ++i) least = sh.reach[i] < least ? sh.reach[i] : least;
        return least == ~0ull ? l : least;
    }
    // The token of a row of V at which the kept mass in index order passes u times the whole, all that are kept being listed: (its comp, or 0) in one thread.
    // Sums of the kept tokens of 512 equal ranges of indexes, then those of one range against each other.
    __device__ __forceinline__ fqs_u64 drawn(fqs_u64 least, float u, int V) {
        const int per = (V + 511) / 512;                  // at most 64
        fqs_u64* const sums = sh.digit[0];
        __syncthreads();
        if (t < 512) sums[t] = 0;
        if (t == 0) {
            sh.found = -1;
            sh.last = 0;
        }
        __syncthreads();
        for (int i = t; i < n; i += THREADS) {
            const fqs_u64 c = sh.list[i];
            if (c >= least) atomicAdd(&sums[(0xFFFFF - (int)(c & 0xFFFFF)) / per], mass_of(c));
        }
        __syncthreads();
        fqs_u64 all;
        const fqs_u64 own = t < 512 ? sums[t] : 0ull, cum = fqs_scan<THREADS>(own, sh.scan, all), target = (fqs_u64)((double)u * (double)all);
        if (cum > target && cum - own <= target) {        // (one thread's: u * all is below all)
            sh.found = t;
            sh.found_before = cum - own;
        }
        __syncthreads();
        const int range = sh.found;
        for (int i = t; i < n; i += THREADS) {
            const fqs_u64 c = sh.list[i];
            if (c >= least && (0xFFFFF - (int)(c & 0xFFFFF)) / per == range) sums[atomicAdd(&sh.last, 1)] = c;   // (no sum is read any more)
        }
        __syncthreads();
        if (t >= 64) return 0;
        const int count = sh.last;
        const fqs_u64 c = t < count ? sums[t] : 0ull;
        const unsigned weight = t < count ? (unsigned)mass_of(c) : 0u;
        fqs_u64 before = sh.found_before;
        for (int i = 0; i < count; ++i)                   // (a lower index: more in the low twenty bits)
            before += (unsigned)__builtin_amdgcn_readlane((int)(unsigned)c & 0xFFFFF, i) > ((unsigned)c & 0xFFFFFu) ? (unsigned)__builtin_amdgcn_readlane((int)weight, i) : 0u;
        return before <= target && target < before + weight ? c : 0ull;
    }
    // mass of the tokens of bins lo .. hi from `least` on
    __device__ __forceinline__ fqs_u64 kept_in(int lo, int hi, fqs_u64 least) {
        fqs_u64 m = 0, all;
        each(lo, hi, [&](fqs_u64 c) __attribute__((always_inline)) { if (c >= least) m += mass_of(c); });
        fqs_scan<THREADS>(m, sh.scan, all);
        return all;
    }
};

// At device scope: past the caches of an XCD.
__device__ __forceinline__ void fqs_store(fqs_u64* p, fqs_u64 v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ fqs_u64 fqs_fetch(const fqs_u64* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

template <bool WIDE>
__global__ __launch_bounds__(FQS_T1) void fqs_draw_kernel(fq_sample_args a, fqs_work w) {
    __shared__ fqs_shared<FQS_LIST> sh;
    __shared__ fqs_u64 part_mass[FQS_MOST_PARTS];         // kept mass of each part
    const int own_part = blockIdx.x, b = blockIdx.y, t = threadIdx.x, lane = t & 63, parts = w.plan.parts, per = w.plan.per;
    const int skew = fqs_skew<WIDE>(a, b), chunks = (a.V + skew + 7) / 8, mine = per / FQS_T1;
    float x[4][8];
#pragma unroll
    for (int u = 0; u < 4; ++u) {                         // (requested before it is known that they are looked at)
        const int c = own_part * per + u * FQS_T1 + t;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] = -__builtin_inff();
        if (u < mine && c < chunks) fqs_load<WIDE>(a, b, skew, c, x[u]);
    }
    const float part_top = w.top[(size_t)b * parts + own_part];
    fqs_u64 bins[FQS_BINS / FQS_T1];
#pragma unroll
    for (int i = 0; i < FQS_BINS / FQS_T1; ++i) bins[i] = w.bins[((size_t)b * parts + own_part) * FQS_BINS + t + i * FQS_T1];
    fqs_border* const border = w.border + b;
    const float top = border->top, line = border->line;
    if (!(top > -__builtin_inff())) {                     // (NaN)
        if (own_part == 0 && t == 0) {
            a.token[b] = -1;
            if (a.logprob) a.logprob[b] = __builtin_nanf("");
        }
        return;
    }
    const fqs_row r = fqs_parameters(a, b);
    const int end = border->end, low = border->low, high = border->high;
    const bool by_mass = low < FQS_BINS, listing = by_mass || end < FQS_BINS;
    const int first = by_mass ? low : end;                // bins before it are kept whole
    if (!listing && own_part != 0) return;                // every token is kept: one workgroup draws
    if (listing) {
        // the listed tokens: those of bin `end`, and of low .. high
        const float at0 = line - (float)low, at1 = line - (float)high, at2 = line - (float)end;
        unsigned hits = 0u;                               // bit 8 u + e
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = fqs_line(x[u][e], r.steps);
                hits |= (by_mass && y <= at0 && y >= at1) || (end < FQS_BINS && y == at2) ? 1u << (8 * u + e) : 0u;
            }
        const int count = __popc(hits);
        const int before = (int)fqs_wave_scan((unsigned)count);
        int at = 0;
        if (lane == 63 && before > 0) at = atomicAdd(&border->listed, before);
        at = __shfl(at, 63, 64) + before - count;
        while (hits != 0u) {
            const int bit = __ffs((int)hits) - 1;
            hits &= hits - 1u;
            float v = x[0][0];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) v = bit == 8 * u + e ? x[u][e] : v;
            const int c = own_part * per + (bit >> 3) * FQS_T1 + t;
            if (at < FQS_LIST) fqs_store(w.list + (size_t)b * FQS_LIST + at, fqs_comp<WIDE>(v, 8 * c - skew + (bit & 7)));
            ++at;
        }
        fqs_u64 sure = 0, all;
        const int shift = fqs_shift(part_top, line, r.steps);
        const float f = fqs_factor(part_top, top, r.c);
#pragma unroll
        for (int i = 0; i < FQS_BINS / FQS_T1; ++i)
            if (t + i * FQS_T1 + shift < first) sure += fqs_scaled(bins[i] & FQS_MASS, f);
        fqs_scan<FQS_T1>(sure, sh.scan, all);
        if (t == 0) fqs_store(w.sure + (size_t)b * parts + own_part, all);
        // The row's last workgroup goes on.  What it reads of the others was stored and is read at device scope, and every store has been acknowledged there
        // before its workgroup counts itself in (a fence would write back the whole L2 for each).
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (t == 0) sh.last = __hip_atomic_fetch_add(&border->arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1 ? 1 : 0;
        __syncthreads();
        if (!sh.last) return;
    }
    auto tokens = [&](auto f) __attribute__((always_inline)) {
        for (int c = t; c < chunks; c += FQS_T1) {
            float v[8];
            fqs_load<WIDE>(a, b, skew, c, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) f(v[e], 8 * c - skew + e);
        }
    };
    fqs_finder<WIDE, FQS_T1, decltype(sh), decltype(tokens)> find = {r, sh, tokens, t, 0, top, line};
    fqs_u64 least = border->least, kept;                  // kept tokens: comp >= least
    if (listing) {
        find.n = __hip_atomic_load(&border->listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (find.n <= FQS_LIST)
            for (int i = t; i < find.n; i += FQS_T1) sh.list[i] = fqs_fetch(w.list + (size_t)b * FQS_LIST + i);
    }
    if (t == 0) sh.found = 0;
    if (t < parts) {
        if (listing) {
            part_mass[t] = fqs_fetch(w.sure + (size_t)b * parts + t);
        } else {
            // (min-p may end beyond the bins: of a part whose best lies below that nothing is kept, though its tokens may have a mass together)
            const float best = w.top[(size_t)b * parts + t];
            part_mass[t] = fqs_comp<WIDE>(best, 0) >= least ? fqs_scaled(w.total[(size_t)b * parts + t], fqs_factor(best, top, r.c)) : 0ull;
        }
    }
    __syncthreads();
    if (listing) least = find.least(*border);
    if (listing) {
        find.each(first, by_mass ? high : end, [&](fqs_u64 c) __attribute__((always_inline)) {
            if (c >= least) atomicAdd(&part_mass[((int)(0xFFFFF - (c & 0xFFFFF)) + skew) / 8 / per], find.mass_of(c));
        });
        __syncthreads();
    }
    // the part, then the token, at which the mass in index order passes u times the whole
    const fqs_u64 own = t < parts ? part_mass[t] : 0, cum = fqs_scan<FQS_T1>(own, sh.scan, kept);
    const float u = fminf(fmaxf(a.u[b], 0.0f), 0x1.fffffep-1f);
    const fqs_u64 target = (fqs_u64)((double)u * (double)kept);
    if (cum > target && cum - own <= target) {            // (one thread's: u * kept is below kept)
        sh.found = t;
        sh.found_before = cum - own;
    }
    __syncthreads();
    const int part = sh.found;
    const float best = w.top[(size_t)b * parts + part];
    float y[4][8];
    fqs_u64 m = 0;
    const int c0 = part * per + 4 * t;                    // four chunks of a thread, one behind the other
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (4 * t + i < per) fqs_load<WIDE>(a, b, skew, c0 + i, y[i]);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) y[i][e] = -__builtin_inff();
    }
    // comp >= least as a value and the last index that is kept of it (a bound below -infinity's keeps all; -infinity itself has no mass)
    const bool all_kept = least <= fqs_comp<WIDE>(-__builtin_inff(), 0);
    const float bound = all_kept ? -__builtin_inff() : fqs_value<WIDE>(least);
    const int last_index = 0xFFFFF - (int)(least & 0xFFFFF);
    auto mass = [&](int i, int e) __attribute__((always_inline)) {
        const float v = y[i][e];
        return v > bound || (v == bound && 8 * (c0 + i) - skew + e <= last_index) ? (unsigned)fqs_mass(v, best, r.c) : 0u;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) m += mass(i, e);
    fqs_u64 in_part, at = fqs_scan<FQS_T1>(m, sh.scan, in_part) - m;
    // (the part's own sum and the bins' may differ by rounding: the last token with a mass then)
    double want = (double)(target - sh.found_before) / (double)fqs_factor(best, top, r.c);
    if (!(want < (double)in_part)) want = in_part > 0 ? (double)(in_part - 1) : 0.0;
    if ((double)at <= want && want < (double)(at + m)) {
        int token = -1;
        float value = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (token >= 0) continue;
                at += mass(i, e);
                if ((double)at > want) {
                    token = 8 * (c0 + i) - skew + e;
                    value = y[i][e];
                }
            }
        a.token[b] = token;
        if (a.logprob) a.logprob[b] = (float)(((double)value - (double)top) / r.T - log((double)border->total / FQS_UNIT));
    }
}

// A row for one workgroup: all of it in one kernel, without scratch.  Bound by one compute unit's vector instructions and by its steps' latency.  In a
// graph, against the three kernels: 1 x 5000 11 us (28), 1 x 32000 14.5 (27), 64 rows of any filters 19 and 35 (32 and 35); 64 x 50000 would take 51 (37).
// FP32: 1 x 32000 14, 64 x 32000 34.
// Where top-k, or min-p with top-p, leave at most 2048 tokens above a border known beforehand, these are listed in the pass that sums exponentials, and
// nothing is binned: 1 x 32000 with top-k 50 and top-p 26 us before.  Otherwise the steps are those of the three kernels, with one unit for all masses.
// Wave w has the chunks 64 n w .. 64 n (w + 1) - 1, n of a lane, 64 apart, and CHUNKS of all fit LDS.
template <bool WIDE, int CHUNKS>
__global__ __launch_bounds__(1024) void fqs_row_kernel(fq_sample_args a) {
    constexpr int THREADS = 1024, WAVES = THREADS / 64, SIZE = WIDE ? 2 : 1;
    __shared__ fqs_shared<FQS_ROW_LIST> sh;
    __shared__ fqs_bin_ends found;
    __shared__ fqs_u64 mass_of_bin[FQS_BINS];
    __shared__ unsigned count_of_bin[FQS_BINS];
    __shared__ float wave_top[WAVES];
    __shared__ int listed;
    __shared__ fq_v4i held[SIZE * CHUNKS];
    const int b = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int skew = fqs_skew<WIDE>(a, b), chunks = (a.V + skew + 7) / 8, n = (chunks + THREADS - 1) / THREADS, c0 = 64 * n * wave + lane;
    // f(chunk number, its eight logits) for this lane's; the first time they are fetched
    auto each = [&](auto fetched, auto f) __attribute__((always_inline)) {
        auto get = [&](int c) __attribute__((always_inline)) {
            fqs_pack<WIDE> x;
            if constexpr (!fetched) {
                x = fqs_load_pack<WIDE>(a, b, skew, c);
            } else {
#pragma unroll
                for (int u = 0; u < SIZE; ++u) x.w[u] = held[SIZE * c + u];   // (its own wave's)
            }
            return x;
        };
        int i = 0;
        for (; i + 4 <= n; i += 4) {
            fqs_pack<WIDE> x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = get(c0 + 64 * (i + u));
#pragma unroll
            for (int u = 0; u < 4; ++u) f(c0 + 64 * (i + u), x[u]);
        }
        for (; i < n; ++i) f(c0 + 64 * i, get(c0 + 64 * i));
    };
    const fqs_row r = fqs_parameters(a, b);
    if (t < FQS_BINS) {
        mass_of_bin[t] = 0;
        count_of_bin[t] = 0;
    }
    if (t == 0) listed = 0;
    float top = -__builtin_inff();
    int bad = r.bad ? 1 : 0;
    each(std::false_type(), [&](int c, const fqs_pack<WIDE>& x) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < SIZE; ++u) held[SIZE * c + u] = x.w[u];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = x[e];
            bad |= !(v < __builtin_inff()) ? 1 : 0;
            top = fmaxf(top, v);
        }
    });
    top = fqs_wave_max(top);
    if (lane == 0) wave_top[wave] = top;
    bad = __syncthreads_or(bad);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) top = fmaxf(top, wave_top[i]);
    if (bad || !(top > -__builtin_inff())) {
        if (t == 0) {
            a.token[b] = -1;
            if (a.logprob) a.logprob[b] = __builtin_nanf("");
        }
        return;
    }
    const float line = fqs_line(top, r.steps);
    // `cut`: nothing below it is kept.  top-k: of the chunks' largest logits the k-th is at most the k-th of all; min-p: its own border.
    float cut = -__builtin_inff();
    bool listing = false;
    if (r.k > 0 && 2 * r.k <= chunks && fabsf(line) < 0x1p99f) {
        each(std::true_type(), [&](int, const fqs_pack<WIDE>& x) __attribute__((always_inline)) {
            const float d = line - fqs_line(x.most(), r.steps);
            if (d < (float)FQS_BINS) atomicAdd(&count_of_bin[(int)d], 1u);
        });
        if (t == 0) sh.found = FQS_BINS;
        __syncthreads();
        unsigned count = 0, counts = 0;
        if (t < FQS_BINS) {
            count = count_of_bin[t];
            counts = fqs_wave_scan(count);
            if (lane == 63) found.counts[wave] = counts;
        }
        __syncthreads();
        if (t < FQS_BINS) {
            count_of_bin[t] = 0;
#pragma unroll
            for (int i = 0; i < FQS_BINS / 64; ++i) counts += i < wave ? (unsigned)found.counts[i] : 0u;
            if (counts >= (unsigned)r.k && counts - count < (unsigned)r.k) sh.found = t;
        }
        __syncthreads();
        if (sh.found < FQS_BINS) {
            const float x = (line - (float)sh.found) / r.steps;
            cut = x - fmaxf(fabsf(x) * 0x1p-20f, 0x1p-149f / r.steps);   // (a number in that bin is not below, nor one whose steps underflow to it)
            listing = true;
        }
    }
    fqs_u64 least = 0;
    if (r.low > 0.0f) {
        const float x = fqs_lowest(r, top);
        least = fqs_least_of(x, WIDE);
        cut = fmaxf(cut, x);
        listing = listing || r.p < 1.0f;
    }
    auto note = [&](int c, const fqs_pack<WIDE>& x, float from) __attribute__((always_inline)) {
        if (!(x.most() >= from)) return;
        unsigned hits = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) hits |= x[e] >= from ? 1u << e : 0u;
        if (hits == 0u) return;
        int at = atomicAdd(&listed, __popc(hits));
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (hits >> e & 1u) {
                if (at < FQS_ROW_LIST) sh.list[at] = fqs_comp<WIDE>(x[e], 8 * c - skew + e);
                ++at;
            }
    };
    // the mass of all tokens: in whole numbers where top-p alone takes its part of it (8 x 32000 15.6 us for 15.2); otherwise it is the log-probability's,
    // and FP32's (a thread's numbers in their order)
    const bool by_mass_alone = r.p < 1.0f && r.k == 0 && !(r.low > 0.0f);
    fqs_u64 total;
    if (by_mass_alone) {
        fqs_u64 sum = 0;
        each(std::true_type(), [&](int, const fqs_pack<WIDE>& x) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += fqs_mass(x[e], top, r.c);
        });
        fqs_scan<THREADS>(sum, sh.scan, total);
    } else {
        float sum = 0.f;
        each(std::true_type(), [&](int c, const fqs_pack<WIDE>& x) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += __builtin_amdgcn_exp2f((x[e] - top) * r.c);
            if (listing) note(c, x, cut);
        });
        fqs_scan<THREADS>((fqs_u64)(sum * FQS_UNIT), sh.scan, total);
    }
    const float u = fminf(fmaxf(a.u[b], 0.0f), 0x1.fffffep-1f);
    auto answer = [&](int token, float value) __attribute__((always_inline)) {
        a.token[b] = token;
        if (a.logprob) a.logprob[b] = (float)(((double)value - (double)top) / r.T - log((double)total / FQS_UNIT));
    };
    if (r.k > 0 || r.p < 1.0f) {
        auto tokens = [&](auto f) __attribute__((always_inline)) {
            each(std::true_type(), [&](int c, const fqs_pack<WIDE>& x) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) f(x[e], 8 * c - skew + e);
            });
        };
        fqs_finder<WIDE, THREADS, decltype(sh), decltype(tokens)> find = {r, sh, tokens, t, listed, top, line};
        if (listing && find.n <= FQS_ROW_LIST) {
            least = find.n <= 256 ? find.least_of_few(least, mass_of_bin, count_of_bin) : find.least_of_listed(least);
            const fqs_u64 c = find.drawn(least, u, a.V);
            if (c != 0) answer(0xFFFFF - (int)(c & 0xFFFFF), fqs_value<WIDE>(c));
            return;
        } else {
            // numbers and masses in bins.  top-p alone: tokens with less than half (1 - p) / V of the mass do not reach what it leaves out
            const float lightest = by_mass_alone ? 0.49f * (1.0f - fmaxf(r.p, 0.0f)) * ((float)total * (1.0f / FQS_UNIT)) / (float)a.V : 0.0f;
            __syncthreads();
            if (t == 0) listed = 0;
            each(std::true_type(), [&](int, const fqs_pack<WIDE>& x) __attribute__((always_inline)) {
                if (!(x.most() >= cut)) return;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = x[e], weight = __builtin_amdgcn_exp2f((v - top) * r.c), d = line - fqs_line(v, r.steps);
                    if (v >= cut && weight >= lightest && d < (float)FQS_BINS) {
                        if (r.k > 0) atomicAdd(&count_of_bin[(int)d], 1u);
                        if (r.p < 1.0f) atomicAdd(&mass_of_bin[(int)d], (fqs_u64)fqs_units(weight));
                    }
                }
            });
            __syncthreads();
            fqs_border o = {top, line, total, total, 0, 0, 0, FQS_BINS, FQS_BINS, FQS_BINS, 0, 0};
            fqs_find_borders(o, r, WIDE, t < FQS_BINS ? count_of_bin[t] : 0u, t < FQS_BINS ? mass_of_bin[t] : 0ull, by_mass_alone ? total : 0, line, found);
            const bool by_mass = o.low < FQS_BINS;
            least = o.least;
            if (by_mass || o.end < FQS_BINS) {
                const float at0 = line - (float)o.low, at1 = line - (float)o.high, at2 = line - (float)o.end;
                each(std::true_type(), [&](int c, const fqs_pack<WIDE>& x) __attribute__((always_inline)) {
                    const float y = fqs_line(x.most(), r.steps);
                    if (!((by_mass && y >= at1) || (o.end < FQS_BINS && y >= at2))) return;
                    unsigned hits = 0u;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float y = fqs_line(x[e], r.steps);
                        hits |= (by_mass && y <= at0 && y >= at1) || (o.end < FQS_BINS && y == at2) ? 1u << e : 0u;
                    }
                    if (hits == 0u) return;
                    int at = atomicAdd(&listed, __popc(hits));
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (hits >> e & 1u) {
                            if (at < FQS_ROW_LIST) sh.list[at] = fqs_comp<WIDE>(x[e], 8 * c - skew + e);
                            ++at;
                        }
                });
                __syncthreads();
                find.n = listed;
                least = find.least(o);
            }
        }
    }
    // the wave, the chunk and the token at which the kept mass in index order passes u times the whole
    const bool all_kept = least <= fqs_comp<WIDE>(-__builtin_inff(), 0);
    const float bound = all_kept ? -__builtin_inff() : fqs_value<WIDE>(least);
    const int last_index = 0xFFFFF - (int)(least & 0xFFFFF);
    auto mass = [&](int c, const fqs_pack<WIDE>& x, int e) __attribute__((always_inline)) {
        const float v = x[e];
        return v > bound || (v == bound && 8 * c - skew + e <= last_index) ? fqs_mass(v, top, r.c) : 0ull;
    };
    fqs_u64 own = 0;
    each(std::true_type(), [&](int c, const fqs_pack<WIDE>& x) __attribute__((always_inline)) {
        if (!(x.most() >= bound)) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) own += mass(c, x, e);
    });
    own = fqs_wave_sum(own);
    __syncthreads();
    if (lane == 0) sh.scan[wave] = own;
    __syncthreads();
    fqs_u64 before = 0, kept = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        before += i < wave ? sh.scan[i] : 0ull;
        kept += sh.scan[i];
    }
    const fqs_u64 target = (fqs_u64)((double)u * (double)kept);
    if (!(before <= target && target < before + own)) return;
    each(std::true_type(), [&](int c, const fqs_pack<WIDE>& x) __attribute__((always_inline)) {
        fqs_u64 m = 0;
        if (!__any(x.most() >= bound)) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) m += mass(c, x, e);
        fqs_u64 at = fqs_wave_scan(m);
        const fqs_u64 all = fqs_last_lane(at);
        at += before - m;
        before += all;
        if (at > target || target >= at + m) return;
        int token = -1;
        float value = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (token >= 0) continue;
            at += mass(c, x, e);
            if (at > target) {
                token = 8 * c - skew + e;
                value = x[e];
            }
        }
        answer(token, value);
    });
}

// Rows that one workgroup takes: up to 4096 chunks.
bool fqs_one_workgroup(int V) { return V + 7 <= 4096 * 8; }

template <bool WIDE>
void fqs_launch_row(const fq_sample_args& a, hipStream_t stream) {
    if (a.V + 7 <= 1024 * 8) hipLaunchKernelGGL((fqs_row_kernel<WIDE, 1024>), dim3((unsigned)a.B), dim3(1024), 0, stream, a);
    else hipLaunchKernelGGL((fqs_row_kernel<WIDE, 4096>), dim3((unsigned)a.B), dim3(1024), 0, stream, a);
}

}  // namespace

size_t fq_sample_scratch_bytes(int B, int V) {
    if (fqs_one_workgroup(V)) return 0;
    const size_t rows = (size_t)B * fqs_choose(B, V).parts;
    return rows * (8 * FQS_BINS + 16) + (size_t)B * (8 * FQS_LIST + sizeof(fqs_border)) + (rows * 4 + 15) / 16 * 16;
}

void fq_launch_sample(const fq_sample_args& a, void* scratch, hipStream_t stream) {
    if (fqs_one_workgroup(a.V)) {
        if (a.wide) fqs_launch_row<true>(a, stream);
        else fqs_launch_row<false>(a, stream);
        return;
    }
    fqs_work w;
    w.plan = fqs_choose(a.B, a.V);
    const size_t rows = (size_t)a.B * w.plan.parts;
    w.bins = static_cast<fqs_u64*>(scratch);
    w.total = w.bins + rows * FQS_BINS;
    w.sure = w.total + rows;
    w.list = w.sure + rows;
    w.border = reinterpret_cast<fqs_border*>(w.list + (size_t)a.B * FQS_LIST);
    w.top = reinterpret_cast<float*>(w.border + a.B);
    const dim3 grid((unsigned)w.plan.parts, (unsigned)a.B);
    if (a.wide) hipLaunchKernelGGL(fqs_parts_kernel<true>, grid, dim3(FQS_T1), 0, stream, a, w);
    else hipLaunchKernelGGL(fqs_parts_kernel<false>, grid, dim3(FQS_T1), 0, stream, a, w);
    hipLaunchKernelGGL(fqs_borders_kernel, dim3((unsigned)a.B), dim3(FQS_BINS), 0, stream, a, w);
    if (a.wide) hipLaunchKernelGGL(fqs_draw_kernel<true>, grid, dim3(FQS_T1), 0, stream, a, w);
    else hipLaunchKernelGGL(fqs_draw_kernel<false>, grid, dim3(FQS_T1), 0, stream, a, w);
}
