// Residual addition and root-mean-square norm in front of a quantised layer (include/fireq_norm.h):
//     h = bf16(x + r),  y = h * w / sqrt(mean h^2 + eps),  codes = E4M3(y / beta),  beta = max |y| / 448
// in one pass over the row: with t = max |h w| the row's two statistics, sum h^2 and t, come out of one reduction, beta is
// t * rstd / 448 and a code is E4M3(448 h w / t) -- rstd cancels, so no value waits for it, and adds no rounding.
// Bound by HBM: 7 bytes per element with the residual, 3 without (bf16 output: 8 and 4).
//
// Between two blocks with a norm on both sides (include/fireq_norm_block.h) the stream takes x by its own norm, a gate and a factor first:
//     h = bf16(r + scale * gate * (x * post / sqrt(mean x^2 + eps)))
// The same bytes and one more reduction over the row, which is in registers by then (in a second pass over rows that the registers do not hold).  The
// norm's sums are added in the order of the other forms, so that it is that of the stream, bit for bit.  Measured, calls back to back: 8192 x 4096 to
// E4M3 45 us (235 MB, 5.2 TB/s: the rate of a copy), 1000 x 5120 to bf16 with a gate row for each of 7 sequences 9.8 us (41 MB, 4.2 TB/s, vector
// instructions nearly as busy), one row 3.6 us in a graph.  With a prepared workspace, in a graph, without it in brackets: 100 x 4096 4.3 us (3.9),
// 1000 x 5120 10.5 (9.8), 4096 x 4096 21.1 (20.6), 8192 x 4096 37.5 (36.2).
#include <type_traits>
#include "fq_common.h"
#include "fq_kernels.h"

namespace {

enum { FQN_BF16 = 0, FQN_CODES = 1, FQN_CODES_ZP = 2 };   // what leaves: bf16, codes and scale, and the GEMM's zero-point terms too

// The sum of a wave, in every lane.
__device__ __forceinline__ float fqn_wave_sum(float v) {
    v = fq_row16_sum(v);
    const int b = (int)__float_as_uint(v);
    return (__uint_as_float((unsigned)__builtin_amdgcn_readlane(b, 0)) + __uint_as_float((unsigned)__builtin_amdgcn_readlane(b, 16))) +
           (__uint_as_float((unsigned)__builtin_amdgcn_readlane(b, 32)) + __uint_as_float((unsigned)__builtin_amdgcn_readlane(b, 48)));
}

__device__ __forceinline__ unsigned fqn_pack_bf16(float a, float b) {
    return __builtin_bit_cast(unsigned, __builtin_convertvector((fq_v2f){a, b}, fq_v2bf));
}

// Eight bf16 sums, each rounded once.
__device__ __forceinline__ fq_v4i fqn_add8(fq_v4i x, fq_v4i r) {
    fq_v4i h;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        h[j] = (int)fqn_pack_bf16(fq_bf16_lo(x[j]) + fq_bf16_lo(r[j]), fq_bf16_hi(x[j]) + fq_bf16_hi(r[j]));
    return h;
}

// One chunk's part of the statistics.  The largest |h w| is searched among the bit patterns: a NaN lies above all numbers.
__device__ __forceinline__ void fqn_take8(fq_v4i h, fq_v4i w, float& ss, unsigned& top) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float a = fq_bf16_lo(h[j]), b = fq_bf16_hi(h[j]);
        ss = fmaf(a, a, ss);
        ss = fmaf(b, b, ss);
        const unsigned p = __float_as_uint(a * fq_bf16_lo(w[j])) & 0x7FFFFFFFu, q = __float_as_uint(b * fq_bf16_hi(w[j])) & 0x7FFFFFFFu;
        top = p > top ? p : top;
        top = q > top ? q : top;
    }
}

template <class F>
__device__ __forceinline__ fq_v2i fqn_codes8(fq_v4i h, fq_v4i w, F quotient) {
    fq_v2i o;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        int r = 0;
        r = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(fq_bf16_lo(h[2 * j]) * fq_bf16_lo(w[2 * j])),
                                            quotient(fq_bf16_hi(h[2 * j]) * fq_bf16_hi(w[2 * j])), r, false);
        r = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(fq_bf16_lo(h[2 * j + 1]) * fq_bf16_lo(w[2 * j + 1])),
                                            quotient(fq_bf16_hi(h[2 * j + 1]) * fq_bf16_hi(w[2 * j + 1])), r, true);
        o[j] = r;
    }
    return o;
}

struct fqn_none {};

// Eight numbers of the stream, each rounded once: r + scale * g * (x * f * p).
__device__ __forceinline__ fq_v4i fqn_branch8(fq_v4i x, fq_v4i r, fq_v4i p, fq_v4i g, float f, float scale) {
    fq_v4i h;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        h[j] = (int)fqn_pack_bf16(fmaf(scale, fq_bf16_lo(g[j]) * (fq_bf16_lo(x[j]) * f * fq_bf16_lo(p[j])), fq_bf16_lo(r[j])),
                                  fmaf(scale, fq_bf16_hi(g[j]) * (fq_bf16_hi(x[j]) * f * fq_bf16_hi(p[j])), fq_bf16_hi(r[j])));
    return h;
}
__device__ __forceinline__ float fqn_squares8(fq_v4i x, float ss) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        ss = fmaf(fq_bf16_lo(x[j]), fq_bf16_lo(x[j]), ss);
        ss = fmaf(fq_bf16_hi(x[j]), fq_bf16_hi(x[j]), ss);
    }
    return ss;
}

// WPR waves per row with up to CH chunks (16 bytes, 8 numbers) of it per thread; workgroups of max(4, WPR) waves.  The row and
// the weights stay in registers between the reduction and the conversion; rows that do not fit are read twice (REREAD).
// X, R, H and Y may be one array (no __restrict__): a chunk is read and written by one thread only, and a thread requests all of
// its chunks before it stores any.
template <int WPR, int CH, bool RES, int OUT, bool REREAD, bool BRANCH>
__global__ __launch_bounds__(WPR > 4 ? 64 * WPR : 256) void fqn_kernel(const uint16_t* X, const uint16_t* R, const uint16_t* __restrict__ Wt,
                                                                      float eps, uint16_t* H, uint16_t* Y, uint8_t* __restrict__ A,
                                                                      float* __restrict__ a_scale, int K, uint16_t* __restrict__ planes, int M,
                                                                      std::conditional_t<BRANCH, fq_norm_branch, fqn_none> branch) {
    static_assert(!(OUT == FQN_CODES_ZP && REREAD), "the zero-point terms are summed from registers");
    static_assert(RES || !BRANCH, "the branch is added to a residual");
    constexpr int WAVES = WPR > 4 ? WPR : 4, ROWS = WAVES / WPR, T = 64 * WPR;
    constexpr int MAXG = T * CH / 16 + 16;                // groups of a row, padded
    constexpr bool ZP = OUT == FQN_CODES_ZP;
    // the sums are those of twice the waves with two chunks a thread, bit for bit: a thread has chunks 0 and 2 of one of them, 1 and 3 of another
    constexpr bool HALVES = BRANCH && !REREAD && (WPR == 4 || WPR == 8) && (CH == 3 || CH == 4);
    __shared__ float red_sum[HALVES ? 2 * WAVES : WAVES];
    __shared__ unsigned red_top[WAVES];
    __shared__ __attribute__((aligned(16))) uint16_t zrow[ZP ? ROWS : 1][2][ZP ? MAXG : 8];   // [row][plane][group]
    const int row = (int)threadIdx.x / T, t = (int)threadIdx.x % T, m = (int)blockIdx.x * ROWS + row;
    if (ZP && M <= FQ_KSPLIT_MAX_M) {                     // the arrival counters behind the planes start at zero
        const int G = K >> 7, C2 = 2 * ((G + 15) >> 4);
        unsigned* counters = reinterpret_cast<unsigned*>(planes + (size_t)2 * C2 * M * 8);
        for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < FQ_KSPLIT_COUNTERS; i += gridDim.x * blockDim.x) counters[i] = 0u;
    }
    const bool on = m < M;                                // (rows past M repeat the last one and store nothing)
    const size_t at = (size_t)(on ? m : M - 1) * K;
    const int nchunk = K >> 3;
    const fq_v4i *x = reinterpret_cast<const fq_v4i*>(X + at), *r = reinterpret_cast<const fq_v4i*>(R + (RES ? at : 0));
    const fq_v4i* w = reinterpret_cast<const fq_v4i*>(Wt);
    fq_v4i* hs = reinterpret_cast<fq_v4i*>(H + (RES ? at : 0));
    float ss = 0.f, other = 0.f;
    unsigned top = 0u;
    fq_v4i keep[CH], wt[CH];
    constexpr int ONES = 0x3F803F80;                      // bf16 ones, where there is no weight or gate
    // the block form: 1 / sqrt(mean x^2 + eps) of the row (1 without that norm); NaN for a row that has none, or no gate
    auto branch_factor = [&](float xx, bool lost) __attribute__((always_inline)) {
        float f = 1.0f;
        if constexpr (BRANCH) {
            __shared__ float red_x[WAVES];
            if (branch.post) {
                xx = fqn_wave_sum(xx);
                if (WPR > 1) {
                    if ((t & 63) == 0) red_x[(int)threadIdx.x >> 6] = xx;
                    __syncthreads();
                    xx = red_x[row * WPR];
#pragma unroll
                    for (int i = 1; i < WPR; ++i) xx += red_x[row * WPR + i];
                }
                f = xx < __builtin_inff() ? 1.0f / sqrtf(xx / (float)K + eps) : __builtin_nanf("");
            }
            if (lost) f = __builtin_nanf("");
        }
        return f;
    };
    const fq_v4i *post = nullptr, *gate = nullptr;
    bool lost = false;
    if constexpr (BRANCH) {
        const int mm = on ? m : M - 1, g = branch.rows ? branch.rows[mm] : branch.gates == 1 ? 0 : mm;
        lost = branch.gate && (unsigned)g >= (unsigned)branch.gates;
        post = reinterpret_cast<const fq_v4i*>(branch.post);
        if (branch.gate) gate = reinterpret_cast<const fq_v4i*>(branch.gate + (size_t)(lost ? 0 : g) * K);
    }
    if constexpr (BRANCH && !REREAD) {
        fq_v4i add[CH], pw[CH], gt[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = t + i * T < nchunk ? t + i * T : nchunk - 1;
            keep[i] = x[c];
            add[i] = r[c];
            wt[i] = w[c];
            pw[i] = post ? post[c] : (fq_v4i){ONES, ONES, ONES, ONES};
            gt[i] = gate ? gate[c] : (fq_v4i){ONES, ONES, ONES, ONES};
        }
        float xx = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (t + i * T < nchunk) xx = fqn_squares8(keep[i], xx);
        const float f = branch_factor(xx, lost);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            keep[i] = fqn_branch8(keep[i], add[i], pw[i], gt[i], f, branch.scale);
            if (t + i * T >= nchunk) keep[i] = (fq_v4i){0, 0, 0, 0};
            fqn_take8(keep[i], wt[i], HALVES && i % 2 == 1 ? other : ss, top);
        }
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (on && t + i * T < nchunk) hs[t + i * T] = keep[i];
    } else if constexpr (BRANCH) {
        float xx = 0.f;
        for (int c = t; c < nchunk; c += T) xx = fqn_squares8(x[c], xx);
        const float f = branch_factor(xx, lost);
        for (int c = t; c < nchunk; c += T) {
            const fq_v4i ones = {ONES, ONES, ONES, ONES}, h = fqn_branch8(x[c], r[c], post ? post[c] : ones, gate ? gate[c] : ones, f, branch.scale);
            if (on) hs[c] = h;
            fqn_take8(h, w[c], ss, top);
        }
    } else if (!REREAD) {
        fq_v4i add[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) {                    // all requested before the first is used; past the row's end its last chunk again
            const int c = t + i * T < nchunk ? t + i * T : nchunk - 1;
            keep[i] = x[c];
            if (RES) add[i] = r[c];
            wt[i] = w[c];
        }
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (RES) keep[i] = fqn_add8(keep[i], add[i]);
            if (t + i * T >= nchunk) keep[i] = (fq_v4i){0, 0, 0, 0};
            fqn_take8(keep[i], wt[i], ss, top);
        }
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (RES && on && t + i * T < nchunk) hs[t + i * T] = keep[i];
    } else {
        for (int c = t; c < nchunk; c += T) {
            fq_v4i h = x[c];
            if (RES) {
                h = fqn_add8(h, r[c]);
                if (on) hs[c] = h;
            }
            fqn_take8(h, w[c], ss, top);
        }
    }
    ss = fqn_wave_sum(ss);
    top = fq_wave_max(top);
    if (WPR > 1) {                                        // (a workgroup is one row, or four waves of one row)
        const int wave = (int)threadIdx.x >> 6, first = row * WPR;
        if (HALVES) other = fqn_wave_sum(other);
        if ((t & 63) == 0) {
            red_sum[wave] = ss;
            if (HALVES) red_sum[WAVES + wave] = other;
            red_top[wave] = top;
        }
        __syncthreads();
        ss = red_sum[first];
        top = red_top[first];
#pragma unroll
        for (int i = 1; i < WPR; ++i) {
            ss += red_sum[first + i];
            top = red_top[first + i] > top ? red_top[first + i] : top;
        }
        if (HALVES)
#pragma unroll
            for (int i = 0; i < WPR; ++i) ss += red_sum[WAVES + i];
    }
    const float rstd = 1.0f / sqrtf(ss / (float)K + eps), tf = __uint_as_float(top), ymax = tf * rstd;
    const bool bad = !(ss < __builtin_inff()) || top >= 0x7F800000u || (OUT != FQN_BF16 && !(ymax < __builtin_inff()));
    if (OUT == FQN_BF16) {
        fq_v4i* y = reinterpret_cast<fq_v4i*>(Y + at);
        const float f = bad ? __builtin_nanf("") : rstd;
        auto put = [&](int c, fq_v4i h, fq_v4i g) __attribute__((always_inline)) {
            fq_v4i o;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                o[j] = (int)fqn_pack_bf16(fq_bf16_lo(h[j]) * f * fq_bf16_lo(g[j]), fq_bf16_hi(h[j]) * f * fq_bf16_hi(g[j]));
            y[c] = o;
        };
        if (REREAD) {
            if (on)
                for (int c = t; c < nchunk; c += T) put(c, RES ? hs[c] : x[c], w[c]);
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i)
                if (on && t + i * T < nchunk) put(t + i * T, keep[i], wt[i]);
        }
        return;
    }
    if (t == 0 && on) a_scale[m] = bad ? __builtin_nanf("") : top == 0u ? 1.0f : ymax / 448.0f;
    fq_v2i* a = reinterpret_cast<fq_v2i*>(A + at);
    // h w is exact in FP32 (8 bits each); 448 h w / t by one exact residual step behind h w * (448 / t), as a correctly rounded quotient.
    // Rows whose t lies outside [2^-100, 2^110] divide by t first: 448 / t or 448 h w may pass FP32's range there.
    const float mul = bad || top == 0u ? 0.f : 448.0f / tf, rt = bad || top == 0u ? 0.f : 1.0f / tf;
    auto put = [&](auto tiny, int c, fq_v4i h, fq_v4i g) __attribute__((always_inline)) {
        fq_v2i o = {0, 0};
        if (!bad) {
            if constexpr (decltype(tiny)::value) o = fqn_codes8(h, g, [&](float v) { return tf > 0.f ? v / tf * 448.0f : 0.f; });
            else
                o = fqn_codes8(h, g, [&](float v) {
                    const float q = v * mul;
                    return fmaf(fmaf(q, tf, -448.0f * v), -rt, q);
                });
        }
        if (on) a[c] = o;
        if (ZP) {
            // a group is 16 consecutive chunks = 16 consecutive lanes, all here or all absent (K is a multiple of 128)
            float z = fq_row16_sum(fq_sum8(o));
            if ((t & 15) == 0) {
                z *= -0.015625f;
                const _Float16 hi = (_Float16)z, lo = (_Float16)(z - (float)hi);
                zrow[row][0][c >> 4] = __builtin_bit_cast(uint16_t, hi);
                zrow[row][1][c >> 4] = __builtin_bit_cast(uint16_t, lo);
            }
        }
    };
    auto convert = [&](auto tiny) __attribute__((always_inline)) {
        if (REREAD) {
            if (on)
                for (int c = t; c < nchunk; c += T) put(tiny, c, RES ? hs[c] : x[c], w[c]);
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i)
                if (t + i * T < nchunk) put(tiny, t + i * T, keep[i], wt[i]);
        }
    };
    if (__builtin_amdgcn_readfirstlane((int)(top != 0u && !(tf >= 0x1p-100f && tf <= 0x1p110f)))) convert(std::true_type());
    else convert(std::false_type());
    if (ZP) {
        const int G = K >> 7, C2 = 2 * ((G + 15) >> 4);
        for (int g = G + t; g < 8 * C2; g += T) zrow[row][0][g] = zrow[row][1][g] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * C2 * ROWS; i += 64 * WAVES) {
            const int rr = i % ROWS, pu = i / ROWS, plane = pu / C2, unit = pu - plane * C2, mm = blockIdx.x * ROWS + rr;
            if (mm < M)
                *reinterpret_cast<fq_v4i*>(planes + (((size_t)plane * C2 + unit) * M + mm) * 8) =
                    *reinterpret_cast<const fq_v4i*>(&zrow[rr][plane][8 * unit]);
        }
    }
}

// Waves per row and chunks per thread, us with residual from a graph, the choice here first:
//     1 x 4096      <4, 2> 2.9; <8, 1> 2.8; <2, 4> 3.3; <1, 8> 4.3      8192 x 4096   <4, 2> 42.5 (5.5 TB/s); <8, 1> 43.1; <2, 4> 43.7; <1, 8> 46.4
//     1000 x 5120   <8, 2> 8.2; <4, 3> 8.1; <4, 4> 8.5; <16, 1> 9.3     6000 x 5120   <8, 2> 39.7; <4, 3> 40.3; <4, 4> 40.5; <16, 1> 44.1
//     1000 x 8192   <8, 2> 10.5; <4, 4> 10.9; <16, 1> 11.7              4096 x 8192   <8, 2> 42.7; <4, 4> 43.8; <16, 1> 44.9
//     64 x 11008    <16, 2> 4.2; <8, 4> 4.4; <4, 8> 4.9                 2000 x 11008  <16, 2> 30.3; <8, 4> 29.6; <4, 8> 31.0
//     1 x 16384     <16, 2> 3.9; <8, 4> 4.1; <4, 8> 4.6                 2048 x 16384  <16, 2> 44.9; <8, 4> 45.0; <4, 8> 45.8
//     8192 x 2048   <1, 4> 21.1 and 8192 x 1024 11.8 (one wave a row); 300 x 2048 <4, 2> 3.5; <2, 4> 3.6; <1, 8> 4.5
template <bool RES, int OUT, class BR>
void fqn_launch(const uint16_t* X, const uint16_t* R, const uint16_t* W, float eps, uint16_t* H, uint16_t* Y, uint8_t* A, float* a_scale,
                int M, int K, uint16_t* planes, const BR& branch, hipStream_t stream) {
    constexpr bool BRANCH = std::is_same<BR, fq_norm_branch>::value;
#define FQN_LAUNCH(WPR_, CH_, REREAD_) \
    hipLaunchKernelGGL((fqn_kernel<WPR_, CH_, RES, OUT, REREAD_, BRANCH>), dim3((unsigned)((M + (WPR_ > 4 ? 1 : 4 / WPR_) - 1) / (WPR_ > 4 ? 1 : 4 / WPR_))), \
                       dim3(WPR_ > 4 ? 64 * WPR_ : 256), 0, stream, X, R, W, eps, H, Y, A, a_scale, K, planes, M, branch)
    if (K > 16384) {
        if constexpr (OUT != FQN_CODES_ZP) {              // (no zero-point terms for rows this long)
            // (row, residual and weights of more than 32768 numbers do not fit the registers where bf16 leaves: 512 x 40960
            // 68.3 us held, 40.2 read twice; the codes' kernel 33.5 held, 36.0 read twice)
            constexpr int HELD = BRANCH || (RES && OUT == FQN_BF16) ? 32768 : 65536;
            if (K > HELD) FQN_LAUNCH(16, 1, true);
            else if constexpr (HELD > 32768) {
                if (K > 32768) FQN_LAUNCH(16, 8, false);
                else FQN_LAUNCH(16, 4, false);
            }
            else FQN_LAUNCH(16, 4, false);
        }
    } else if (BRANCH && K > 8192) {
        // (fewer waves of a row, and of the two sums that the branch needs: us, the choice here first, then the plain forms': 1000 x 5120 <4, 3> 10.1,
        // <8, 2> 11.5; 8192 x 5120 to E4M3 55, 65; 4096 x 10240 <8, 3> 72, <16, 2> 103; 1000 x 16384 <8, 4> 23, 31; up to 8192 numbers <8, 2> is as fast
        // as <4, 4>: 1000 x 8192 13.6, 13.3; 16 x 8192 4.1, 4.3)
        if constexpr (BRANCH) {
            if (K > 12288) FQN_LAUNCH(8, 4, false);
            else FQN_LAUNCH(8, 3, false);
        }
    } else if (K > 8192) FQN_LAUNCH(16, 2, false);
    else if (BRANCH && K > 4096 && K <= 6144) {
        if constexpr (BRANCH) FQN_LAUNCH(4, 3, false);
    } else if (K > 4096) FQN_LAUNCH(8, 2, false);
    else if (K > 2048 || M <= 1536) FQN_LAUNCH(4, 2, false);
    else FQN_LAUNCH(1, 4, false);
#undef FQN_LAUNCH
}

}  // namespace

void fq_launch_rmsnorm(const uint16_t* X, const uint16_t* R, const uint16_t* W, float eps, uint16_t* H, uint16_t* Y, int M, int K,
                       hipStream_t stream) {
    if (R) fqn_launch<true, FQN_BF16>(X, R, W, eps, H, Y, nullptr, nullptr, M, K, nullptr, fqn_none(), stream);
    else fqn_launch<false, FQN_BF16>(X, nullptr, W, eps, nullptr, Y, nullptr, nullptr, M, K, nullptr, fqn_none(), stream);
}

void fq_launch_rmsnorm_quant(const uint16_t* X, const uint16_t* R, const uint16_t* W, float eps, uint16_t* H, uint8_t* A, float* a_scale,
                             int M, int K, void* workspace, hipStream_t stream) {
    uint16_t* planes = static_cast<uint16_t*>(workspace);
    if (planes) {
        if (R) fqn_launch<true, FQN_CODES_ZP>(X, R, W, eps, H, nullptr, A, a_scale, M, K, planes, fqn_none(), stream);
        else fqn_launch<false, FQN_CODES_ZP>(X, nullptr, W, eps, nullptr, nullptr, A, a_scale, M, K, planes, fqn_none(), stream);
    } else {
        if (R) fqn_launch<true, FQN_CODES>(X, R, W, eps, H, nullptr, A, a_scale, M, K, nullptr, fqn_none(), stream);
        else fqn_launch<false, FQN_CODES>(X, nullptr, W, eps, nullptr, nullptr, A, a_scale, M, K, nullptr, fqn_none(), stream);
    }
}

void fq_launch_rmsnorm_block(const uint16_t* X, const fq_norm_branch& branch, const uint16_t* R, const uint16_t* W, float eps, uint16_t* H, uint16_t* Y,
                             uint8_t* A, float* a_scale, int M, int K, void* workspace, hipStream_t stream) {
    uint16_t* planes = static_cast<uint16_t*>(workspace);
    if (Y) fqn_launch<true, FQN_BF16>(X, R, W, eps, H, Y, nullptr, nullptr, M, K, nullptr, branch, stream);
    else if (planes) fqn_launch<true, FQN_CODES_ZP>(X, R, W, eps, H, nullptr, A, a_scale, M, K, planes, branch, stream);
    else fqn_launch<true, FQN_CODES>(X, R, W, eps, H, nullptr, A, a_scale, M, K, nullptr, branch, stream);
}
