// What the attention kernels over the paged INT4 cache share (fq_attend.hip: one token per sequence; fq_chunk.hip: any number of them): a
// query tile's operands, unpacked values, and the parts of a row that meet through memory.  The mathematics stands in fq_attend.hip.
#pragma once
#include "fq_common.h"
#include "fq_kernels.h"

namespace {

typedef _Float16 fqa_v8h __attribute__((ext_vector_type(8)));
typedef _Float16 fqa_v2h __attribute__((ext_vector_type(2)));

#define FQA_LIFT 7.0f                                     // log2 of the factor on the probabilities: down to 2^-31 above fp16's smallest
#define FQA_SLACK 6.0f                                    // ... and 2^(7 + 6) is the largest

#define FQA_MFMA_QK(a, b, c) __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4((a), (b), (c), 0, 0, 0, 0, 0, 0)

__device__ __forceinline__ float fqa_over_groups_max(float v) {   // over the four lanes of a query
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
// The lane's values for channel j of 16 (word j / 2 of each of two tiles) as eight fp16 numbers sigma * (code - 8): a word holds, for j
// even and odd, nibbles 0 / 1 (tokens 0, 1 of four) and 2 / 3 (tokens 2, 3) of both halves.  `mask` and `base` are 0x03C003C0 and
// 0x4C004C00 held in registers, for one and-or instead of an and and an or with a literal each.
struct fqa_sigmas { fqa_v2h s[2], n[2]; };                // sigma and -24 sigma of tokens 0, 1 and 2, 3
__device__ __forceinline__ fqa_v2h fqa_value_pair(unsigned w, unsigned mask, unsigned base, fqa_v2h s, fqa_v2h n) {
    return __builtin_elementwise_fma(__builtin_bit_cast(fqa_v2h, (w & mask) | base), s, n);
}
template <int ODD>
__device__ __forceinline__ fqa_v8h fqa_values(int w0, int w1, unsigned mask, unsigned base, const fqa_sigmas& a, const fqa_sigmas& b) {
    const unsigned x = (unsigned)w0, y = (unsigned)w1;
    const fqa_v2h r0 = fqa_value_pair(ODD ? x << 2 : x << 6, mask, base, a.s[0], a.n[0]), r1 = fqa_value_pair(ODD ? x >> 6 : x >> 2, mask, base, a.s[1], a.n[1]);
    const fqa_v2h r2 = fqa_value_pair(ODD ? y << 2 : y << 6, mask, base, b.s[0], b.n[0]), r3 = fqa_value_pair(ODD ? y >> 6 : y >> 2, mask, base, b.s[1], b.n[1]);
    return (fqa_v8h){r0[0], r0[1], r1[0], r1[1], r2[0], r2[1], r3[0], r3[1]};
}

struct fqa_tile { fq_v4i k, v; fq_v2i s; };

#define FQA_LOWEST (-3.0e38f)                             // below every score, and finite: times a scale of 0 it is 0

// A query tile's state.  Scores are kept before the query's factor: s = sum q k * sigma_k, probability 2^(qs * (s - m)).
template <int RT>
struct fqa_state {
    float m[RT], sub[RT];                                 // the reference score (within the slack of the largest so far), LIFT - qs * m
    fq_v4f o[RT][8], l[RT];                               // O^T; sum p, the same in all four
};

template <int RT>
struct fqa_queries {
    fq_v8i q[RT];                                         // codes, as the B operand
    fq_v4f zp[RT];                                        // -2^-6 sum of the codes
    float qs[RT];                                         // factor of a score in log2, not negative
};

// One query (16 lanes of a query tile: 32 bytes each): a negative factor turns the codes' signs instead.
template <int RT>
__device__ __forceinline__ void fqa_take_query(fqa_queries<RT>& Q, int r, const uint8_t* codes, float scale, float out_scale, int g) {
    const fq_v4i* p = reinterpret_cast<const fq_v4i*>(codes + 32 * g);
    const fq_v4i a = p[0], b = p[1];
    const int flip = scale < 0.f ? (int)0x80808080 : 0;
    Q.q[r] = (fq_v8i){a[0] ^ flip, a[1] ^ flip, a[2] ^ flip, a[3] ^ flip, b[0] ^ flip, b[1] ^ flip, b[2] ^ flip, b[3] ^ flip};
    Q.qs[r] = fabsf(scale) * out_scale * (512.0f * 1.44269504088896340736f);
    constexpr int E = (int)FQ_ZP_BYTES;
    const fq_v8i eights = {E, E, E, E, E, E, E, E};
    Q.zp[r] = FQA_MFMA_QK(eights, Q.q[r], ((fq_v4f){0.f, 0.f, 0.f, 0.f}));
}

// What the waves of a workgroup join through LDS.
template <int RT, int WAVES>
struct __attribute__((aligned(16))) fqa_shared {
    float o[WAVES][16 * RT][132], m[WAVES][16 * RT], l[WAVES][16 * RT];
};

// Parts of a row (query head of a sequence), one behind the other: 128 sums and, apart from them, (maximum, sum).
struct fqa_parts {
    float* o;                                             // [B * Hq][slots][128]
    float* ml;                                            // [B * Hq][slots][2]
    int slots;
};

// Parts first, first + STEP, .. of n of a row added to (m, l, o), four requested at a time (po: at the lane's four channels).
template <int STEP>
__device__ __forceinline__ void fqa_add_parts(const fq_v2f* ml, const fq_v4f* po, int first, int n, float& m, float& l, fq_v4f& o) {
    for (int s0 = first; s0 < n; s0 += 4 * STEP) {
        fq_v2f pm[4];
        fq_v4f x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int s = s0 + STEP * u < n ? s0 + STEP * u : s0;
            pm[u] = ml[s];
            x[u] = po[(size_t)s * 32];
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (s0 + STEP * u >= n) pm[u][1] = 0.f;
            if (pm[u][1] != 0.f) top = fmaxf(top, pm[u][0]);   // (an empty part has no sums)
        }
        const float f = __builtin_amdgcn_exp2f(m - top);
        l *= f;
        o *= f;
        m = top;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (pm[u][1] == 0.f) continue;
            const float fu = __builtin_amdgcn_exp2f(pm[u][0] - top);
            l += pm[u][1] * fu;
            o += x[u] * fu;
        }
    }
}

// o / l as four bf16 (a row without tokens: zeros).
__device__ __forceinline__ uint2 fqa_output(fq_v4f o, float l) {
    o *= l == 0.f ? 0.f : 1.0f / l;
    uint2 out;
    out.x = __builtin_bit_cast(unsigned, __builtin_convertvector((fq_v2f){o[0], o[1]}, fq_v2bf));
    out.y = __builtin_bit_cast(unsigned, __builtin_convertvector((fq_v2f){o[2], o[3]}, fq_v2bf));
    return out;
}

// The parts' sums, each brought to the largest maximum.  32 lanes hold the 128 channels of a row; GROUPS of 32 lanes share its parts, four
// requested at a time.  A wave per row for up to 8 parts (no LDS, no barrier; 96 sequences behind a prefix, 32 query heads, 6 parts, the whole
// call 46.8 us, 50.1 with a workgroup each; 1 x 1000 tokens 6.9 and 7.3), a workgroup for more (12 parts 7.9 us, 8.3 with a wave; 32 parts
// 12.4 and 14.0).
template <int GROUPS>
__global__ __launch_bounds__(256) void fqa_join_kernel(fqa_parts parts, uint16_t* __restrict__ O, int rows, const int* __restrict__ starts, int B, int Hq) {
    constexpr int ROWS = 8 / GROUPS;                      // of a workgroup
    __shared__ float wm[GROUPS], wl[GROUPS];
    __shared__ fq_v4f wo[GROUPS][32];
    const int c = threadIdx.x & 31, grp = (int)(threadIdx.x >> 5) % GROUPS, n = parts.slots;
    const int row = (int)(blockIdx.y * gridDim.x + blockIdx.x) * ROWS + (int)(threadIdx.x >> 5) / GROUPS;
    if (row >= rows) return;                              // (one row a workgroup where there is a barrier)
    if (starts && (row / Hq < starts[0] || row / Hq >= starts[B])) return;   // of no sequence: it has no parts
    const fq_v2f* ml = reinterpret_cast<const fq_v2f*>(parts.ml) + (size_t)row * n;
    const fq_v4f* po = reinterpret_cast<const fq_v4f*>(parts.o) + (size_t)row * n * 32 + c;
    float m = FQA_LOWEST, l = 0.f;
    fq_v4f o = {0.f, 0.f, 0.f, 0.f};
    fqa_add_parts<GROUPS>(ml, po, grp, n, m, l, o);
    if (GROUPS == 2) {                                    // the other half of the wave
        const float top = fmaxf(m, __shfl_xor(m, 32, 64)), f = __builtin_amdgcn_exp2f(m - top);
        l *= f;
        l += __shfl_xor(l, 32, 64);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[i] *= f;
            o[i] += __shfl_xor(o[i], 32, 64);
        }
        if (grp) return;
    } else {
        if (c == 0) {
            wm[grp] = m;
            wl[grp] = l;
        }
        wo[grp][c] = o;
        __syncthreads();
        if (grp) return;
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) m = fmaxf(m, wm[i]);
        l = 0.f;
        o = (fq_v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) {
            const float f = __builtin_amdgcn_exp2f(wm[i] - m);
            l += wl[i] * f;
            o += wo[i][c] * f;
        }
    }
    reinterpret_cast<uint2*>(O)[(size_t)row * 32 + c] = fqa_output(o, l);
}

constexpr int FQA_JOIN_FEW = 8;
// starts (or NULL): only the rows of sequences, tokens starts[0] .. starts[B] of Hq rows each.
inline void fqa_join(const fqa_parts& parts, uint16_t* O, int rows, hipStream_t stream, const int* starts = nullptr, int B = 0, int Hq = 1) {
    const int most = 1 << 23, high = (rows + most - 1) / most;   // (a grid has fewer than 2^32 threads in a dimension)
    if (parts.slots <= FQA_JOIN_FEW) hipLaunchKernelGGL(fqa_join_kernel<2>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, parts, O, rows, starts, B, Hq);
    else hipLaunchKernelGGL(fqa_join_kernel<8>, dim3((unsigned)((rows + high - 1) / high), (unsigned)high), dim3(256), 0, stream, parts, O, rows, starts, B, Hq);
}

// Tiles of a part, for `heads` (sequence, key/value head, 16 query rows) of up to `tiles` each; uneven: of several sequences, whose lengths
// differ.  A wave of a part's four takes about 0.25 us a tile beyond 4; a second part costs the joining kernel, 2 us and more.  us, from a
// graph, 32 query and 8 key/value heads unless said otherwise:
//     one workgroup per compute unit           1 x 32001 tokens, parts of 64 (256 workgroups) 12.3; 32 (504) 13.4; 16 (1008) 15.0; 128 (128) 16.0
//                                              1 x 8000, 16 (256) 8.5; 32 9.4; 64 10.9     16 x 4000, 128 (256) 17.1; 64 (512) 18.4; 32 18.5
//     ... but at least 16 tiles                1 x 1000, 16 6.8; 64 8.2
//     ... and up to 64 parts                   1 x 32001, 8 / 1 heads, 32 (63 parts) 9.3; 16 (126) 9.4
//     one part of a short sequence             1 x 600, 7.0 -> 6.4;  with many heads 16 x 1000, 16 10.2; 64 9.5    30 x 700 of 32 heads 26.6 -> 20.5
//     several sequences: parts of 128 tiles or a sixteenth, for the longest may be one of few as long, and would be left to its
//     8 workgroups                             one of 32001 among 200: 8 142 (76 of 16, 42 of 8 sequences); 128 36 (34, 34) for 32 sequences
//                                              0 .. 32001: 32 sequences 152 -> 114, 24 148 -> 82     0 .. 4000: 32 22.4 -> 22.3, 17 22.3 -> 16.5
//     ... which costs even lengths that one    32 x 4000, 250 27.9; 128 30.8    32 x 32001, 2001 183; 128 201    16 x 32001, 1008 97; 128 104
//     workgroup per head suited, and not else  24 x 32001, 2001 161; 128 153    17 x 32001, 2001 154; 128 111     8 x 32001, 512 53.6; 128 55.0
//     more workgroups than compute units: short parts even out different lengths
//                                              37 x 0 .. 6000, 64 31.1; 128 35.2           128 x 0 .. 1500 (1024 heads), 94 30.0; 48 30.4
inline int fqa_part(long long heads, int tiles, long long cus, bool uneven) {
    if (tiles <= 40 || (tiles <= 64 && 2 * heads >= cus)) return tiles;
    const long long want = heads < cus ? cus / heads : 1;
    long long chunk = (tiles + want - 1) / want;
    if (chunk < (tiles + 63) / 64) chunk = (tiles + 63) / 64;
    chunk = chunk < 16 ? 16 : (chunk + 15) / 16 * 16;
    const long long few = heads < 2 * cus ? 64 : 128, longest = tiles / 16 > 128 ? tiles / 16 : 128;
    if (heads * ((tiles + chunk - 1) / chunk) > cus) chunk = chunk > few ? few : chunk;
    else if (uneven && chunk > longest) {
        const long long n = (tiles + longest - 1) / longest;
        chunk = ((tiles + n - 1) / n + 15) / 16 * 16;
    }
    if (chunk < tiles / 60000 + 1) chunk = (tiles / 60000 + 16) / 16 * 16;   // (a grid has 65535 in its second dimension; a step may not pass a part's end)
    return (int)(chunk < tiles ? chunk : tiles);
}

}  // namespace
