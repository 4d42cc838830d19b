// Filling and reading a paged INT4 key/value cache (include/fireq_paged.h holds the layout and the definition).
//
// The rotation of a pair, a c - b s and b c + a s, has bf16 a and b and FP32 c and s: the products are exact in FP64 and the
// difference is rounded there once, then to FP32.  In FP32 the two products' own roundings would leave a code to the order of the
// operations wherever a key lies next to the border between two codes.
#include "fq_common.h"
#include "fq_kernels.h"

namespace {

typedef unsigned fqp_v2u __attribute__((ext_vector_type(2)));

// The largest value of 16 neighbouring lanes as a bit pattern (NaN above all numbers), in each of them.
__device__ __forceinline__ unsigned fqp_absmax(const float x[8]) {
    unsigned top = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned p = __float_as_uint(x[i]) & 0x7FFFFFFFu;
        top = p > top ? p : top;
    }
    return fq_row16_max(top);
}

// byte of token i (0..3) in a word of value codes
__device__ __forceinline__ int fqp_value_byte(int i) { return ((i & 1) << 1) | (i >> 1); }

// sixteen lanes per head: lane j holds dimensions 4 j .. 4 j + 3 and 64 + 4 j .. (x[0..3], x[4..7]), or 8 j .. 8 j + 7 (interleaved)
template <bool INTERLEAVED>
__global__ __launch_bounds__(256) void fqp_append_kernel(const uint16_t* __restrict__ QKV, long long ld, const float* __restrict__ cos_sin,
                                                         int max_positions, const int32_t* __restrict__ positions,
                                                         const int64_t* __restrict__ slots, uint8_t* __restrict__ Q,
                                                         float* __restrict__ q_scale, fq_paged_cache c, long long units, int Hq, int Hkv) {
    const int heads = Hq + 2 * Hkv, j = threadIdx.x & 15;
    const long long unit = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (unit >= units) return;
    const int token = (int)(unit / heads), head = (int)(unit % heads);
    const uint16_t* src = QKV + token * ld + head * 128;
    const bool rotated = head < Hq + Hkv, mixed = INTERLEAVED && rotated;
    fqp_v2u w[2];
    w[0] = *reinterpret_cast<const fqp_v2u*>(src + (mixed ? 8 * j : 4 * j));
    w[1] = *reinterpret_cast<const fqp_v2u*>(src + (mixed ? 8 * j + 4 : 64 + 4 * j));
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = fq_bf16_lo(w[i >> 1][i & 1]);
        x[2 * i + 1] = fq_bf16_hi(w[i >> 1][i & 1]);
    }
    const int pos = positions[token];
    const int64_t slot = slots[token];
    const bool lost = slot >= (int64_t)c.pages * c.page, bad = pos < 0 || pos >= max_positions || lost;
    if (rotated && !bad) {
        const fq_v4f* cs = reinterpret_cast<const fq_v4f*>(cos_sin + ((size_t)pos * 64 + 4 * j) * 2);
        const fq_v4f t[2] = {cs[0], cs[1]};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double cc = t[i >> 1][2 * (i & 1)], ss = t[i >> 1][2 * (i & 1) + 1];
            const int ia = INTERLEAVED ? 2 * i : i, ib = INTERLEAVED ? 2 * i + 1 : 4 + i;
            const double a = x[ia], b = x[ib];
            x[ia] = (float)(a * cc - b * ss);
            x[ib] = (float)(b * cc + a * ss);
        }
    }
    const unsigned top = fqp_absmax(x);
    const bool broken = bad || top >= 0x7F800000u;
    const float amax = __uint_as_float(top);
    if (head < Hq) {
        const size_t at = (size_t)token * Hq + head;
        const float s = broken ? __builtin_nanf("") : top == 0u ? 1.0f : amax / 448.0f;
        if (j == 0) q_scale[at] = s;
        unsigned o[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) q[k] = broken ? 0.f : fminf(fmaxf(x[4 * i + k] / s, -448.f), 448.f);
            int r = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
            o[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], r, true);
        }
        uint8_t* dst = Q + at * 128;
        *reinterpret_cast<unsigned*>(dst + (INTERLEAVED ? 8 * j : 4 * j)) = o[0];
        *reinterpret_cast<unsigned*>(dst + (INTERLEAVED ? 8 * j + 4 : 64 + 4 * j)) = o[1];
        return;
    }
    if (slot < 0 || lost) return;
    const bool value = head >= Hq + Hkv;
    // sigma, and the codes as bytes: cb[0] of x[0..3], cb[1] of x[4..7]
    const int sc = __builtin_amdgcn_cvt_pk_fp8_f32(broken ? 0.f : fminf(amax / 7.0f, 448.0f), 0.f, 0, false) & 0xFF;
    const float sigma = fq_e4m3_to_float((unsigned)sc);
    unsigned cb[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = broken || sc == 0 ? 0.f : fminf(fmaxf(rintf(x[i] / sigma), -8.f), 7.f);
        cb[i >> 2] |= (unsigned)((int)q + 8) << (8 * (i & 3));
    }
    const int t = (int)(slot % c.page);
    uint8_t* tile = c.base + (slot / c.page) * c.page_stride + (head - (value ? Hq + Hkv : Hq)) * c.head_stride + (size_t)(t >> 4) * FQP_TILE;
    const int in = t & 15;
    if (j == 0) tile[2048 + 8 * (in >> 2) + (in & 3) + (value ? 4 : 0)] = broken ? 0x7F : (uint8_t)sc;
    // A byte pairs dimensions d (low nibble) and d + 16: both words change lanes so that every lane has four whole bytes.
    if (mixed) {
        // lane j: 8 j .. 8 j + 7, its partner j ^ 2 the same 16 on or back; a lane with j & 2 keeps the upper four
        const unsigned got = (unsigned)__shfl_xor((int)((j & 2) ? cb[0] : cb[1]), 2, 16);
        const unsigned lo = (j & 2) ? got : cb[0], hi = (j & 2) ? cb[1] : got;
        *reinterpret_cast<unsigned*>(tile + 256 * (j >> 2) + 16 * in + 8 * (j & 1) + ((j & 2) ? 4 : 0)) = lo | (hi << 4);
        return;
    }
    // lane j: 4 j .. and 64 + 4 j .., its partner j ^ 4 the same 16 on or back; a lane with j & 4 keeps the upper half
    const unsigned got = (unsigned)__shfl_xor((int)((j & 4) ? cb[0] : cb[1]), 4, 16);
    const unsigned pair = (j & 4) ? (got | (cb[1] << 4)) : (cb[0] | (got << 4));
    const int g = (j >> 3) + ((j & 4) ? 2 : 0), d = 4 * (j & 3);
    if (!value) {
        *reinterpret_cast<unsigned*>(tile + 256 * g + 16 * in + d) = pair;
    } else {
        uint8_t* v = tile + 1024 + 256 * (in >> 2) + 4 * g + fqp_value_byte(in & 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[16 * (d + i)] = (uint8_t)(pair >> (8 * i));
    }
}

// sixteen lanes per token and head, eight dimensions each
__global__ __launch_bounds__(256) void fqp_read_kernel(fq_paged_cache c, const int64_t* __restrict__ slots, uint16_t* __restrict__ K,
                                                       uint16_t* __restrict__ V, long long units, int Hkv) {
    const int j = threadIdx.x & 15;
    const long long unit = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (unit >= units) return;
    const int64_t slot = slots[unit / Hkv];
    fq_v4i k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
    if (slot >= (int64_t)c.pages * c.page) {
        k = v = (fq_v4i){0x7FC07FC0, 0x7FC07FC0, 0x7FC07FC0, 0x7FC07FC0};
    } else if (slot >= 0) {
        const int t = (int)(slot % c.page), in = t & 15;
        const uint8_t* tile = c.base + (slot / c.page) * c.page_stride + (unit % Hkv) * c.head_stride + (size_t)(t >> 4) * FQP_TILE;
        const uint8_t* sc = tile + 2048 + 8 * (in >> 2) + (in & 3);
        const float ks = fq_e4m3_to_float(sc[0]), vs = fq_e4m3_to_float(sc[4]);
        // dimensions 8 j .. : group j / 4, nibble (j & 2) / 2, bytes 8 (j & 1) ..
        const int sh = 4 * ((j & 2) >> 1);
        const fqp_v2u kw = *reinterpret_cast<const fqp_v2u*>(tile + 256 * (j >> 2) + 16 * in + 8 * (j & 1));
        const uint8_t* vb = tile + 1024 + 256 * (in >> 2) + 128 * (j & 1) + 4 * (j >> 2) + fqp_value_byte(in & 3);
        const bool kn = (sc[0] & 0x7F) == 0x7F, vn = (sc[4] & 0x7F) == 0x7F;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a[2], b[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const unsigned kc = (kw[i >> 1] >> (8 * (2 * (i & 1) + e) + sh)) & 15u, vc = (vb[16 * (2 * i + e)] >> sh) & 15u;
                a[e] = (float)((int)kc - 8) * ks;
                b[e] = (float)((int)vc - 8) * vs;
            }
            k[i] = kn ? 0x7FC07FC0 : (int)((__float_as_uint(a[0]) >> 16) | (__float_as_uint(a[1]) & 0xFFFF0000u));
            v[i] = vn ? 0x7FC07FC0 : (int)((__float_as_uint(b[0]) >> 16) | (__float_as_uint(b[1]) & 0xFFFF0000u));
        }
    }
    *reinterpret_cast<fq_v4i*>(K + unit * 128 + 8 * j) = k;
    *reinterpret_cast<fq_v4i*>(V + unit * 128 + 8 * j) = v;
}

}  // namespace

void fq_launch_kv4_append(const uint16_t* QKV, long long ld, const float* cos_sin, int max_positions, const int32_t* positions,
                          const int64_t* slots, bool interleaved, uint8_t* Q, float* q_scale, const fq_paged_cache& c, int T, int Hq,
                          int Hkv, hipStream_t stream) {
    const long long units = (long long)T * (Hq + 2 * Hkv);
    const dim3 grid((unsigned)((units + 15) / 16));
    if (interleaved)
        hipLaunchKernelGGL((fqp_append_kernel<true>), grid, dim3(256), 0, stream, QKV, ld, cos_sin, max_positions, positions, slots, Q, q_scale, c, units, Hq, Hkv);
    else
        hipLaunchKernelGGL((fqp_append_kernel<false>), grid, dim3(256), 0, stream, QKV, ld, cos_sin, max_positions, positions, slots, Q, q_scale, c, units, Hq, Hkv);
}

void fq_launch_kv4_read(const fq_paged_cache& c, const int64_t* slots, uint16_t* K, uint16_t* V, int n, int Hkv, hipStream_t stream) {
    const long long units = (long long)n * Hkv;
    hipLaunchKernelGGL(fqp_read_kernel, dim3((unsigned)((units + 15) / 16)), dim3(256), 0, stream, c, slots, K, V, units, Hkv);
}
