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

// Where slot s of a cache lies: its page's first byte (of head 0) and its tile and token.  (Tiles of a cache are counted in 32 bits.)
struct fqp_place { long long at; unsigned tile, in; };
__device__ __forceinline__ fqp_place fqp_find(const fq_paged_cache& c, int64_t slot) {
    const unsigned tiles = (unsigned)c.page >> 4, n = (unsigned)(slot >> 4), page = n / tiles;
    return {(long long)page * c.page_stride, n - page * tiles, (unsigned)slot & 15u};
}

// Short quotients (tests/host/paged_quotient_check.c: the codes and scales are those of IEEE divisions).  x / s with the hardware's estimate r of
// 1 / s: one exact residual step behind x * r.  m / N with the constant c = fp32(1 / N): the same, and the IEEE quotient itself.
__device__ __forceinline__ float fqp_quotient(float x, float s, float r) {
    const float q = x * r;
    return fmaf(fmaf(q, s, -x), -r, q);
}
template <int N>
__device__ __forceinline__ float fqp_over(float m) {
    const float c = 1.0f / (float)N, q = m * c;
    return fmaf(fmaf(-(float)N, q, m), c, q);
}

// A row (token) per workgroup, sixteen lanes per head, each for two heads (their loads are all requested first; the rotation of
// the row is loaded once).  Bound by HBM and the vector instructions about alike: 6001 tokens x (32 + 8 + 8) heads (113 MB) 26.9 us (4.2 TB/s);
// 28.9 with IEEE divisions for the scales, 40.4 with them for every code, a head per lane and rows on any XCD.  Lane j holds dimensions 4 j .. 4 j + 3 and 64 + 4 j .. (x[0..3], x[4..7]), or 8 j .. 8 j + 7 (interleaved).
struct fqp_append_args {
    const uint16_t* QKV;
    long long ld;
    const float* cos_sin;
    const int32_t* positions;
    const int64_t* slots;
    uint8_t* Q;
    float* q_scale;
    fq_paged_cache c;
    int max_positions, T, Hq, Hkv;
};
template <bool INTERLEAVED>
__device__ __forceinline__ void fqp_append_head(const fqp_append_args& a, int token, int head, float (&x)[8], const double (&cs)[4], const double (&sn)[4],
                                                bool bad, bool cached, const fqp_place& place, int j) {
    const bool rotated = head < a.Hq + a.Hkv, mixed = INTERLEAVED && rotated;
    if (rotated) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int ia = INTERLEAVED ? 2 * i : i, ib = INTERLEAVED ? 2 * i + 1 : 4 + i;
            const double p = x[ia], q = x[ib];
            x[ia] = (float)(p * cs[i] - q * sn[i]);
            x[ib] = (float)(q * cs[i] + p * sn[i]);
        }
    }
    const unsigned top = fqp_absmax(x);
    const bool broken = bad || top >= 0x7F800000u;
    const float amax = __uint_as_float(top);
    if (head < a.Hq) {
        const size_t at = (size_t)token * a.Hq + head;
        const bool plain = amax >= 0x1p-50f && amax <= 0x1p60f && !broken;   // (everything stays in FP32's normal range)
        const float s = top == 0u ? 1.0f : plain ? fqp_over<448>(amax) : amax / 448.0f;
        if (j == 0) a.q_scale[at] = broken ? __builtin_nanf("") : s;
        unsigned o[2] = {0u, 0u};
        if (plain) {
            const float r = __builtin_amdgcn_rcpf(s);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int w = __builtin_amdgcn_cvt_pk_fp8_f32(fqp_quotient(x[4 * i], s, r), fqp_quotient(x[4 * i + 1], s, r), 0, false);
                o[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(fqp_quotient(x[4 * i + 2], s, r), fqp_quotient(x[4 * i + 3], s, r), w, true);
            }
        } else if (!broken) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float q[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) q[k] = fminf(fmaxf(x[4 * i + k] / s, -448.f), 448.f);
                const int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
                o[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
            }
        }
        uint8_t* dst = a.Q + at * 128;
        if (INTERLEAVED) {
            *reinterpret_cast<fqp_v2u*>(dst + 8 * j) = (fqp_v2u){o[0], o[1]};
        } else {
            *reinterpret_cast<unsigned*>(dst + 4 * j) = o[0];
            *reinterpret_cast<unsigned*>(dst + 64 + 4 * j) = o[1];
        }
        return;
    }
    if (!cached) return;
    const bool value = head >= a.Hq + a.Hkv;
    // sigma, and the codes as bytes: cb[0] of x[0..3], cb[1] of x[4..7]
    const int sc = __builtin_amdgcn_cvt_pk_fp8_f32(broken ? 0.f : fminf(fqp_over<7>(amax), 448.0f), 0.f, 0, false) & 0xFF;
    const float sigma = __builtin_amdgcn_cvt_f32_fp8(sc, 0), r = __builtin_amdgcn_rcpf(sigma);
    unsigned cb[2] = {0x08080808u, 0x08080808u};
    if (!broken && sc != 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            unsigned n[4];                                // the code in the low bits: 1.5 * 2^23 + 8 + code, rounded to nearest even
#pragma unroll
            for (int i = 0; i < 4; ++i)
                n[i] = __float_as_uint(__builtin_amdgcn_fmed3f(fqp_quotient(x[4 * h + i], sigma, r), -8.f, 7.f) + 12582920.0f);
            cb[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(n[3], n[2], 0x0C0C0400u), __builtin_amdgcn_perm(n[1], n[0], 0x0C0C0400u), 0x05040100u) & 0x0F0F0F0Fu;
        }
    }
    const int in = (int)place.in;
    uint8_t* tile = a.c.base + place.at + (head - (value ? a.Hq + a.Hkv : a.Hq)) * a.c.head_stride + (size_t)place.tile * FQP_TILE;
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

// Workgroup i runs on XCD i % 8: 16 rows that follow each other (a tile of a prompt, if it begins with one) go to one XCD, so that the
// pieces of a cache line that they write meet in its L2.
__device__ __forceinline__ int fqp_row_of(int i, int rows) {
    const int whole = rows & ~127;
    return i < whole ? (i & ~127) + (i & 7) * 16 + ((i >> 3) & 15) : i;
}

template <bool INTERLEAVED>
__global__ __launch_bounds__(512) void fqp_append_kernel(fqp_append_args a) {
    const int heads = a.Hq + 2 * a.Hkv, j = threadIdx.x & 15, token = fqp_row_of(blockIdx.x, a.T);
    const int groups = (int)(blockDim.x >> 4), h0 = (int)blockIdx.y * 2 * groups + (int)(threadIdx.x >> 4), h1 = h0 + groups;
    const uint16_t* src = a.QKV + (long long)token * a.ld;
    fqp_v2u w[2][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int h = u ? h1 : h0, hh = h < heads ? h : heads - 1;
        const bool mixed = INTERLEAVED && hh < a.Hq + a.Hkv;
        w[u][0] = *reinterpret_cast<const fqp_v2u*>(src + hh * 128 + (mixed ? 8 * j : 4 * j));
        w[u][1] = *reinterpret_cast<const fqp_v2u*>(src + hh * 128 + (mixed ? 8 * j + 4 : 64 + 4 * j));
    }
    const int pos = a.positions[token];
    const int64_t slot = a.slots[token];
    const bool lost = slot >= (int64_t)a.c.pages * a.c.page, bad = pos < 0 || pos >= a.max_positions || lost, cached = slot >= 0 && !lost;
    double cs[4] = {1., 1., 1., 1.}, sn[4] = {0., 0., 0., 0.};
    if (!bad) {
        const fq_v4f* t = reinterpret_cast<const fq_v4f*>(a.cos_sin + ((size_t)pos * 64 + 4 * j) * 2);
        const fq_v4f t0 = t[0], t1 = t[1];
        cs[0] = t0[0]; sn[0] = t0[1]; cs[1] = t0[2]; sn[1] = t0[3];
        cs[2] = t1[0]; sn[2] = t1[1]; cs[3] = t1[2]; sn[3] = t1[3];
    }
    const fqp_place place = fqp_find(a.c, cached ? slot : 0);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int h = u ? h1 : h0;
        if (h >= heads) break;
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = fq_bf16_lo(w[u][i >> 1][i & 1]);
            x[2 * i + 1] = fq_bf16_hi(w[u][i >> 1][i & 1]);
        }
        fqp_append_head<INTERLEAVED>(a, token, h, x, cs, sn, bad, cached, place, j);
    }
}

// Sixteen lanes per token and head.  Lane j reads, of the key, bytes 8 (j & 1) .. of group j / 4 and keeps one nibble of each: dimensions 8 j ..;
// of the value, the words of n = j (all of the quad's four tokens): channels j + 16 i, which change lanes through LDS to be
// eight neighbours too.  Workgroups that follow each other run on one XCD in runs of 16, for the tokens of a tile share its lines.
// Bound by HBM and the latency of slot, tile and store one after the other: 5000 tokens x 8 heads (26 MB) 7.2 us (3.6 TB/s); 8.5 without the
// runs, 9.7 with a byte load per value code; two or four heads per lane 7.3 and 8.8.
__global__ __launch_bounds__(256) void fqp_read_kernel(fq_paged_cache c, const int64_t* __restrict__ slots, uint16_t* __restrict__ K,
                                                       uint16_t* __restrict__ V, unsigned units, unsigned Hkv) {
    __shared__ __attribute__((aligned(16))) uint16_t turn[16][136];
    const int j = threadIdx.x & 15, own = threadIdx.x >> 4;
    const unsigned unit = (unsigned)fqp_row_of(blockIdx.x, gridDim.x) * 16u + (unsigned)own;
    if (unit >= units) return;                            // (sixteen lanes of a wave at a time; no barrier behind)
    const unsigned token = unit / Hkv, head = unit - token * Hkv;
    const int64_t slot = slots[token];
    const bool lost = slot >= (int64_t)c.pages * c.page;
    fq_v4i k, v;
    if (slot >= 0 && !lost) {
        const fqp_place place = fqp_find(c, slot);
        const int in = (int)place.in;
        const uint8_t* tile = c.base + place.at + head * c.head_stride + (size_t)place.tile * FQP_TILE;
        const fqp_v2u kw = *reinterpret_cast<const fqp_v2u*>(tile + 256 * (j >> 2) + 16 * in + 8 * (j & 1));
        const fq_v4i vw = *reinterpret_cast<const fq_v4i*>(tile + 1024 + 256 * (in >> 2) + 16 * j);
        const fqp_v2u sc = *reinterpret_cast<const fqp_v2u*>(tile + 2048 + 8 * (in >> 2));
        // (a NaN scale's products are NaN in bf16)
        const float ks = __builtin_amdgcn_cvt_f32_fp8((int)(sc[0] >> (8 * (in & 3))), 0), vs = __builtin_amdgcn_cvt_f32_fp8((int)(sc[1] >> (8 * (in & 3))), 0);
        const int sh = 2 * (j & 2), vb = 8 * fqp_value_byte(in & 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned kb = kw[i >> 1] >> (16 * (i & 1) + sh), b = (unsigned)vw[i] >> vb;
            const float k0 = (float)((int)(kb & 15u) - 8) * ks, k1 = (float)((int)((kb >> 8) & 15u) - 8) * ks;
            const float v0 = (float)((int)(b & 15u) - 8) * vs, v1 = (float)((int)((b >> 4) & 15u) - 8) * vs;
            k[i] = (int)((__float_as_uint(k0) >> 16) | (__float_as_uint(k1) & 0xFFFF0000u));
            turn[own][32 * i + j] = (uint16_t)(__float_as_uint(v0) >> 16);
            turn[own][32 * i + 16 + j] = (uint16_t)(__float_as_uint(v1) >> 16);
        }
        // (other lanes' values are read back: a wave's own LDS accesses stay in order, which the fence holds the compiler to)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        v = *reinterpret_cast<const fq_v4i*>(&turn[own][8 * j]);
    } else {
        const int z = lost ? 0x7FC07FC0 : 0;
        k = v = (fq_v4i){z, z, z, z};
    }
    *reinterpret_cast<fq_v4i*>(K + (size_t)unit * 128 + 8 * j) = k;
    *reinterpret_cast<fq_v4i*>(V + (size_t)unit * 128 + 8 * j) = v;
}

}  // namespace

void fq_launch_kv4_append(const uint16_t* QKV, long long ld, const float* cos_sin, int max_positions, const int32_t* positions,
                          const int64_t* slots, bool interleaved, uint8_t* Q, float* q_scale, const fq_paged_cache& c, int T, int Hq,
                          int Hkv, hipStream_t stream) {
    const int heads = Hq + 2 * Hkv, pairs = (heads + 1) / 2, groups = pairs < 32 ? (pairs + 3) / 4 * 4 : 32;
    const dim3 grid((unsigned)T, (unsigned)((pairs + groups - 1) / groups)), block((unsigned)(16 * groups));
    const fqp_append_args a = {QKV, ld, cos_sin, positions, slots, Q, q_scale, c, max_positions, T, Hq, Hkv};
    if (interleaved) hipLaunchKernelGGL((fqp_append_kernel<true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((fqp_append_kernel<false>), grid, block, 0, stream, a);
}

void fq_launch_kv4_read(const fq_paged_cache& c, const int64_t* slots, uint16_t* K, uint16_t* V, int n, int Hkv, hipStream_t stream) {
    const unsigned units = (unsigned)n * (unsigned)Hkv;
    hipLaunchKernelGGL(fqp_read_kernel, dim3((units + 15) / 16), dim3(256), 0, stream, c, slots, K, V, units, (unsigned)Hkv);
}
