// Decode attention over a paged INT4 key/value cache (include/fireq_paged.h): one pass over the tokens with a running maximum and sum.
//
// A wave works on a range of 16-token tiles of one key/value head for RT * 16 query rows.  Everything is transposed, so that no
// operand changes lanes on the way:
//     S^T = K Q^T   v_mfma_f32_16x16x128_f8f6f4 per tile, A = 16 tokens (a lane's 16 bytes of codes: 32 dimensions of one token), B = 16
//                   queries.  Code + 8 as an E4M3 number is the code times 2^-9 (fq_common.h); the zero point is the same for all
//                   tokens of a query, -2^-6 sum q, and the product starts from it.
//     P^T           a lane has 4 tokens (4 g + i, g = lane / 16) of one query (lane % 16): scaled by the keys' sigmas, exponentiated against the
//                   query's maximum so far, multiplied by the values' sigmas and rounded to fp16 (11 bits; 2^7 times the probability, so
//                   that sigma * p stays below 2^16 and reaches 2^-31 of the largest).  Two tiles give the 8 fp16 numbers that a
//                   lane of the B operand of v_mfma_f32_16x16x32_f16 holds, tokens in this order on both sides.
//     O^T = V^T P^T per 16 channels.  A value's code c, shifted to the top of an fp16 mantissa under the exponent of 16, is the number
//                   16 + c: unpacking is a shift and an and-or for two of them.  24 sum p sigma (16 and the zero point) is one more
//                   such product against a constant, taken off at the end.  (As a subnormal fp16 number, c * 2^-24, it would save a
//                   shift, but the matrix cores align products by their factors' exponents, and a subnormal's is far above its value: sums came
//                   out 2^-18 off.)
// O stays in registers and is rescaled where a query's maximum has moved.
#include "fq_common.h"
#include "fq_kernels.h"

namespace {

typedef _Float16 fqa_v8h __attribute__((ext_vector_type(8)));
typedef _Float16 fqa_v2h __attribute__((ext_vector_type(2)));

#define FQA_ZERO (-__builtin_inff())
#define FQA_LIFT 7.0f                                     // log2 of the factor on the probabilities

#define FQA_MFMA_QK(a, b, c) __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4((a), (b), (c), 0, 0, 0, 0, 0, 0)

__device__ __forceinline__ float fqa_over_groups_max(float v) {   // over the four lanes of a query
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float fqa_over_groups_sum(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

// Two codes at bits 6 .. 9 of the halves -> two fp16 numbers 16 + code.
__device__ __forceinline__ int fqa_value_pair(unsigned w) { return (int)((w & 0x03C003C0u) | 0x4C004C00u); }

struct fqa_tile { fq_v4i k, v; fq_v2i s; };

// The tiles of a range one after the other: page numbers 64 at a time in a register, the tile within its page counted along.
struct fqa_cursor {
    const int* pages_of;                                  // the sequence's pages
    const uint8_t* head;                                  // the head's part of page 0
    long long page_stride;
    int last;                                             // the range's last tile
    int tile, page, within, tiles_per_page, first, pages;
    int ids;                                              // lane l: page number first + l
    bool bad;                                             // a page number outside the cache was met
    __device__ __forceinline__ void fetch(int lane) {
        const int last_page = last / tiles_per_page;
        const int p = first + lane < last_page ? first + lane : last_page;
        const int id = pages_of[p];
        const bool ok = (unsigned)id < (unsigned)pages;
        bad |= __any(!ok);
        ids = ok ? id : 0;
    }
    __device__ __forceinline__ void start(int t0, int t1, int lane) {
        tile = t0;
        last = t1 - 1;
        page = first = t0 / tiles_per_page;
        within = t0 - page * tiles_per_page;
        fetch(lane);
    }
    // the next tile's bytes; behind the range its last tile again
    __device__ __forceinline__ fqa_tile next(int lane) {
        const int id = __builtin_amdgcn_readlane(ids, page - first);
        const uint8_t* p = head + id * page_stride + within * FQP_TILE;
        fqa_tile t;
        t.k = *reinterpret_cast<const fq_v4i*>(p + 16 * lane);
        t.v = *reinterpret_cast<const fq_v4i*>(p + 1024 + 16 * lane);
        t.s = *reinterpret_cast<const fq_v2i*>(p + 2048 + 8 * (lane >> 4));
        if (tile < last) {
            ++tile;
            if (++within == tiles_per_page) {
                within = 0;
                if (++page - first == 64) {
                    first = page;
                    fetch(lane);
                }
            }
        }
        return t;
    }
};

template <int RT>
struct fqa_state {
    float m[RT], l[RT];                                   // maximum (in log2), this lane's part of the sum
    fq_v4f o[RT][8], z[RT];                               // O^T and its zero-point part
};

// Tiles t0 .. t1 of a head's tokens below `len`, NT (even) tiles a step.
template <int RT, int NT>
__device__ __forceinline__ void fqa_range(fqa_cursor& cur, int t0, int t1, int len, const fq_v8i (&q)[RT], const float (&qs)[RT],
                                          fqa_state<RT>& st, int lane) {
    const int g = lane >> 4;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        st.m[r] = FQA_ZERO;
        st.l[r] = 0.f;
        st.z[r] = (fq_v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) st.o[r][j] = (fq_v4f){0.f, 0.f, 0.f, 0.f};
    }
    fq_v4f zp[RT];
    constexpr int E = (int)FQ_ZP_BYTES;
    const fq_v8i eights = {E, E, E, E, E, E, E, E};
#pragma unroll
    for (int r = 0; r < RT; ++r) zp[r] = FQA_MFMA_QK(eights, q[r], ((fq_v4f){0.f, 0.f, 0.f, 0.f}));
    const fq_v4i offset = {0x4E004E00, 0x4E004E00, 0x4E004E00, 0x4E004E00};   // 24 in fp16
    fqa_tile buf[NT];
    cur.start(t0, t1, lane);
#pragma unroll
    for (int i = 0; i < NT; ++i) buf[i] = cur.next(lane);
    for (int tb = t0; tb < t1; tb += NT) {
        fqa_tile now[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) now[i] = buf[i];
        if (tb + NT < t1) {
#pragma unroll
            for (int i = 0; i < NT; ++i) buf[i] = cur.next(lane);
        }
        const bool tail = (tb + NT) * 16 > len;
        fq_v4f p[RT][NT];
        float vs[NT][4];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const fq_v8i a = fq_unpack_chunk(now[i].k);
            const fq_v2f s01 = __builtin_amdgcn_cvt_pk_f32_fp8(now[i].s[0], false), s23 = __builtin_amdgcn_cvt_pk_f32_fp8(now[i].s[0], true);
            const fq_v2f v01 = __builtin_amdgcn_cvt_pk_f32_fp8(now[i].s[1], false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8(now[i].s[1], true);
            const float ks[4] = {s01[0], s01[1], s23[0], s23[1]};
            vs[i][0] = v01[0]; vs[i][1] = v01[1]; vs[i][2] = v23[0]; vs[i][3] = v23[1];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const fq_v4f c = FQA_MFMA_QK(a, q[r], zp[r]);
#pragma unroll
                for (int e = 0; e < 4; ++e) p[r][i][e] = c[e] * ks[e] * qs[r];
            }
        }
        if (tail) {
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if ((tb + i) * 16 + 4 * g + e >= len) {
                        vs[i][e] = 0.f;
#pragma unroll
                        for (int r = 0; r < RT; ++r) p[r][i][e] = FQA_ZERO;
                    }
        }
        fq_v4i pt[RT][NT / 2];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = p[r][0][0];
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, p[r][i][e]);
            top = fqa_over_groups_max(top);
            if (__any(top > st.m[r])) {
                const float m = fmaxf(st.m[r], top), f = __builtin_amdgcn_exp2f(st.m[r] - m);
                st.m[r] = m;
                st.l[r] *= f;
                st.z[r] *= f;
#pragma unroll
                for (int j = 0; j < 8; ++j) st.o[r][j] *= f;
            }
            const float sub = st.m[r] - FQA_LIFT;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float a = __builtin_amdgcn_exp2f(p[r][i][e] - sub), b = __builtin_amdgcn_exp2f(p[r][i][e + 1] - sub);
                    st.l[r] += a + b;
                    pt[r][i / 2][2 * (i & 1) + e / 2] = __builtin_bit_cast(int, __builtin_convertvector((fq_v2f){a * vs[i][e], b * vs[i][e + 1]}, fqa_v2h));
                }
        }
#pragma unroll
        for (int i = 0; i < NT / 2; ++i) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
                st.z[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(fqa_v8h, offset), __builtin_bit_cast(fqa_v8h, pt[r][i]), st.z[r], 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned w0 = (unsigned)now[2 * i].v[j >> 1], w1 = (unsigned)now[2 * i + 1].v[j >> 1];
                const fq_v4i a = j & 1 ? (fq_v4i){fqa_value_pair(w0 << 2), fqa_value_pair(w0 >> 6), fqa_value_pair(w1 << 2), fqa_value_pair(w1 >> 6)}
                                       : (fq_v4i){fqa_value_pair(w0 << 6), fqa_value_pair(w0 >> 2), fqa_value_pair(w1 << 6), fqa_value_pair(w1 >> 2)};
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    st.o[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(fqa_v8h, a), __builtin_bit_cast(fqa_v8h, pt[r][i]), st.o[r][j], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        st.l[r] = fqa_over_groups_sum(st.l[r]);
        if (cur.bad) st.l[r] = __builtin_nanf("");
#pragma unroll
        for (int j = 0; j < 8; ++j) st.o[r][j] -= st.z[r];
    }
}

// Parts of a row (query head of a sequence), one behind the other: 128 sums and, apart from them, (maximum, sum).
struct fqa_parts {
    float* o;                                             // [B * Hq][slots][128]
    float* ml;                                            // [B * Hq][slots][2]
    int slots;
};

// Own tokens: a workgroup takes `chunk` tiles of one sequence for 16 query rows of a key/value head, its waves share them.
template <int WAVES, int NT>
__global__ __launch_bounds__(64 * WAVES) void fqa_own_kernel(fq_attend_args a, fqa_parts parts, int chunk, int first_slot, int row_tiles) {
    __shared__ float wm[WAVES][16], wl[WAVES][16];
    __shared__ float wo[WAVES][16][132];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int b = blockIdx.z, kv = blockIdx.y / row_tiles, rt = blockIdx.y % row_tiles, G = a.Hq / a.Hkv;
    const int raw = a.lens[b];
    const long long most = (long long)a.width * a.c.page;
    const int cap = a.max_len < most ? a.max_len : (int)most;
    const bool too_long = raw > cap;
    const int len = raw > cap ? cap : raw < 0 ? 0 : raw, tiles = (len + 15) >> 4;
    const int c0 = (int)blockIdx.x * chunk;
    const int rows = G - 16 * rt < 16 ? G - 16 * rt : 16;
    const int row0 = b * a.Hq + kv * G + 16 * rt;
    const bool direct = parts.slots == 1;
    if (c0 >= tiles) {
        if (direct) {                                     // no tokens at all
            for (int i = threadIdx.x; i < rows * 16; i += 64 * WAVES)
                reinterpret_cast<fq_v4i*>(a.O)[(size_t)row0 * 16 + i] = too_long ? (fq_v4i){0x7FC07FC0, 0x7FC07FC0, 0x7FC07FC0, 0x7FC07FC0} : (fq_v4i){0, 0, 0, 0};
        } else if ((int)threadIdx.x < rows) {
            float* ml = parts.ml + ((size_t)(row0 + threadIdx.x) * parts.slots + first_slot + blockIdx.x) * 2;
            ml[0] = FQA_ZERO;
            ml[1] = too_long ? __builtin_nanf("") : 0.f;
        }
        return;
    }
    const int c1 = c0 + chunk < tiles ? c0 + chunk : tiles;
    // the waves' shares: steps of NT tiles
    const int steps = (c1 - c0 + NT - 1) / NT, per = (steps + WAVES - 1) / WAVES * NT;
    const int t0 = c0 + wave * per, t1 = t0 + per < c1 ? t0 + per : c1;
    if (t0 < t1) {
        const size_t row = (size_t)row0 + (n < rows ? n : 0);
        const fq_v4i* qp = reinterpret_cast<const fq_v4i*>(a.Q + row * 128 + 32 * g);
        const fq_v4i qa = qp[0], qb = qp[1];
        const fq_v8i q[1] = {{qa[0], qa[1], qa[2], qa[3], qb[0], qb[1], qb[2], qb[3]}};
        const float qs[1] = {a.q_scale[row] * a.out_scale * (512.0f * 1.44269504088896340736f)};
        fqa_cursor cur;
        cur.pages_of = a.table + (size_t)b * a.width;
        cur.head = a.c.base + kv * a.c.head_stride;
        cur.page_stride = a.c.page_stride;
        cur.tiles_per_page = a.c.page >> 4;
        cur.pages = a.c.pages;
        cur.bad = too_long;
        fqa_state<1> st;
        fqa_range<1, NT>(cur, t0, t1, len, q, qs, st, lane);
        if (g == 0) {
            wm[wave][n] = st.m[0];
            wl[wave][n] = st.l[0];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            *reinterpret_cast<fq_v4f*>(&wo[wave][n][16 * j + 4 * g]) = st.o[0][j];
    } else if (g == 0) {
        wm[wave][n] = FQA_ZERO;
        wl[wave][n] = 0.f;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * 32; i += 64 * WAVES) {   // four channels of a row
        const int r = i >> 5, c = 4 * (i & 31);
        float top = FQA_ZERO, l = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, wm[w][r]);
        fq_v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (wl[w][r] == 0.f) continue;                // (a wave without tokens; a NaN is kept)
            const float f = __builtin_amdgcn_exp2f(wm[w][r] - top);
            l += wl[w][r] * f;
            o += *reinterpret_cast<const fq_v4f*>(&wo[w][r][c]) * f;
        }
        if (direct) {
            const float inv = 1.0f / l;
            o *= inv;
            uint2 out;
            out.x = __builtin_bit_cast(unsigned, __builtin_convertvector((fq_v2f){o[0], o[1]}, fq_v2bf));
            out.y = __builtin_bit_cast(unsigned, __builtin_convertvector((fq_v2f){o[2], o[3]}, fq_v2bf));
            *reinterpret_cast<uint2*>(a.O + (size_t)(row0 + r) * 128 + c) = out;
        } else {
            const size_t at = (size_t)(row0 + r) * parts.slots + first_slot + blockIdx.x;
            *reinterpret_cast<fq_v4f*>(parts.o + at * 128 + c) = o;
            if (c == 0) {
                parts.ml[at * 2] = top;
                parts.ml[at * 2 + 1] = l;
            }
        }
    }
}

// The shared prefix: a wave takes `chunk` tiles for RT * 16 of a key/value head's B * G query rows.
template <int RT, int NT>
__global__ __launch_bounds__(256) void fqa_prefix_kernel(fq_attend_args a, fqa_parts parts, int chunk) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int kv = blockIdx.z, G = a.Hq / a.Hkv, rows = a.B * G;
    const int first = ((int)blockIdx.y * 4 + wave) * RT * 16;
    if (first >= rows) return;
    const int tiles = (a.prefix + 15) >> 4, t0 = (int)blockIdx.x * chunk, t1 = t0 + chunk < tiles ? t0 + chunk : tiles;
    fq_v8i q[RT];
    float qs[RT];
    size_t at[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int i = first + 16 * r + n, k = i < rows ? i : rows - 1;
        at[r] = (size_t)(k / G) * a.Hq + kv * G + k % G;
        const fq_v4i* qp = reinterpret_cast<const fq_v4i*>(a.Q + at[r] * 128 + 32 * g);
        const fq_v4i qa = qp[0], qb = qp[1];
        q[r] = (fq_v8i){qa[0], qa[1], qa[2], qa[3], qb[0], qb[1], qb[2], qb[3]};
        qs[r] = a.q_scale[at[r]] * a.out_scale * (512.0f * 1.44269504088896340736f);
    }
    fqa_cursor cur;
    cur.pages_of = a.shared;
    cur.head = a.c.base + kv * a.c.head_stride;
    cur.page_stride = a.c.page_stride;
    cur.tiles_per_page = a.c.page >> 4;
    cur.pages = a.c.pages;
    cur.bad = false;
    fqa_state<RT> st;
    fqa_range<RT, NT>(cur, t0, t1, a.prefix, q, qs, st, lane);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (first + 16 * r + n >= rows) continue;
        const size_t s = at[r] * parts.slots + blockIdx.x;
#pragma unroll
        for (int j = 0; j < 8; ++j) *reinterpret_cast<fq_v4f*>(parts.o + s * 128 + 16 * j + 4 * g) = st.o[r][j];
        if (g == 0) {
            parts.ml[s * 2] = st.m[r];
            parts.ml[s * 2 + 1] = st.l[r];
        }
    }
}

// One wave per row: the parts' sums, each brought to the largest maximum.
__global__ __launch_bounds__(256) void fqa_join_kernel(fqa_parts parts, uint16_t* __restrict__ O, int rows) {
    const int lane = threadIdx.x & 63, row = (int)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    const float* ml = parts.ml + (size_t)row * parts.slots * 2;
    const float* po = parts.o + (size_t)row * parts.slots * 128;
    float top = FQA_ZERO;
    for (int s = lane; s < parts.slots; s += 64) top = fmaxf(top, ml[2 * s]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    float l = 0.f, x = 0.f, y = 0.f;
    for (int s = 0; s < parts.slots; ++s) {
        const float pl = ml[2 * s + 1];
        if (pl == 0.f) continue;
        const float f = __builtin_amdgcn_exp2f(ml[2 * s] - top);
        l += pl * f;
        const fq_v2f o = *reinterpret_cast<const fq_v2f*>(po + (size_t)s * 128 + 2 * lane);
        x += o[0] * f;
        y += o[1] * f;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    reinterpret_cast<unsigned*>(O)[(size_t)row * 64 + lane] = __builtin_bit_cast(unsigned, __builtin_convertvector((fq_v2f){x * inv, y * inv}, fq_v2bf));
}

struct fqa_plan { int own_chunk, own_slots, prefix_chunk, prefix_slots; };

fqa_plan fqa_choose(int B, int Hq, int Hkv, int max_len, int prefix) {
    fqa_plan p = {0, 0, 0, 0};
    const int G = Hq / Hkv, row_tiles = (G + 15) / 16, cus = fq_device_cus();
    const int tiles = max_len > 0 ? (int)(((long long)max_len + 15) / 16) : 1;   // (one empty part says so where a length passes 0)
    {
        // workgroups of four waves, about four for each compute unit
        const long long heads = (long long)B * Hkv * row_tiles;
        long long want = (4ll * cus + heads - 1) / heads;
        long long chunk = (tiles + want - 1) / want;
        chunk = chunk < 16 ? 16 : chunk > 128 ? 128 : (chunk + 15) / 16 * 16;
        p.own_chunk = (int)chunk;
        p.own_slots = (int)((tiles + chunk - 1) / chunk);
    }
    if (prefix > 0) {
        const int pt = (int)(((long long)prefix + 15) / 16);
        const long long groups = ((long long)B * G + 127) / 128 * Hkv;
        long long want = (2ll * cus + groups - 1) / groups;
        long long chunk = (pt + want - 1) / want;
        chunk = chunk < 8 ? 8 : chunk > 64 ? 64 : (chunk + 3) / 4 * 4;
        p.prefix_chunk = (int)chunk;
        p.prefix_slots = (int)((pt + chunk - 1) / chunk);
    }
    return p;
}

}  // namespace

size_t fq_attend_scratch_bytes(int B, int Hq, int Hkv, int max_len, int prefix) {
    const fqa_plan p = fqa_choose(B, Hq, Hkv, max_len, prefix);
    const size_t slots = (size_t)p.own_slots + p.prefix_slots;
    return slots <= 1 && prefix <= 0 ? 0 : slots * B * Hq * 130 * sizeof(float);
}

void fq_launch_attend(const fq_attend_args& a, void* scratch, hipStream_t stream) {
    const fqa_plan p = fqa_choose(a.B, a.Hq, a.Hkv, a.max_len, a.prefix);
    const int slots = p.own_slots + p.prefix_slots, G = a.Hq / a.Hkv, row_tiles = (G + 15) / 16;
    const bool join = slots > 1 || a.prefix > 0;
    fqa_parts parts = {static_cast<float*>(scratch), static_cast<float*>(scratch) + (size_t)slots * a.B * a.Hq * 128, join ? slots : 1};
    if (p.prefix_slots)
        hipLaunchKernelGGL((fqa_prefix_kernel<2, 4>), dim3(p.prefix_slots, (a.B * G + 127) / 128, a.Hkv), dim3(256), 0, stream, a, parts, p.prefix_chunk);
    hipLaunchKernelGGL((fqa_own_kernel<4, 4>), dim3(p.own_slots, a.Hkv * row_tiles, a.B), dim3(256), 0, stream, a, parts, p.own_chunk, p.prefix_slots, row_tiles);
    if (join)
        hipLaunchKernelGGL(fqa_join_kernel, dim3((unsigned)((a.B * a.Hq + 3) / 4)), dim3(256), 0, stream, parts, a.O, a.B * a.Hq);
}
