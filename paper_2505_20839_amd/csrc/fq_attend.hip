// Decode attention over a paged INT4 key/value cache (include/fireq_paged.h): one pass over the tokens with a running maximum and sum.
//
// A wave works on a range of 16-token tiles of one key/value head for RT * 16 query rows.  Everything is transposed, so that no
// operand changes lanes on the way:
//     S^T = K Q^T   v_mfma_f32_16x16x128_f8f6f4 per tile, A = 16 tokens (a lane's 16 bytes of codes: 32 dimensions of one token), B = 16
//                   queries.  Code + 8 as an E4M3 number is the code times 2^-9 (fq_common.h); the zero point is the same for all
//                   tokens of a query, -2^-6 sum q, and the product starts from it.
//     P^T           a lane has 4 tokens (4 g + i, g = lane / 16) of one query (lane % 16): scaled by the keys' sigmas, exponentiated against the
//                   query's maximum so far and rounded to fp16 (11 bits).  Two tiles give the 8 fp16 numbers that a lane of the B
//                   operand of v_mfma_f32_16x16x32_f16 holds, tokens in this order on both sides.
//     O^T = V^T P^T per 16 channels.  A value's code c, shifted to the top of an fp16 mantissa under the exponent of 16, is the number
//                   16 + c; one packed fused multiply-add with the token's sigma and -24 sigma makes it sigma * (c - 8), exact in fp16 (8 bits).
//                   (As subnormal fp16 numbers, c * 2^-24, the codes would save a shift, but the matrix cores align products by their
//                   factors' exponents, and a subnormal's is far above its value: sums came out 2^-18 off.)
//     sum p         one more such product, against ones: the sum of the same rounded numbers.
// O stays in registers.  A query's maximum moves only when a score passes it by more than FQA_SLACK powers of two, which fp16 has room
// for: the lanes of a query compare their own scores with it, and only then with each other.
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

// The tiles of a range one after the other: page numbers 64 at a time in a register, the tile within its page counted along.
struct fqa_cursor {
    const int* pages_of;                                  // the sequence's pages
    const uint8_t* head;                                  // the head's part of page 0
    unsigned page_stride;                                 // in 16 bytes
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
    // the bytes of the next NT tiles; behind the range its last tile again
    template <int NT>
    __device__ __forceinline__ void next(fqa_tile (&t)[NT], int lane) {
        if (page - first > 64 - NT) {
            first = page;
            fetch(lane);
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int id = __builtin_amdgcn_readlane(ids, page - first);
            const uint8_t* p = head + (((unsigned long long)(unsigned)id * page_stride) << 4) + (unsigned)(within * FQP_TILE);
            t[i].k = *reinterpret_cast<const fq_v4i*>(p + 16 * lane);
            t[i].v = *reinterpret_cast<const fq_v4i*>(p + 1024 + 16 * lane);
            t[i].s = *reinterpret_cast<const fq_v2i*>(p + 2048 + 8 * (lane >> 4));
            const int on = tile < last ? 1 : 0;
            tile += on;
            within += on;
            const int over = within == tiles_per_page ? 1 : 0;
            page += over;
            within = over ? 0 : within;
        }
    }
};

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

// NT (even) tiles from tile tb on.  TAIL: tokens from `len` on are masked.
template <int RT, int NT, bool TAIL>
__device__ __forceinline__ void fqa_step(const fqa_tile (&now)[NT], int tb, int len, const fqa_queries<RT>& Q, fqa_state<RT>& st, unsigned mask,
                                         unsigned base, int g) {
    fq_v8i k[NT];
    float ks[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        k[i] = fq_unpack_chunk(now[i].k);
        const fq_v2f s01 = __builtin_amdgcn_cvt_pk_f32_fp8(now[i].s[0], false), s23 = __builtin_amdgcn_cvt_pk_f32_fp8(now[i].s[0], true);
        ks[i][0] = s01[0]; ks[i][1] = s01[1]; ks[i][2] = s23[0]; ks[i][3] = s23[1];
    }
    auto masked = [&](int i, int e) __attribute__((always_inline)) { return TAIL && (tb + i) * 16 + 4 * g + e >= len; };
    fq_v4i pt[RT][NT / 2];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float s[NT][4], top = FQA_LOWEST;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const fq_v4f c = FQA_MFMA_QK(k[i], Q.q[r], Q.zp[r]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[i][e] = masked(i, e) ? FQA_LOWEST : c[e] * ks[i][e];
                top = fmaxf(top, s[i][e]);
            }
        }
        if (__any((top - st.m[r]) * Q.qs[r] > FQA_SLACK)) {
            const float m = fmaxf(st.m[r], fqa_over_groups_max(top)), f = __builtin_amdgcn_exp2f((st.m[r] - m) * Q.qs[r]);
            st.m[r] = m;
            st.sub[r] = fmaf(m, -Q.qs[r], FQA_LIFT);
            st.l[r] *= f;
#pragma unroll
            for (int j = 0; j < 8; ++j) st.o[r][j] *= f;
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                float p[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) p[u] = masked(i, e + u) ? 0.f : __builtin_amdgcn_exp2f(fmaf(s[i][e + u], Q.qs[r], st.sub[r]));
                pt[r][i / 2][2 * (i & 1) + e / 2] = __builtin_bit_cast(int, __builtin_convertvector((fq_v2f){p[0], p[1]}, fqa_v2h));
            }
    }
    constexpr int ONE = 0x3C003C00;
    const fq_v4i ones = {ONE, ONE, ONE, ONE};
#pragma unroll
    for (int i = 0; i < NT / 2; ++i) {
        fqa_sigmas sg[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int w = now[2 * i + u].s[1];
            fq_v2f v01 = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
#pragma unroll
            for (int e = 0; e < 2; ++e) {                 // (whatever the bytes behind the end are)
                v01[e] = masked(2 * i + u, e) ? 0.f : v01[e];
                v23[e] = masked(2 * i + u, 2 + e) ? 0.f : v23[e];
            }
            sg[u].s[0] = __builtin_convertvector(v01, fqa_v2h);
            sg[u].s[1] = __builtin_convertvector(v23, fqa_v2h);
            sg[u].n[0] = sg[u].s[0] * (fqa_v2h){(_Float16)-24.f, (_Float16)-24.f};
            sg[u].n[1] = sg[u].s[1] * (fqa_v2h){(_Float16)-24.f, (_Float16)-24.f};
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
            st.l[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(fqa_v8h, ones), __builtin_bit_cast(fqa_v8h, pt[r][i]), st.l[r], 0, 0, 0);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const fqa_v8h even = fqa_values<0>(now[2 * i].v[w], now[2 * i + 1].v[w], mask, base, sg[0], sg[1]);
            const fqa_v8h odd = fqa_values<1>(now[2 * i].v[w], now[2 * i + 1].v[w], mask, base, sg[0], sg[1]);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                st.o[r][2 * w] = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, __builtin_bit_cast(fqa_v8h, pt[r][i]), st.o[r][2 * w], 0, 0, 0);
                st.o[r][2 * w + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, __builtin_bit_cast(fqa_v8h, pt[r][i]), st.o[r][2 * w + 1], 0, 0, 0);
            }
        }
    }
}

// Tiles t0 .. t1 of a head's tokens below `len`, NT tiles a step, the next AHEAD steps' bytes on their way meanwhile (buffers that
// change roles in an unrolled loop, so that no register is copied).
template <int RT, int NT, int AHEAD>
__device__ __forceinline__ void fqa_range(fqa_cursor& cur, int t0, int t1, int len, const fqa_queries<RT>& Q, fqa_state<RT>& st, int lane) {
    const int g = lane >> 4;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        st.m[r] = FQA_LOWEST;
        st.sub[r] = fmaf(FQA_LOWEST, -Q.qs[r], FQA_LIFT);
        st.l[r] = (fq_v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) st.o[r][j] = (fq_v4f){0.f, 0.f, 0.f, 0.f};
    }
    unsigned mask = 0x03C003C0u, base = 0x4C004C00u;
    asm("" : "+s"(mask));
    asm("" : "+v"(base));
    fqa_tile buf[AHEAD + 1][NT];
    const int whole = len >> 4 < t1 ? len >> 4 : t1;      // tiles below need no mask
    int tb = t0;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (u == 0 || tb + u * NT < t1) cur.next(buf[u], lane);
    while (tb + (AHEAD + 1) * NT <= whole) {
#pragma unroll
        for (int u = 0; u <= AHEAD; ++u) {
            cur.next(buf[(u + AHEAD) % (AHEAD + 1)], lane);
            fqa_step<RT, NT, false>(buf[u], tb + u * NT, len, Q, st, mask, base, g);
        }
        tb += (AHEAD + 1) * NT;
    }
    if (tb + AHEAD * NT < t1) cur.next(buf[AHEAD], lane);
#pragma unroll
    for (int u = 0; u <= AHEAD; ++u)
        if (tb + u * NT < t1) fqa_step<RT, NT, true>(buf[u], tb + u * NT, len, Q, st, mask, base, g);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        st.m[r] *= Q.qs[r];
        if (cur.bad) st.l[r][0] = __builtin_nanf("");
    }
}

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

// A workgroup's work: tiles c0 .. c1 of one key/value head for `rows` (up to 16 RT) query rows, numbered by row_of(0 .. rows - 1).  Its waves
// share the tiles out and join their sums through LDS; the result is a part of each row, or (finish) its output, with the `earlier` parts that a
// kernel before has left added.
template <int RT, int WAVES>
struct __attribute__((aligned(16))) fqa_shared {
    float o[WAVES][16 * RT][132], m[WAVES][16 * RT], l[WAVES][16 * RT];
};
template <int RT, int WAVES, int NT, int AHEAD, class F>
__device__ __forceinline__ void fqa_group(const fq_attend_args& a, const fqa_parts& parts, fqa_shared<RT, WAVES>& sh, int c0, int c1, int len,
                                          const int* pages_of, bool bad, int kv, int rows, F row_of, int slot, bool finish, int earlier) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    // the waves' shares: steps of NT tiles
    const int steps = (c1 - c0 + NT - 1) / NT, per = (steps + WAVES - 1) / WAVES * NT;
    const int t0 = c0 + wave * per, t1 = t0 + per < c1 ? t0 + per : c1;
    if (t0 < t1) {
        fqa_cursor cur;
        cur.pages_of = pages_of;
        cur.head = a.c.base + kv * a.c.head_stride;
        cur.page_stride = (unsigned)(a.c.page_stride >> 4);
        cur.tiles_per_page = a.c.page >> 4;
        cur.pages = a.c.pages;
        cur.bad = bad;
        cur.start(t0, t1, lane);
        fqa_queries<RT> Q;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const size_t row = row_of(16 * r + n < rows ? 16 * r + n : 0);
            fqa_take_query(Q, r, a.Q + row * 128, a.q_scale[row], a.out_scale, g);
        }
        fqa_state<RT> st;
        fqa_range<RT, NT, AHEAD>(cur, t0, t1, len, Q, st, lane);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            if (g == 0) {
                sh.m[wave][16 * r + n] = st.m[r];
                sh.l[wave][16 * r + n] = st.l[r][0];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) *reinterpret_cast<fq_v4f*>(&sh.o[wave][16 * r + n][16 * j + 4 * g]) = st.o[r][j];
        }
    } else if (lane < 16 * RT) {
        sh.m[wave][lane] = FQA_LOWEST;
        sh.l[wave][lane] = bad ? __builtin_nanf("") : 0.f;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * 32; i += 64 * WAVES) {   // four channels of a row
        const int r = i >> 5, c = 4 * (i & 31);
        float top = FQA_LOWEST, l = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, sh.m[w][r]);
        fq_v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (sh.l[w][r] == 0.f) continue;              // (a wave without tokens; a NaN is kept)
            const float f = __builtin_amdgcn_exp2f(sh.m[w][r] - top);
            l += sh.l[w][r] * f;
            o += *reinterpret_cast<const fq_v4f*>(&sh.o[w][r][c]) * f;
        }
        const size_t row = row_of(r);
        if (finish) {
            fqa_add_parts<1>(reinterpret_cast<const fq_v2f*>(parts.ml) + row * parts.slots, reinterpret_cast<const fq_v4f*>(parts.o) + row * parts.slots * 32 + (i & 31), 0,
                             earlier, top, l, o);
            *reinterpret_cast<uint2*>(a.O + row * 128 + c) = fqa_output(o, l);
        } else {
            const size_t at = row * parts.slots + slot;
            *reinterpret_cast<fq_v4f*>(parts.o + at * 128 + c) = o;
            if (c == 0) {
                parts.ml[at * 2] = top;
                parts.ml[at * 2 + 1] = l;
            }
        }
    }
}

// Own tokens: a workgroup takes `chunk` tiles of one sequence for 16 query rows of a key/value head.  Heads are the fastest index and chunks the
// slowest: workgroup i runs on XCD i % 8, and with chunks (of which a short sequence has the first ones only) or sequences fastest some
// XCDs got most of the work (37 sequences of 0 to 6000 tokens 37.0 us, 31.9 with a number of chunks that happened to spread them).
// Where there is enough to read, between HBM and issue: 64 x 8192 tokens (545 MB, 547 fetched) 102 us, 5.3 TB/s (a large copy 5.1, a kernel that only
// reads 7), vector and matrix instructions 55 and 13 % of the busy cycles; 37 x 0 .. 6000 (105 MB) 24.
// One workgroup per compute unit and less is bound by a wave's chain: start, length, page table and first tiles 3 us, then 0.5 us for two tiles (1 x
// 32001 tokens 10.0, 33 MB).  Two or eight waves a workgroup, four tiles a step, bytes two steps ahead were slower on most lengths.
// With shared_slots, the first workgroups of a sequence take a shared prefix instead, in chunks of shared_chunk tiles.  finish: a sequence's tokens
// are one part, whose workgroup writes the output, with the `earlier` parts of the prefix's kernel added.
template <int WAVES, int NT, int AHEAD>
__global__ __launch_bounds__(64 * WAVES, 4) void fqa_own_kernel(fq_attend_args a, fqa_parts parts, int chunk, int first_slot, int row_tiles, int shared_slots,
                                                                int shared_chunk, int finish, int earlier) {
    __shared__ fqa_shared<1, WAVES> sh;
    const int heads = a.Hkv * row_tiles, b = (int)blockIdx.x / heads, kv = (int)blockIdx.x % heads / row_tiles, rt = (int)blockIdx.x % row_tiles;
    const bool shared = (int)blockIdx.y < shared_slots;
    const int G = a.Hq / a.Hkv, raw = shared ? a.prefix : a.lens[b];
    const long long most = (long long)a.width * a.c.page;
    const int cap = shared ? raw : a.max_len < most ? a.max_len : (int)most;
    const bool too_long = raw > cap;
    const int len = raw > cap ? cap : raw < 0 ? 0 : raw, tiles = (len + 15) >> 4, per = shared ? shared_chunk : chunk;
    const int c0 = (shared ? (int)blockIdx.y : (int)blockIdx.y - shared_slots) * per, c1 = c0 + per < tiles ? c0 + per : tiles;
    const int rows = G - 16 * rt < 16 ? G - 16 * rt : 16;
    const int row0 = b * a.Hq + kv * G + 16 * rt, slot = first_slot + (int)blockIdx.y;
    if (c0 >= tiles && earlier == 0) {                    // no tokens
        if (finish) {
            constexpr int N = 0x7FC07FC0;
            for (int i = threadIdx.x; i < rows * 16; i += 64 * WAVES)
                reinterpret_cast<fq_v4i*>(a.O)[(size_t)row0 * 16 + i] = too_long ? (fq_v4i){N, N, N, N} : (fq_v4i){0, 0, 0, 0};
        } else if ((int)threadIdx.x < rows) {
            float* ml = parts.ml + ((size_t)(row0 + threadIdx.x) * parts.slots + slot) * 2;
            ml[0] = FQA_LOWEST;
            ml[1] = too_long ? __builtin_nanf("") : 0.f;
        }
        return;
    }
    fqa_group<1, WAVES, NT, AHEAD>(a, parts, sh, c0, c1, len, shared ? a.shared : a.table + (size_t)b * a.width, too_long, kv, rows, 
                                    [=](int i) { return (size_t)row0 + i; }, slot, finish != 0, earlier);
}

// The shared prefix: a workgroup takes `chunk` tiles for 16 RT of a key/value head's B * G query rows.  Workgroups with the same tiles of a
// head follow each other at a distance of Hkv, so that with 8 heads (or a multiple) they run on one XCD and find them in its L2.
// 384 rows of each of 8 heads x 12000 tokens (18.9 GFLOP) 32.4 us: 1.83 us per 1000 tokens (880 TFLOP/s; vector instructions 67 %, matrix instructions
// 23 % of the busy cycles, behind each other in two waves per SIMD) and 10.5 for the start, gathering the rows, and 8 MB of parts.  The whole call at an earlier
// state: RT = 2 54.0, 1 60.9, 3 56.1 (one wave per SIMD).
template <int RT, int WAVES, int NT, int AHEAD>
__global__ __launch_bounds__(64 * WAVES, 2) void fqa_prefix_kernel(fq_attend_args a, fqa_parts parts, int chunk, int row_groups) {
    __shared__ fqa_shared<RT, WAVES> sh;
    const int kv = (int)(blockIdx.x % a.Hkv), group = (int)(blockIdx.x / a.Hkv % row_groups), slot = (int)(blockIdx.x / a.Hkv / row_groups);
    const int G = a.Hq / a.Hkv, all = a.B * G, first = group * 16 * RT, rows = all - first < 16 * RT ? all - first : 16 * RT;
    const int tiles = (a.prefix + 15) >> 4, c0 = slot * chunk, c1 = c0 + chunk < tiles ? c0 + chunk : tiles;
    fqa_group<RT, WAVES, NT, AHEAD>(a, parts, sh, c0, c1, a.prefix, a.shared, false, kv, rows,
                                    [&](int i) { return (size_t)((first + i) / G) * a.Hq + kv * G + (first + i) % G; }, slot, false, 0);
}

// The parts' sums, each brought to the largest maximum.  32 lanes hold the 128 channels of a row; GROUPS of 32 lanes share its parts, four
// requested at a time.  A wave per row for up to 8 parts (no LDS, no barrier; 96 sequences behind a prefix, 32 query heads, 6 parts, the whole
// call 46.8 us, 50.1 with a workgroup each; 1 x 1000 tokens 6.9 and 7.3), a workgroup for more (12 parts 7.9 us, 8.3 with a wave; 32 parts
// 12.4 and 14.0).
template <int GROUPS>
__global__ __launch_bounds__(256) void fqa_join_kernel(fqa_parts parts, uint16_t* __restrict__ O, int rows) {
    constexpr int ROWS = 8 / GROUPS;                      // of a workgroup
    __shared__ float wm[GROUPS], wl[GROUPS];
    __shared__ fq_v4f wo[GROUPS][32];
    const int c = threadIdx.x & 31, grp = (int)(threadIdx.x >> 5) % GROUPS, row = (int)blockIdx.x * ROWS + (int)(threadIdx.x >> 5) / GROUPS, n = parts.slots;
    if (row >= rows) return;                              // (one row a workgroup where there is a barrier)
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

constexpr int FQA_OWN_WAVES = 4, FQA_OWN_NT = 2, FQA_OWN_AHEAD = 1, FQA_PREFIX_RT = 2, FQA_PREFIX_WAVES = 4, FQA_PREFIX_NT = 2, FQA_PREFIX_AHEAD = 1;
constexpr int FQA_PREFIX_WANT = 2, FQA_PREFIX_MIN = 16, FQA_APART = 24000, FQA_APART_FEW = 48000, FQA_JOIN_FEW = 8, FQA_FINISH = 16;

// own_chunk and own_slots: tiles of a part of a sequence, and parts of the longest; the same for the prefix, which is worked on for
// row_groups groups of rows together, or (row_groups 0) for each sequence apart, like its own tokens.  finish: the kernel of a sequence's own
// tokens, where they are one part, adds the prefix's up to FQA_FINISH parts itself and writes the output; otherwise a third kernel joins all.
struct fqa_plan {
    int own_chunk, own_slots, prefix_chunk, prefix_slots, row_groups;
    bool finish() const { return own_slots == 1 && (prefix_slots == 0 || (row_groups != 0 && prefix_slots <= FQA_FINISH)); }
    int slots() const { return prefix_slots + (finish() ? 0 : own_slots); }   // parts of a row that go through memory
};

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
int fqa_part(long long heads, int tiles, long long cus, bool uneven) {
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

fqa_plan fqa_choose(int B, int Hq, int Hkv, int max_len, int prefix) {
    fqa_plan p = {0, 0, 0, 0, 0};
    const int G = Hq / Hkv, row_tiles = (G + 15) / 16, cus = fq_device_cus();
    const long long heads = (long long)B * Hkv * row_tiles;
    const int tiles = max_len > 0 ? (int)(((long long)max_len + 15) / 16) : 1;   // (one empty part says so where a length passes 0)
    p.own_chunk = fqa_part(heads, tiles, cus, B > 1);
    p.own_slots = (tiles + p.own_chunk - 1) / p.own_chunk;
    if (prefix > 0) {
        const int pt = (int)(((long long)prefix + 15) / 16);
        // Apart: no groups of rows to gather and half the start of a kernel, but every sequence unpacks the prefix again.  us, apart / together (32
        // query, 8 key/value heads, 50 tokens of their own): 8 x 1100 (4416 tiles) 8.1 / 12.0, 64 x 300 (9728) 10.5 / 13.2, 16 x 2000 (16000) 11.1 / 11.9,
        // 32 x 2000 (32000) 15.5 / 12.4, 16 x 4000 15.3 / 13.5, 64 x 1000 15.2 / 13.5; rows that fill no group: 4 x 16000 (32000 tiles, 16 rows)
        // 16.1 / 17.8, 2 x 48000 (48000) 20.5 / 21.0, 2 x 56000 22.8 / 22.4, 4 x 26000 (52000) 21.9 / 19.4
        if (heads * pt <= ((long long)B * G <= 8 * FQA_PREFIX_RT ? FQA_APART_FEW : FQA_APART)) {
            p.prefix_chunk = fqa_part(heads, pt, cus, false);
            p.prefix_slots = (pt + p.prefix_chunk - 1) / p.prefix_chunk;
            return p;
        }
        p.row_groups = (int)(((long long)B * G + 16 * FQA_PREFIX_RT - 1) / (16 * FQA_PREFIX_RT));
        const long long groups = (long long)p.row_groups * Hkv, room = FQA_PREFIX_WANT * (long long)cus;   // workgroups, and how many run at once
        // as few parts as fill whole rounds of them to seven eighths, up to 16 parts
        long long want = 1;
        for (long long w = 1, best = 0; w <= 16 && best < 14; ++w) {
            const long long used = 16 * groups * w / ((groups * w + room - 1) / room * room);
            if (used > best) {
                best = used;
                want = w;
            }
        }
        if (want < room / groups) want = room / groups;
        long long chunk = (pt + want - 1) / want;
        chunk = chunk < FQA_PREFIX_MIN ? FQA_PREFIX_MIN : (chunk + 7) / 8 * 8;
        p.prefix_chunk = (int)chunk;
        p.prefix_slots = (int)((pt + chunk - 1) / chunk);
    }
    return p;
}

}  // namespace

size_t fq_attend_scratch_bytes(int B, int Hq, int Hkv, int max_len, int prefix) {
    return (size_t)fqa_choose(B, Hq, Hkv, max_len, prefix).slots() * B * Hq * 130 * sizeof(float);
}

void fq_launch_attend(const fq_attend_args& a, void* scratch, hipStream_t stream) {
    const fqa_plan p = fqa_choose(a.B, a.Hq, a.Hkv, a.max_len, a.prefix);
    const int slots = p.slots(), row_tiles = (a.Hq / a.Hkv + 15) / 16;
    const fqa_parts parts = {static_cast<float*>(scratch), static_cast<float*>(scratch) + (size_t)slots * a.B * a.Hq * 128, slots};
    if (p.row_groups)
        hipLaunchKernelGGL((fqa_prefix_kernel<FQA_PREFIX_RT, FQA_PREFIX_WAVES, FQA_PREFIX_NT, FQA_PREFIX_AHEAD>), dim3((unsigned)(p.prefix_slots * p.row_groups * a.Hkv)),
                           dim3(64 * FQA_PREFIX_WAVES), 0, stream, a, parts, p.prefix_chunk, p.row_groups);
    const int apart = p.row_groups ? 0 : p.prefix_slots;
    hipLaunchKernelGGL((fqa_own_kernel<FQA_OWN_WAVES, FQA_OWN_NT, FQA_OWN_AHEAD>), dim3((unsigned)(a.B * a.Hkv * row_tiles), apart + p.own_slots),
                       dim3(64 * FQA_OWN_WAVES), 0, stream, a, parts, p.own_chunk, p.prefix_slots - apart, row_tiles, apart, p.prefix_chunk, p.finish() ? 1 : 0,
                       p.finish() ? p.prefix_slots : 0);
    if (!p.finish()) {
        const int rows = a.B * a.Hq;
        if (slots <= FQA_JOIN_FEW) hipLaunchKernelGGL(fqa_join_kernel<2>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, stream, parts, a.O, rows);
        else hipLaunchKernelGGL(fqa_join_kernel<8>, dim3((unsigned)rows), dim3(256), 0, stream, parts, a.O, rows);
    }
}
