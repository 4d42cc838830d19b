// Attention of new tokens, one or many of each sequence, over the paged INT4 cache (include/fireq_chunk.h): prompts, chunks of prompts and
// single tokens, with a range of tokens for each row, a window, scores capped by a tanh and a bias by distance.
//
// Rows are (token, query head) pairs of a key/value head, a token's heads one behind the other; 16 RT of them are a wave's query tile, and
// the products are those of fq_attend.hip (S^T = K Q^T in FP8, O^T = V^T P^T in fp16, sums in FP32).  What differs:
//     ranges     a row's tokens are lo <= t < hi.  A wave takes the tiles that any of its rows has; where all of its rows have all of a step's
//                tokens, no score is compared with a range.
//     shape      x = cap tanh(out_scale q k / cap) - slope |pos - t|, in units of log2 e.  tanh(y) = y P(y^2) of three terms while every |y| is
//                at most 5/16 (relative error 2^-19), of five up to 5/8 (2^-23), 1 - 2 / (1 + exp(2 y)) above.  A distance is counted from the row's
//                nearest token: a constant less for all scores of a row, and exact in FP32 where it counts.
//     broken     a value whose scale is NaN must not reach the rows that do not see its token (0 * NaN): its NaN moves to the key's scale,
//                which makes the probabilities NaN of those rows only that see it; so does a tile of a page outside the cache.
#include <type_traits>

#include "fq_attend.h"

namespace {

// log2 e * cap * the coefficients of tanh(y) / y in y^2, least squares in relative error
#define FQC_SMALL 0.625f
#define FQC_TINY 0.3125f
struct fqc_shape {
    float t[3];                                           // |y| <= FQC_TINY: 2^-19
    float k[5];                                           // |y| <= FQC_SMALL: 2^-23
    float k1, k2;                                         // log2 e * cap and twice that
};

constexpr int FQC_MANY_ROWS = 128;                       // of a workgroup with many rows

struct fqc_args {
    const uint8_t* Q;
    const float* q_scale;
    fq_paged_cache c;
    const int32_t *table, *starts, *lens, *first, *end;
    const float* slopes;
    int width, window, T, B, Hq, Hkv, max_len, slots, chunk;   // parts of a row, and tiles of one at least
    float out_scale, inv_cap;                             // inv_cap: 1 / cap (0: uncapped)
    fqc_shape shape;
    uint16_t* O;
};

// The tiles of a range one after the other, as in fq_attend.hip; a tile of a page outside the cache has NaN scales.
struct fqc_cursor {
    const int* pages_of;
    const uint8_t* head;
    unsigned page_stride;                                 // in 16 bytes
    int last, tile, page, within, tiles_per_page, first, pages;
    int ids;                                              // lane l: page number first + l
    __device__ __forceinline__ void fetch(int lane) {
        const int last_page = last / tiles_per_page;
        const int p = first + lane < last_page ? first + lane : last_page;
        const int id = pages_of[p];
        ids = (unsigned)id < (unsigned)pages ? id : -1;
    }
    __device__ __forceinline__ void start(int t0, int t1, int lane) {
        tile = t0;
        last = t1 - 1;
        page = first = t0 / tiles_per_page;
        within = t0 - page * tiles_per_page;
        fetch(lane);
    }
    // where the next NT tiles lie; bit i of `lost`: tile i's page is outside.  Behind the range its last tile again.
    template <int NT>
    __device__ __forceinline__ void places(const uint8_t* (&p)[NT], unsigned& lost, int lane) {
        if (page - first > 64 - NT) {
            first = page;
            fetch(lane);
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int id = __builtin_amdgcn_readlane(ids, page - first);
            lost |= id < 0 ? 1u << i : 0u;
            p[i] = head + (((unsigned long long)(unsigned)(id < 0 ? 0 : id) * page_stride) << 4) + (unsigned)(within * FQP_TILE);
            const int on = tile < last ? 1 : 0;
            tile += on;
            within += on;
            const int over = within == tiles_per_page ? 1 : 0;
            page += over;
            within = over ? 0 : within;
        }
    }
    // the bytes of the next NT tiles; bit i of the answer: tile i's page is outside (its scales are made NaN when they have arrived)
    template <int NT>
    __device__ __forceinline__ unsigned next(fqa_tile (&t)[NT], int lane) {
        const uint8_t* p[NT];
        unsigned lost = 0u;
        places(p, lost, lane);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p[i]), 0, FQP_TILE, 0x00020000);
            t[i].k = __builtin_bit_cast(fq_v4i, __builtin_amdgcn_raw_buffer_load_b128(r, 16 * lane, 0, 0));
            t[i].v = __builtin_bit_cast(fq_v4i, __builtin_amdgcn_raw_buffer_load_b128(r, 16 * lane, 1024, 0));
            t[i].s = __builtin_bit_cast(fq_v2i, __builtin_amdgcn_raw_buffer_load_b64(r, 8 * (lane >> 4), 2048, 0));
        }
        return lost;
    }
};

// The same for a longer walk: where 64 of them lie is worked out at a time, a tile a lane, from page numbers requested 64 tiles before;
// a step reads two lanes and adds.  A tile of a page outside the cache has NaN scales.
struct fqc_walk {
    const int* pages_of;
    const uint8_t* head;
    unsigned page_stride;                                 // in 16 bytes
    int last, tile, first, tiles_per_page, pages;
    int id;                                               // lane l: the page of tile first + 64 + l
    unsigned lo, hi;                                      // lane l: where tile first + l lies
    unsigned long long lost;                              // bit l: its page is outside the cache
    __device__ __forceinline__ int page_of(int lane) const {
        const int t = first + lane < last ? first + lane : last;
        return (int)((unsigned)t / (unsigned)tiles_per_page);
    }
    __device__ __forceinline__ void window(int lane) {    // the window whose pages are in `id`, from tile `first` on
        const int t = first + lane < last ? first + lane : last, page = page_of(lane);
        const bool ok = (unsigned)id < (unsigned)pages;
        const unsigned long long at = ((unsigned long long)(ok ? (unsigned)id : 0u) * page_stride << 4) + (unsigned)((t - page * tiles_per_page) * FQP_TILE);
        lo = (unsigned)at;
        hi = (unsigned)(at >> 32);
        lost = __ballot(!ok);
        first += 64;
        id = pages_of[page_of(lane)];
        first -= 64;
    }
    __device__ __forceinline__ void start(int t0, int t1, int lane) {
        tile = first = t0;
        last = t1 - 1;
        id = pages_of[page_of(lane)];
        window(lane);
    }
    // before every step's `places`; all steps take the same number of tiles, a divisor of 64
    __device__ __forceinline__ void refill(int lane) {
        if (tile - first >= 64) {
            first += 64;
            window(lane);
        }
    }
    // where tiles i and i + 1 of the next ones lie; bits 0 and 1: their pages are outside.  Behind the range its last tile again.
    __device__ __forceinline__ unsigned places(int i, const uint8_t* (&p)[2]) const {
        const int j = tile - first + i;
#pragma unroll
        for (int u = 0; u < 2; ++u)
            p[u] = head + ((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)hi, j + u) << 32 | (unsigned)__builtin_amdgcn_readlane((int)lo, j + u));
        return (unsigned)(lost >> j) & 3u;
    }
};

// A wave's rows: lane n (and n + 16, ..) has row 16 r + n of each query tile r.
template <int RT>
struct fqc_rows {
    int lo[RT], hi[RT];                                   // its tokens
    int pos[RT], near[RT];                                // its own place, and the distance of its nearest token
    float slope[RT];                                      // -log2 e * slope
};

// A NaN in a value's scale moves to the key's (four of each: s[0] keys, s[1] values).
__device__ __forceinline__ void fqc_move_nans(fq_v2i& s) {
    const unsigned bad = (((unsigned)s[1] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u, bytes = (bad >> 7) * 0xFFu;
    s[0] = (int)((unsigned)s[0] | (bytes & 0x7F7F7F7Fu));
    s[1] = (int)((unsigned)s[1] & ~bytes);
}

// Products c of a lane's RT rows and NT times 4 tokens (`first` + i * STEP + e), with the keys' sigmas ks -> probabilities, eight of them a lane's part of
// the B operand of a product with values.  STEP 16: a row's tokens are shared out among four lanes, 16 apart, STEP 8: two, 32 apart; rescale(r, x)
// multiplies its sums.  whole: every row has all of the tokens; otherwise the others' scores become -infinity, whose probability is 0 beside any finite
// reference (a row's before its first token too, and its factor is not 0).  The query tiles go through each stage together: one branch for all, and each
// one's chain of instructions beside the others'.
template <int RT, int NT, int STEP, bool CAP, bool BIAS, class F>
__device__ __forceinline__ void fqc_probabilities(const fq_v4f (&c)[RT][NT], const float (&ks)[NT][4], int first, const float (&qs)[RT],
                                                  const fqc_rows<RT>& rows, const fqc_shape& shape, float (&m)[RT], float (&sub)[RT], bool whole,
                                                  fq_v4i (&pt)[RT][NT / 2], F rescale) {
    constexpr bool SHAPED = CAP || BIAS;
    // scores: before the row's factor f = qs, or, with a shape, whole
    float s[RT][NT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[r][i][e] = BIAS && !CAP ? c[r][i][e] * ks[i][e] * qs[r] : c[r][i][e] * ks[i][e];
    if (CAP) {
        // y = t * qs; while every |y| is small, the polynomial alone
        float most = 0.f;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(s[r][i][e]));
            most = fmaxf(most, top * qs[r]);
        }
        auto small = [&](float u) __attribute__((always_inline)) {
            return fmaf(fmaf(fmaf(fmaf(shape.k[4], u, shape.k[3]), u, shape.k[2]), u, shape.k[1]), u, shape.k[0]);
        };
        if (!__any(!(most <= FQC_TINY))) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = s[r][i][e] * qs[r], u = y * y;
                        s[r][i][e] = y * fmaf(fmaf(shape.t[2], u, shape.t[1]), u, shape.t[0]);
                    }
        } else if (!__any(!(most <= FQC_SMALL))) {
            asm volatile("" : "+v"(most));                // (branches: nothing of one beside another)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = s[r][i][e] * qs[r];
                        s[r][i][e] = y * small(y * y);
                    }
        } else {
            float two = 2.0f * 1.44269504088896340736f;
            asm volatile("" : "+v"(two));
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = s[r][i][e] * qs[r], z = y * small(y * y);
                        const float far = fmaf(-shape.k2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y * two) + 1.0f), shape.k1);
                        s[r][i][e] = fabsf(y) <= FQC_SMALL ? z : far;
                    }
        }
    }
    if (BIAS) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int d = rows.pos[r] - (first + i * STEP + e), away = (d < 0 ? -d : d) - rows.near[r];
                    s[r][i][e] = fmaf(rows.slope[r], (float)away, s[r][i][e]);
                }
    }
    if (!whole) {
        int here = first;
        asm volatile("" : "+v"(here));                    // (a branch, not selections in every step)
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int at = here - rows.lo[r], n = rows.hi[r] - rows.lo[r];
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[r][i][e] = (unsigned)(at + STEP * i + e) < (unsigned)n ? s[r][i][e] : -__builtin_inff();
        }
    }
    float top[RT];
    bool past = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        top[r] = FQA_LOWEST;
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) top[r] = fmaxf(top[r], s[r][i][e]);
        past = past || (SHAPED ? top[r] - m[r] : (top[r] - m[r]) * qs[r]) > FQA_SLACK;
    }
    if (__any(past))
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const float f = SHAPED ? 1.0f : qs[r], half = fmaxf(top[r], __shfl_xor(top[r], 32, 64));
            const float over = STEP == 16 ? fmaxf(half, __shfl_xor(half, 16, 64)) : half;
            // (a row that is not past its slack keeps its reference and its term, whatever the others do)
            const bool on = (over - m[r]) * f > FQA_SLACK;
            const float best = on ? over : m[r], x = __builtin_amdgcn_exp2f((m[r] - best) * f);
            m[r] = best;
            sub[r] = on ? fmaf(best, -f, FQA_LIFT) : sub[r];
            rescale(r, x);
        }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                float p[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) p[u] = __builtin_amdgcn_exp2f(SHAPED ? s[r][i][e + u] + sub[r] : fmaf(s[r][i][e + u], qs[r], sub[r]));
                pt[r][i / 2][2 * (i & 1) + e / 2] = __builtin_bit_cast(int, __builtin_convertvector((fq_v2f){p[0], p[1]}, fqa_v2h));
            }
}

// Values as fq_attend.hip has them, one shift less for each word: a code in bits 4 .. 7 of a half under the exponent of 1024 is the number 1024 + 16 c, and
// one fused multiply-add with sigma / 16 and -72 sigma makes it sigma * (c - 8), exact (72 sigma has 8 bits and is at most 32256).
__device__ __forceinline__ fqa_sigmas fqc_value_sigmas(int w) {
    fqa_sigmas s;
    const fqa_v2h a = __builtin_convertvector(__builtin_amdgcn_cvt_pk_f32_fp8(w, false), fqa_v2h);
    const fqa_v2h b = __builtin_convertvector(__builtin_amdgcn_cvt_pk_f32_fp8(w, true), fqa_v2h);
    s.s[0] = a * (fqa_v2h){(_Float16)0.0625f, (_Float16)0.0625f};
    s.s[1] = b * (fqa_v2h){(_Float16)0.0625f, (_Float16)0.0625f};
    s.n[0] = a * (fqa_v2h){(_Float16)-72.f, (_Float16)-72.f};
    s.n[1] = b * (fqa_v2h){(_Float16)-72.f, (_Float16)-72.f};
    return s;
}
#define FQC_VALUE_MASK 0x00F000F0u
#define FQC_VALUE_BASE 0x64006400u
// Four tokens' values of a word: nibbles 0 and 2 (tokens 0, 1 and 2, 3 of one channel), 1 and 3 (of the channel 16 on).
__device__ __forceinline__ void fqc_values4(int w, unsigned mask, unsigned base, const fqa_sigmas& a, fq_v2i& even, fq_v2i& odds) {
    const unsigned x = (unsigned)w;
    even = (fq_v2i){__builtin_bit_cast(int, fqa_value_pair(x << 4, mask, base, a.s[0], a.n[0])),
                    __builtin_bit_cast(int, fqa_value_pair(x >> 4, mask, base, a.s[1], a.n[1]))};
    odds = (fq_v2i){__builtin_bit_cast(int, fqa_value_pair(x, mask, base, a.s[0], a.n[0])),
                    __builtin_bit_cast(int, fqa_value_pair(x >> 8, mask, base, a.s[1], a.n[1]))};
}
// The lane's values for channels j and j + 1 of 16, j even: word w of each of two tiles (nibble 0: channel j of tokens 0, 1; 2: of tokens 2, 3; 1 and
// 3: j + 1).
__device__ __forceinline__ void fqc_values(int w0, int w1, unsigned mask, unsigned base, const fqa_sigmas& a, const fqa_sigmas& b, fqa_v8h& even,
                                           fqa_v8h& odds) {
    const unsigned x = (unsigned)w0, y = (unsigned)w1;
    const fqa_v2h e0 = fqa_value_pair(x << 4, mask, base, a.s[0], a.n[0]), e1 = fqa_value_pair(x >> 4, mask, base, a.s[1], a.n[1]);
    const fqa_v2h e2 = fqa_value_pair(y << 4, mask, base, b.s[0], b.n[0]), e3 = fqa_value_pair(y >> 4, mask, base, b.s[1], b.n[1]);
    const fqa_v2h o0 = fqa_value_pair(x, mask, base, a.s[0], a.n[0]), o1 = fqa_value_pair(x >> 8, mask, base, a.s[1], a.n[1]);
    const fqa_v2h o2 = fqa_value_pair(y, mask, base, b.s[0], b.n[0]), o3 = fqa_value_pair(y >> 8, mask, base, b.s[1], b.n[1]);
    even = (fqa_v8h){e0[0], e0[1], e1[0], e1[1], e2[0], e2[1], e3[0], e3[1]};
    odds = (fqa_v8h){o0[0], o0[1], o1[0], o1[1], o2[0], o2[1], o3[0], o3[1]};
}
#define FQC_MFMA_PV(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(fqa_v8h, (a)), __builtin_bit_cast(fqa_v8h, (b)), (c), 0, 0, 0)
#define FQC_ONES ((fq_v4i){0x3C003C00, 0x3C003C00, 0x3C003C00, 0x3C003C00})

// NT (even) tiles from tile tb on.
template <int RT, int NT, bool CAP, bool BIAS>
__device__ __forceinline__ void fqc_step(fqa_tile (&now)[NT], unsigned lost, int tb, const fqa_queries<RT>& Q, const fqc_rows<RT>& rows,
                                         const fqc_shape& shape, fqa_state<RT>& st, bool whole, unsigned mask, unsigned base, int g) {
    unsigned odd = 0u;
#pragma unroll
    for (int i = 0; i < NT; ++i) odd |= ((unsigned)now[i].s[1] & 0x7F7F7F7Fu) + 0x01010101u;
    if (lost != 0u || __any((odd & 0x80808080u) != 0u))
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            now[i].s |= lost >> i & 1u ? 0x7F7F7F7F : 0;
            fqc_move_nans(now[i].s);
        }
    float ks[NT][4];
    fq_v4f c[RT][NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const fq_v8i k = fq_unpack_chunk(now[i].k);
#pragma unroll
        for (int r = 0; r < RT; ++r) c[r][i] = FQA_MFMA_QK(k, Q.q[r], Q.zp[r]);
        if (RT == 1) __builtin_amdgcn_sched_barrier(0);   // (both tiles' operands at once are registers: 2 % of a large batch)
        const fq_v2f s01 = __builtin_amdgcn_cvt_pk_f32_fp8(now[i].s[0], false), s23 = __builtin_amdgcn_cvt_pk_f32_fp8(now[i].s[0], true);
        ks[i][0] = s01[0]; ks[i][1] = s01[1]; ks[i][2] = s23[0]; ks[i][3] = s23[1];
    }
    fq_v4i pt[RT][NT / 2];
    auto rescale = [&](int r, float x) __attribute__((always_inline)) {
        st.l[r] *= x;
#pragma unroll
        for (int j = 0; j < 8; ++j) st.o[r][j] *= x;
    };
    fqc_probabilities<RT, NT, 16, CAP, BIAS>(c, ks, 16 * tb + 4 * g, Q.qs, rows, shape, st.m, st.sub, whole, pt, rescale);
#pragma unroll
    for (int i = 0; i < NT / 2; ++i) {
        const fqa_sigmas sg[2] = {fqc_value_sigmas(now[2 * i].s[1]), fqc_value_sigmas(now[2 * i + 1].s[1])};
#pragma unroll
        for (int r = 0; r < RT; ++r) st.l[r] = FQC_MFMA_PV(FQC_ONES, pt[r][i], st.l[r]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            fqa_v8h even, odds;
            fqc_values(now[2 * i].v[w], now[2 * i + 1].v[w], mask, base, sg[0], sg[1], even, odds);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                st.o[r][2 * w] = FQC_MFMA_PV(even, pt[r][i], st.o[r][2 * w]);
                st.o[r][2 * w + 1] = FQC_MFMA_PV(odds, pt[r][i], st.o[r][2 * w + 1]);
            }
        }
    }
}

template <int RT, bool CAP, bool BIAS>
__device__ __forceinline__ void fqc_begin(const fqa_queries<RT>& Q, fqa_state<RT>& st) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        // below every score (sums of 128 products of FP8 numbers and codes, at most 10^9; with a shape, FP32's own range)
        st.m[r] = CAP || BIAS ? FQA_LOWEST : -1.0e30f;
        st.sub[r] = CAP || BIAS ? -FQA_LOWEST : fminf(fmaf(1.0e30f, Q.qs[r], FQA_LIFT), -FQA_LOWEST);   // (a factor of 1e-30 never passes the slack)
        st.l[r] = (fq_v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) st.o[r][j] = (fq_v4f){0.f, 0.f, 0.f, 0.f};
    }
}

// Tiles t0 .. t1 for a wave's rows, the first ones' bytes in `a`; from token `whole0` to `whole1` all rows have all tokens.
template <int RT, int NT, bool CAP, bool BIAS>
__device__ __forceinline__ void fqc_range(fqc_cursor& cur, fqa_tile (&a)[NT], unsigned lost_a, int t0, int t1, int whole0, int whole1,
                                          const fqa_queries<RT>& Q, const fqc_rows<RT>& rows, const fqc_shape& shape, fqa_state<RT>& st, int lane) {
    const int g = lane >> 4;
    fqc_begin<RT, CAP, BIAS>(Q, st);
    unsigned mask = FQC_VALUE_MASK, base = FQC_VALUE_BASE;
    asm("" : "+s"(mask));
    asm("" : "+v"(base));
    auto step = [&](fqa_tile (&now)[NT], unsigned lost, int tb) __attribute__((always_inline)) {
        // (a step past t1 repeats the last tile behind its end: its tokens are masked there, for `whole1` is at most 16 t1)
        fqc_step<RT, NT, CAP, BIAS>(now, lost, tb, Q, rows, shape, st, tb * 16 >= whole0 && (tb + NT) * 16 <= whole1, mask, base, g);
    };
    fqa_tile b[NT];
    unsigned lost_b = 0u;
    for (int tb = t0; tb < t1; tb += 2 * NT) {
        if (tb + NT < t1) lost_b = cur.next(b, lane);
        step(a, lost_a, tb);
        if (tb + NT >= t1) break;
        if (tb + 2 * NT < t1) lost_a = cur.next(a, lane);
        step(b, lost_b, tb + NT);
    }
    if (!(CAP || BIAS))
#pragma unroll
        for (int r = 0; r < RT; ++r) st.m[r] *= Q.qs[r];
}

// The least of a wave's lanes, for all.
__device__ __forceinline__ int fqc_wave_min(int v) { return (int)(~fq_wave_max(~((unsigned)v ^ 0x80000000u)) ^ 0x80000000u); }

__device__ __forceinline__ int fqc_clamp(int v, int hi) { return v < 0 ? 0 : v > hi ? hi : v; }

// Query tiles of `rows` rows: those of sequence b are numbered from starts[b] * G / rows + b on, which leaves each sequence room for what it can
// need without anyone knowing their lengths.  The sequence of tile k (or -1), 64 candidates at a time; its first tile, rows and length.
struct fqc_sequence { int b, tile0, start, stop, len; };
__device__ __forceinline__ fqc_sequence fqc_sequence_of(const fqc_args& a, int k, int G, int rows, int lane) {
    int lo = 0, n = a.B;
    while (true) {
        const int stride = (n + 63) >> 6, i = lo + lane * stride;
        const bool in = i < lo + n;
        const int raw = in ? a.starts[i] : 0, len = in && stride == 1 ? a.lens[i] : 0, behind = stride == 1 ? a.starts[lo + n] : 0;
        const int first = fqc_clamp(raw, a.T);
        const int at = in ? (int)((unsigned)(first * G) / (unsigned)rows) + i : 0;   // (T * G is below 2^25, rows a power of two)
        const unsigned long long below = __ballot(in && at <= k);
        if (below == 0ull) return {-1, 0, 0, 0, 0};
        const int count = __popcll(below) - 1;
        lo += count * stride;
        n = n - count * stride < stride ? n - count * stride : stride;
        if (stride > 1) continue;
        const int next = __builtin_amdgcn_readlane(first, count < 63 ? count + 1 : 63);
        return {lo, __builtin_amdgcn_readlane(at, count), __builtin_amdgcn_readlane(first, count),
                count < 63 && count + 1 < __popcll(__ballot(in)) ? next : fqc_clamp(behind, a.T), __builtin_amdgcn_readlane(len, count)};
    }
}

// What a workgroup works on: rows row0 .. row0 + nrows - 1 of the (new token, query head) pairs of sequence b under key/value head kv.
struct fqc_place {
    int b, kv, G, start, count, row0, nrows, raw, len;
    bool too_long;
    __device__ __forceinline__ void take(const fqc_args& a, int sequence, int first, int stop, int length) {
        b = sequence;
        G = a.Hq / a.Hkv;
        kv = (int)(blockIdx.x % a.Hkv);
        start = first;
        count = stop - first;
        raw = length;
        const long long room = (long long)a.width * a.c.page;
        const int cap = a.max_len < room ? a.max_len : (int)room;
        too_long = raw > cap;
        len = too_long ? cap : raw < 0 ? 0 : raw;
    }
    // k: the workgroup's query tile, of ROWS rows
    template <int ROWS>
    __device__ __forceinline__ bool find(const fqc_args& a, int k, int lane) {
        const fqc_sequence q = fqc_sequence_of(a, k, a.Hq / a.Hkv, ROWS, lane);
        if (q.b < 0) return false;
        take(a, q.b, q.start, q.stop, q.len);
        row0 = (k - q.tile0) * ROWS;                        // (T * G is bounded: 32 bits hold it)
        if (count <= 0 || count * G <= row0 || row0 < 0) return false;   // (row0 < 0: starts that decrease)
        nrows = count * G - row0 < ROWS ? count * G - row0 : ROWS;
        return true;
    }
    __device__ __forceinline__ int token(int i) const { return count == 1 ? 0 : (int)((unsigned)(row0 + i) / (unsigned)G); }   // of row i, among the new ones
    __device__ __forceinline__ size_t row(const fqc_args& a, int i) const {
        const int t = token(i);
        return (size_t)(start + t) * a.Hq + kv * G + (row0 + i - t * G);
    }
};

// The ranges of a wave's rows (first .. of the workgroup's), and what they have together: tokens tok0 .. tok1, all of them those from whole0 to whole1.
// none: rows without a token, which take any range and are zeros in the end.
struct fqc_span { int tok0, tok1, whole0, whole1; unsigned none; };
template <int RT, bool BIAS>
__device__ __forceinline__ fqc_span fqc_take_rows(const fqc_args& a, const fqc_place& at, int first_row, int n, fqc_rows<RT>& rows) {
    fqc_span sp;
    sp.none = 0u;
    int lo = 0x7FFFFFFF, hi = 0x7FFFFFFF, wlo = 0x7FFFFFFF, whi = 0x7FFFFFFF;   // the least lo and hi, and of minus them
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int i = first_row + 16 * r + n < at.nrows ? first_row + 16 * r + n : 0, t = at.token(i);
        const int pos = at.raw - at.count + t;
        int f = a.first ? a.first[at.start + t] : 0, e = a.end ? a.end[at.start + t] : pos + 1;
        if (a.window > 0 && pos >= a.window && f <= pos - a.window) f = pos - a.window + 1;   // (a shorter place leaves all; below 0 it would pass 32 bits)
        f = f < 0 ? 0 : f;
        e = e > at.len ? at.len : e;
        const bool none = f >= e, empty = none || first_row + 16 * r + n >= at.nrows;
        sp.none |= empty ? 1u << r : 0u;
        rows.lo[r] = none ? 0 : f;
        rows.hi[r] = none ? 0x7FFFFFFF : e;
        if (BIAS) {
            rows.pos[r] = pos;
            rows.near[r] = none ? 0 : pos < f ? f - pos : pos >= e ? pos - (e - 1) : 0;
            const float slope = a.slopes[at.kv * at.G + (at.row0 + i - t * at.G)] * -1.44269504088896340736f;
            rows.slope[r] = slope < -0x1p127f ? -0x1p127f : slope;   // (finite: the nearest token's distance is 0; a NaN stays)
        }
        if (!none) {
            lo = f < lo ? f : lo;
            whi = -e < whi ? -e : whi;
        }
        wlo = -rows.lo[r] < wlo ? -rows.lo[r] : wlo;
        hi = rows.hi[r] < hi ? rows.hi[r] : hi;
    }
    if (at.count == 1) {                                  // one token: one range
        lo = __builtin_amdgcn_readfirstlane(lo);
        whi = __builtin_amdgcn_readfirstlane(whi);
        sp.tok0 = lo;
        sp.tok1 = whi == 0x7FFFFFFF ? 0 : -whi;
        sp.whole0 = -__builtin_amdgcn_readfirstlane(wlo);
        sp.whole1 = __builtin_amdgcn_readfirstlane(hi);
        return sp;
    }
    sp.tok0 = fqc_wave_min(lo);
    const int last = fqc_wave_min(whi);
    sp.tok1 = last == 0x7FFFFFFF ? 0 : -last;
    sp.whole0 = -fqc_wave_min(wlo);
    sp.whole1 = fqc_wave_min(hi);
    return sp;
}
template <int RT, bool CAP, bool BIAS>
__device__ __forceinline__ void fqc_take_queries(const fqc_args& a, const fqc_place& at, int first_row, int n, int g, fqa_queries<RT>& Q) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const size_t row = at.row(a, first_row + 16 * r + n < at.nrows ? first_row + 16 * r + n : 0);
        fqa_take_query(Q, r, a.Q + row * 128, a.q_scale[row], a.out_scale, g);
        if (!(CAP || BIAS)) Q.qs[r] = Q.qs[r] < 1.0e-30f ? 1.0e-30f : Q.qs[r];   // (a NaN stays)
        if (CAP) Q.qs[r] *= a.inv_cap * 0.693147180559945309417f;   // (a capped score's factor has no log2 e)
    }
}

// Few rows: a sequence's rows of one key/value head, and part blockIdx.y of the tokens that its rows have, shared out among the waves, which meet in LDS.
// Bound by the tiles' bytes, 130 a token, and by their latency: 37 capped sequences of up to 6000 tokens 33 us in a graph (106 MB, 3.2 TB/s; vector
// instructions 48 % of the busy cycles, waits 49 % of the waves' time), 30 without a cap, 64 x 8192 plain 109 to 111 (4.9 TB/s, a copy's rate), one of
// 32001 with a bias 16 (14 without).  Registers for four waves a SIMD are too few: 38, 30, 128 and 20 with them.  A sequence with more rows than max_new
// promised is worked on in turns.
template <int RT, int KVW, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * KVW, 2) void fqc_few_kernel(fqc_args a, fqa_parts parts) {
    constexpr int ROWS = 16 * RT, NT = 2;
    __shared__ fqa_shared<RT, KVW> sh;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = (int)(blockIdx.x / a.Hkv);
    fqc_place at;
    at.take(a, b, fqc_clamp(a.starts[b], a.T), fqc_clamp(a.starts[b + 1], a.T), a.lens[b]);
    const int all_rows = at.count > 0 ? at.count * at.G : 0;
    at.row0 = 0;
    if (a.slots > 1 && (long long)blockIdx.y * a.chunk * 16 >= at.len) {   // behind the sequence's end, wherever its rows' tokens begin
        for (int i = threadIdx.x; i < all_rows; i += 64 * KVW) {
            float* ml = parts.ml + (at.row(a, i) * parts.slots + blockIdx.y) * 2;
            ml[0] = FQA_LOWEST;
            ml[1] = at.too_long ? __builtin_nanf("") : 0.f;
        }
        return;
    }
    for (; at.row0 < all_rows; at.row0 += ROWS) {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));                    // (nothing of a turn is kept in registers for the next)
        const int n = lane & 15, g = lane >> 4;
        at.nrows = all_rows - at.row0 < ROWS ? all_rows - at.row0 : ROWS;
        fqc_rows<RT> rows;
        const fqc_span sp = fqc_take_rows<RT, BIAS>(a, at, 0, n, rows);
        const int tok0 = sp.tok0, tok1 = sp.tok1, whole0 = sp.whole0, whole1 = sp.whole1, nrows = at.nrows;
        const unsigned none = sp.none;
        const bool too_long = at.too_long;
        const int first_tile = tok1 > 0 ? tok0 >> 4 : 0, all = tok1 > 0 ? ((tok1 + 15) >> 4) - first_tile : 0;
        // this workgroup's part, and the waves' shares: steps of NT tiles
        const int even = ((all + a.slots - 1) / a.slots + NT - 1) / NT * NT, part = even > a.chunk ? even : a.chunk, c0 = first_tile + (int)blockIdx.y * part;
        const int c1 = c0 + part < first_tile + all ? c0 + part : first_tile + all;
        const int share = c1 > c0 ? ((c1 - c0 + NT - 1) / NT + KVW - 1) / KVW * NT : 0, t0 = c0 + wave * share, t1 = t0 + share < c1 ? t0 + share : c1;
        fqa_state<RT> st;
        const bool work = t0 < t1;
        if (work) {
            fqc_cursor cur;
            cur.pages_of = a.table + (size_t)at.b * a.width;
            cur.head = a.c.base + at.kv * a.c.head_stride;
            cur.page_stride = (unsigned)(a.c.page_stride >> 4);
            cur.tiles_per_page = a.c.page >> 4;
            cur.pages = a.c.pages;
            cur.start(t0, t1, lane);
            fqa_queries<RT> Q;
            fqa_tile ahead[NT];
            const unsigned lost = cur.next(ahead, lane);      // (on their way while the queries are taken)
            fqc_take_queries<RT, CAP, BIAS>(a, at, 0, n, g, Q);
            fqc_range<RT, NT, CAP, BIAS>(cur, ahead, lost, t0, t1, whole0, whole1 < 16 * t1 ? whole1 : 16 * t1, Q, rows, a.shape, st, lane);
        }
        if (work) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if (g == 0) {
                    sh.m[wave][16 * r + n] = st.m[r];
                    sh.l[wave][16 * r + n] = too_long ? __builtin_nanf("") : (none >> r & 1u) != 0u ? 0.f : st.l[r][0];
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) *reinterpret_cast<fq_v4f*>(&sh.o[wave][16 * r + n][16 * j + 4 * g]) = st.o[r][j];
            }
        } else if (lane < ROWS) {
            sh.m[wave][lane] = FQA_LOWEST;
            sh.l[wave][lane] = too_long ? __builtin_nanf("") : 0.f;
        }
        __syncthreads();
        for (int i = 64 * wave + lane; i < nrows * 32; i += 64 * KVW) {  // four channels of a row
            const int r = i >> 5, c = 4 * (i & 31);
            float top = FQA_LOWEST, l = 0.f;
#pragma unroll
            for (int w = 0; w < KVW; ++w)
                if (sh.l[w][r] != 0.f) top = fmaxf(top, sh.m[w][r]);
            fq_v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < KVW; ++w) {
                if (sh.l[w][r] == 0.f) continue;          // (a wave without tokens of this row; a NaN is kept)
                const float f = __builtin_amdgcn_exp2f(sh.m[w][r] - top);
                l += sh.l[w][r] * f;
                o += *reinterpret_cast<const fq_v4f*>(&sh.o[w][r][c]) * f;
            }
            const size_t row = at.row(a, r);
            if (a.slots == 1) {
                *reinterpret_cast<uint2*>(a.O + row * 128 + c) = fqa_output(o, l);
            } else {
                const size_t place = row * parts.slots + blockIdx.y;
                *reinterpret_cast<fq_v4f*>(parts.o + place * 128 + c) = o;
                if (c == 0) {
                    parts.ml[place * 2] = top;
                    parts.ml[place * 2 + 1] = l;
                }
            }
        }
        if (at.row0 + ROWS < all_rows) __syncthreads();       // (max_new was too small: the next rows in the same LDS)
    }
}

// Many rows: four waves with 32 rows each walk the same tokens, 64 of a step.  Each wave unpacks a quarter of the step's codes into LDS, where all read
// their operands; the next step's codes are unpacked beside this one's score products, and those behind it are on their way.  The products are
// v_mfma_f32_32x32x64_f8f6f4 and v_mfma_f32_32x32x16_f16, transposed as in fq_attend.hip: A = 32 tokens (two tiles), B = 32 rows; a lane then has, of one row
// (lane % 32), the tokens 8 k + 4 h + e (h = lane / 32), and a tile's eight are its part of the B operand of a product with 32 channels, values in the same
// order.  (A vector instruction costs half as much beside a product of 32 x 32 as beside one of 16 x 16, measured with two waves a SIMD.)  sum p: of the
// rounded numbers, two to an instruction.
// Bound by instructions: vector 76 %, matrix 28 % of the busy cycles.  8192 new tokens under 32 heads, 8 of keys: 505 to 528 us causal (1041 to 1090
// TFLOP/s, at the card's power: its clock falls to 2 GHz), 665 to 715 capped with a prefix seen whole (820 to 880); 4096 with a bias 190 to 204 (673);
// 2048 49 to 52; a tile's own cost shows in 5000 tokens behind a window of one, 22 (60 MB).  Kept on the way there, on the capped one: operands unpacked
// once a workgroup and not by each wave (1201 us from 2491), masks and tanh's ranges in branches (969, 773), three terms of tanh (719).  16 x 16
// products took 696 and, causal, 530 to 558; 64 rows a wave spill.
struct fqc_stage {
    fq_v4i k[2][2][2][64];                                // keys' bytes: pair of tiles, 64 dimensions, low and high nibbles, lane
    fq_v4i v[4][4][64];                                   // values in fp16: tile, 32 channels, lane
    float ks[4][16];                                      // keys' sigmas
};
struct fqc_fetched { fq_v4i k; fq_v2i v[2], s[2]; unsigned bad; };   // a wave's quarter: keys of one tile, half the values of its pair
#define FQC_MFMA32_QK(a, b, c) __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4((a), (b), (c), 0, 0, 0, 0, 0, 0)
#define FQC_MFMA32_PV(a, b, c) __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(fqa_v8h, (a)), __builtin_bit_cast(fqa_v8h, (b)), (c), 0, 0, 0)

template <bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void fqc_many_kernel(fqc_args a, fqa_parts parts) {
    constexpr int NT = 4;
    __shared__ fqc_stage stage[2];
    __shared__ int span[4][2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
    fqc_place at;
    // (later rows of a prompt have more tokens: they begin)
    if (!at.find<FQC_MANY_ROWS>(a, a.T * (a.Hq / a.Hkv) / FQC_MANY_ROWS + a.B - 1 - (int)(blockIdx.x / a.Hkv), lane)) return;
    fqc_rows<1> rows;
    const int first_row = 32 * wave;
    const fqc_span sp = fqc_take_rows<1, BIAS>(a, at, first_row, n, rows);
    if (lane == 0) {
        span[wave][0] = sp.tok1 > 0 ? sp.tok0 : 0x7FFFFFFF;
        span[wave][1] = sp.tok1;
    }
    __syncthreads();
    int tok0 = 0x7FFFFFFF, tok1 = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        tok0 = span[w][0] < tok0 ? span[w][0] : tok0;
        tok1 = span[w][1] > tok1 ? span[w][1] : tok1;
    }
    tok0 = __builtin_amdgcn_readfirstlane(tok0);
    tok1 = __builtin_amdgcn_readfirstlane(tok1);
    const int first_tile = tok1 > 0 ? tok0 >> 4 : 0, all = tok1 > 0 ? ((tok1 + 15) >> 4) - first_tile : 0;
    const int even = ((all + a.slots - 1) / a.slots + NT - 1) / NT * NT, part = even > a.chunk ? even : a.chunk, t0 = first_tile + (int)blockIdx.y * part;
    const int t1 = t0 + part < first_tile + all ? t0 + part : first_tile + all;
    const int whole0 = sp.whole0, whole1 = sp.whole1 < 16 * t1 ? sp.whole1 : 16 * t1;
    // this lane's row: its codes (dimensions 64 u + 32 h ..), their zero point, its factor
    const int own_row = first_row + n;
    const size_t row = at.row(a, own_row < at.nrows ? own_row : 0);
    const float scale = a.q_scale[row];
    fq_v4i codes[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) codes[u] = reinterpret_cast<const fq_v4i*>(a.Q + row * 128 + 64 * (u >> 1) + 32 * h)[u & 1];
    int spare = 0;                                        // the stage that no wave reads any more
    float m[1] = {FQA_LOWEST}, l = 0.f;
    fq_v16f o[4] = {};
    unsigned mask = FQC_VALUE_MASK, base = FQC_VALUE_BASE;
    asm("" : "+s"(mask));
    asm("" : "+v"(base));
    if (t0 < t1) {
        fqc_walk cur;
        cur.pages_of = a.table + (size_t)at.b * a.width;
        cur.head = a.c.base + at.kv * a.c.head_stride;
        cur.page_stride = (unsigned)(a.c.page_stride >> 4);
        cur.tiles_per_page = a.c.page >> 4;
        cur.pages = a.c.pages;
        cur.start(t0, t1, lane);
        const int pair = wave & 1, half = wave >> 1;       // tiles 2 pair and 2 pair + 1; words 2 half and 2 half + 1 of their values
        const int t = lane & 15, g = lane >> 4;            // where a lane's bytes of a tile belong: token (channel) t, dimensions (tokens) of quarter g
        auto fetch = [&](fqc_fetched& f) __attribute__((always_inline)) {
            const uint8_t* p[2];
            f.bad = cur.places(2 * pair, p);
            cur.tile += NT;
            __amdgpu_buffer_rsrc_t r[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) r[i] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p[i]), 0, FQP_TILE, 0x00020000);
            f.k = __builtin_bit_cast(fq_v4i, __builtin_amdgcn_raw_buffer_load_b128(half ? r[1] : r[0], 16 * lane, 0, 0));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f.v[i] = __builtin_bit_cast(fq_v2i, __builtin_amdgcn_raw_buffer_load_b64(r[i], 16 * lane, 1024 + 8 * half, 0));
                f.s[i] = __builtin_bit_cast(fq_v2i, __builtin_amdgcn_raw_buffer_load_b64(r[i], 8 * g, 2048, 0));
            }
        };
        auto mend = [&](fqc_fetched& f) __attribute__((always_inline)) {
            const unsigned odd = (((unsigned)f.s[0][1] & 0x7F7F7F7Fu) + 0x01010101u) | (((unsigned)f.s[1][1] & 0x7F7F7F7Fu) + 0x01010101u);
            if (f.bad != 0u || __any((odd & 0x80808080u) != 0u))
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    f.s[i] |= f.bad >> i & 1u ? 0x7F7F7F7F : 0;
                    fqc_move_nans(f.s[i]);
                }
        };
        auto unpack = [&](const fqc_fetched& f, fqc_stage& to) __attribute__((always_inline)) {
            const int tile = 2 * pair + half, place = 32 * (g & 1) + 16 * half + t;
            const fq_v8i k = fq_unpack_chunk(f.k);
            to.k[pair][g >> 1][0][place] = (fq_v4i){k[0], k[1], k[2], k[3]};
            to.k[pair][g >> 1][1][place] = (fq_v4i){k[4], k[5], k[6], k[7]};
            const fqa_sigmas s[2] = {fqc_value_sigmas(f.s[0][1]), fqc_value_sigmas(f.s[1][1])};
#pragma unroll
            for (int i = 0; i < 2; ++i)                   // (tile of the pair)
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    fq_v2i even, odds;
                    fqc_values4(f.v[i][w], mask, base, s[i], even, odds);
                    fq_v2i* dst = reinterpret_cast<fq_v2i*>(&to.v[2 * pair + i][2 * half + w][32 * (g & 1) + t]) + (g >> 1);
                    dst[0] = even;
                    dst[32] = odds;                       // 16 lanes on
                }
            const int w = half ? f.s[1][0] : f.s[0][0];
            const fq_v2f s01 = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), s23 = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            *reinterpret_cast<fq_v4f*>(&to.ks[tile][4 * g]) = (fq_v4f){s01[0], s01[1], s23[0], s23[1]};   // (by all lanes of a group, the same)
        };
        fqc_fetched f;
        fetch(f);
        // (on its way while the queries are taken)
        fq_v8i q[2];
        float qs[1] = {fabsf(scale) * a.out_scale * (512.0f * 1.44269504088896340736f)};
        fq_v16f zp = {};
        {
            const int flip = scale < 0.f ? (int)0x80808080 : 0;
            constexpr int E = (int)FQ_ZP_BYTES;
            const fq_v8i eights = {E, E, E, E, E, E, E, E};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const fq_v4i x = codes[2 * u] ^ flip, y = codes[2 * u + 1] ^ flip;
                q[u] = (fq_v8i){x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                zp = FQC_MFMA32_QK(eights, q[u], zp);
            }
            if (!(CAP || BIAS)) qs[0] = qs[0] < 1.0e-30f ? 1.0e-30f : qs[0];   // (a NaN stays)
            if (CAP) qs[0] *= a.inv_cap * 0.693147180559945309417f;   // (a capped score's factor has no log2 e)
        }
        // (what the reference and its term begin with: fqc_begin)
        m[0] = CAP || BIAS ? FQA_LOWEST : -1.0e30f;
        float sub[1] = {CAP || BIAS ? -FQA_LOWEST : fminf(fmaf(1.0e30f, qs[0], FQA_LIFT), -FQA_LOWEST)};
        mend(f);
        unpack(f, stage[0]);
        if (t0 + NT < t1) {
            cur.refill(lane);
            fetch(f);
        }
        // a step whose operands stage u holds; MORE: the next one's are unpacked beside its score products, and those behind are requested
        auto step = [&](auto more, int u, int now) __attribute__((always_inline)) {
            constexpr bool MORE = decltype(more)::value;
            __syncthreads();                              // this step's operands are there, and the other stage is free
            if (MORE) {
                cur.refill(lane);
                mend(f);
            }
            const fqc_stage& from = stage[u];
            fq_v4f c[1][2 * NT];
            float ks[2 * NT][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                fq_v16f x = zp;
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    const fq_v4i lo = from.k[i][d][0][lane], hi = from.k[i][d][1][lane];
                    x = FQC_MFMA32_QK(((fq_v8i){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}), q[d], x);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) c[0][4 * i + k] = (fq_v4f){x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]};
            }
#pragma unroll
            for (int k = 0; k < 2 * NT; ++k) {
                const fq_v4f s = *reinterpret_cast<const fq_v4f*>(&from.ks[k >> 1][8 * (k & 1) + 4 * h]);
#pragma unroll
                for (int e = 0; e < 4; ++e) ks[k][e] = s[e];
            }
            if (MORE) {
                unpack(f, stage[u ^ 1]);
                fetch(f);                                 // (behind the range the last tile again)
            }
            if (now * 16 >= sp.tok1 || (now + NT) * 16 <= sp.tok0) return;   // (none of this wave's rows has any of the tokens)
            const bool whole = now * 16 >= whole0 && (now + NT) * 16 <= whole1;
            fq_v4i pt[1][NT];
            auto rescale = [&](int, float x) __attribute__((always_inline)) {
                l *= x;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] *= x;
            };
            fqc_probabilities<1, 2 * NT, 8, CAP, BIAS>(c, ks, 16 * now + 4 * h, qs, rows, a.shape, m, sub, whole, pt, rescale);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int two = pt[0][i][e];          // (a bit cast of the element itself takes the first one's bits)
                    l = __builtin_amdgcn_fdot2(__builtin_bit_cast(fqa_v2h, two), (fqa_v2h){(_Float16)1.f, (_Float16)1.f}, l, false);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = FQC_MFMA32_PV(from.v[i][j][lane], pt[0][i], o[j]);
            }
        };
        int now = t0;
        for (; now + 2 * NT < t1; now += 2 * NT) {
            step(std::true_type(), 0, now);
            step(std::true_type(), 1, now + NT);
        }
        if (now + NT < t1) {
            step(std::true_type(), 0, now);
            step(std::false_type(), 1, now + NT);
            spare = 0;
        } else {
            step(std::false_type(), 0, now);
            spare = 1;
        }
        if (!(CAP || BIAS)) m[0] *= qs[0];
    }
    l += __shfl_xor(l, 32, 64);
    const bool zero = t0 >= t1 || sp.none != 0u;
    l = at.too_long ? __builtin_nanf("") : zero ? 0.f : l;
    if (t0 < t1) {
        // 128 bytes of every row at a time through the stage that is free, so that they leave side by side (16 bytes a row apart took 7 us more for
        // 5000 tokens of 32 heads)
        constexpr int PITCH = 144;
        static_assert(sizeof(fqc_stage) >= 4 * 32 * PITCH, "a part for each wave");
        uint8_t* const mine = reinterpret_cast<uint8_t*>(&stage[spare]) + wave * 32 * PITCH;
        auto leave = [&](uint8_t* dst, size_t stride) __attribute__((always_inline)) {   // (a wave's own LDS accesses stay in order)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 8 * i + (lane >> 3);
                const size_t to = (size_t)(unsigned)__shfl((int)row, r, 64);
                const fq_v4i x = *reinterpret_cast<const fq_v4i*>(mine + r * PITCH + 16 * (lane & 7));
                if (first_row + r < at.nrows) *reinterpret_cast<fq_v4i*>(dst + to * stride + 16 * (lane & 7)) = x;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        if (a.slots == 1) {
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const fq_v16f& y = o[j + k / 4];
                    const fq_v4f x = {y[4 * (k & 3)], y[4 * (k & 3) + 1], y[4 * (k & 3) + 2], y[4 * (k & 3) + 3]};
                    *reinterpret_cast<uint2*>(mine + n * PITCH + 16 * k + 8 * h) = fqa_output(zero ? (fq_v4f){0.f, 0.f, 0.f, 0.f} : x, l);
                }
                leave(reinterpret_cast<uint8_t*>(a.O) + 64 * j, 256);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    *reinterpret_cast<fq_v4f*>(mine + n * PITCH + 32 * k + 16 * h) = (fq_v4f){o[j][4 * k], o[j][4 * k + 1], o[j][4 * k + 2], o[j][4 * k + 3]};
                leave(reinterpret_cast<uint8_t*>(parts.o) + 512 * (size_t)blockIdx.y + 128 * j, (size_t)parts.slots * 512);
            }
        }
    }
    if (own_row >= at.nrows) return;
    if (a.slots > 1) {
        const size_t place = row * parts.slots + blockIdx.y;
        if (h == 0) {
            parts.ml[place * 2] = m[0];
            parts.ml[place * 2 + 1] = l;
        }
    } else if (t0 >= t1) {
        fq_v4i* dst = reinterpret_cast<fq_v4i*>(a.O + row * 128 + 64 * h);
        constexpr int N = 0x7FC07FC0;
#pragma unroll
        for (int k = 0; k < 8; ++k) dst[k] = at.too_long ? (fq_v4i){N, N, N, N} : (fq_v4i){0, 0, 0, 0};
    }
}

// few: 16 * few rows of a query tile, whose tokens four waves share out (0: many rows); slots: parts of a row's tokens, chunk: tiles of one at least
// (a multiple of 4; more where that many parts would not hold a row's tokens).  `tokens` bounds those of a row.
//     few      up to 32 rows of a head.  16 x 4000 tokens under 32 heads, 8 of keys: 4 new tokens each 24 us (40 by the kernel of many rows), 8 each 31 (41);
//              for 16 rows the wider tile takes 28.  With 64 rows they meet: 54 and 61, two such sequences 23 and 20, one of 30000 35 and 30.
//     parts    of many rows: one workgroup a compute unit, or two where that pays.  A step of 64 tokens takes about 1.2 us with one and 1.8 with two, 1.6 and
//              2.5 with a cap or a bias; a part adds 1040 bytes a row to what is joined, at 6 TB/s, and with more than 8 a row takes a workgroup there
//              (1.3 ns a row).  us by the parts, one sequence, the choice here first:
//                  plain, half a microsecond a step saved: 500 tokens at 4000, 4 parts 46; 2 53     33 at 30000, 32 40; 16 47     640 at 4000, 3 54; 1 78
//                  1000 at 1400, 1 32; 2 41     1000 behind a window of 1024, 1 32; 2 41     but 200 at 4096, 9 38; 8 28; 4 30 (its join)
//                  capped, what its steps cost: 640 at 4000, 3 69; 1 107     640 at 1400, 3 35; 1 41     768 at 1400, 1 42; 2 44     1000 at 1400, 1 42; 2 50
//                  1000 at 4000, 2 99; 1 107     256 at 4096, 8 36; 4 49     200 at 30000, 9 149; 4 204     64 at 30000, 32 57; 16 88     200 behind a window
//                  of 4096, 4 38; 9 43     500 at 1400, 2 34; 4 33
//                  several: 2 x 320 at 1400, 3 38; 1 41     5 x 128, 3 37; 1 41     but 7 x 92 at 1392, 3 48; 1 41     3 x 40 at 8000, 8 53; 16 49
struct fqc_plan { int few, slots, chunk; };
fqc_plan fqc_choose(int T, int B, int Hq, int Hkv, int max_new, int tokens, bool shaped) {
    const int G = Hq / Hkv, cus = fq_device_cus();
    const long long most = (long long)(max_new < T ? max_new : T) * G;
    fqc_plan p = {most <= 16 ? 1 : most <= 32 ? 2 : 0, 1, 4};
    const int rows = p.few ? 16 * p.few : FQC_MANY_ROWS, tiles = tokens > 0 ? (int)(((long long)tokens + 15) / 16) : 1;
    const long long query_tiles = ((long long)T * G + rows - 1) / rows, units = (p.few || query_tiles < B ? B : query_tiles) * Hkv;
    if (p.few) {
        p.chunk = (fqa_part(units, tiles, cus, B > 1) + 3) / 4 * 4;
        p.slots = (tiles + p.chunk - 1) / p.chunk;
    } else {
        const long long one = cus / units > 1 ? cus / units : 1, room = tiles / 8;
        const long long two = 2 * cus / units;
        const double part = (double)T * Hq * 1040 / 6.0e6, steps = tiles / 4;   // us
        double saved = 0.5 * steps / one, joined = one > 1 ? one * part : 2.5 + 2 * part;
        if (shaped) {
            saved = two > one ? 1.6 * steps * (1.0 / one - 1.53 / two) : 0.0;
            joined = one > 1 ? (two - one) * part : 2.5 + two * part;
            if (two > FQA_JOIN_FEW) joined += 1.3e-3 * T * Hq;
        }
        const long long want = saved > joined ? two : one, slots = want < room ? want : room;
        p.slots = (int)(slots < 1 ? 1 : slots > 64 ? 64 : slots);
    }
    return p;
}
// For a call: a window may leave a row fewer tokens than max_len.  Never more parts than the scratch is for.
fqc_plan fqc_choose(const fq_chunk_args& x) {
    const fqc_plan most = fqc_choose(x.T, x.B, x.Hq, x.Hkv, x.max_new, x.max_len, false);
    const long long span = (long long)x.window + (most.few ? 16 * most.few : FQC_MANY_ROWS) / (x.Hq / x.Hkv) + 15;   // (of a query tile, from a tile's beginning)
    fqc_plan p = fqc_choose(x.T, x.B, x.Hq, x.Hkv, x.max_new, x.window > 0 && !x.end && span < x.max_len ? (int)span : x.max_len, x.cap > 0.f || x.slopes);
    p.slots = p.slots < most.slots ? p.slots : most.slots;
    return p;
}

template <int FEW, bool CAP, bool BIAS>
void fqc_launch(const fqc_args& a, const fqa_parts& parts, hipStream_t stream) {
    const long long query_tiles = FEW != 0 ? a.B : (long long)a.T * (a.Hq / a.Hkv) / FQC_MANY_ROWS + a.B;
    const dim3 grid((unsigned)(query_tiles * a.Hkv), (unsigned)a.slots);
    if constexpr (FEW != 0) hipLaunchKernelGGL((fqc_few_kernel<FEW, 4, CAP, BIAS>), grid, dim3(256), 0, stream, a, parts);
    else hipLaunchKernelGGL((fqc_many_kernel<CAP, BIAS>), grid, dim3(256), 0, stream, a, parts);
}
template <int FEW>
void fqc_launch(const fqc_args& a, const fqa_parts& parts, hipStream_t stream) {
    const bool cap = a.inv_cap != 0.f, bias = a.slopes != nullptr;
    if (cap && bias) fqc_launch<FEW, true, true>(a, parts, stream);
    else if (cap) fqc_launch<FEW, true, false>(a, parts, stream);
    else if (bias) fqc_launch<FEW, false, true>(a, parts, stream);
    else fqc_launch<FEW, false, false>(a, parts, stream);
}

}  // namespace

size_t fq_chunk_scratch_bytes(int T, int B, int Hq, int Hkv, int max_new, int max_len) {
    const int slots = fqc_choose(T, B, Hq, Hkv, max_new, max_len, false).slots;
    return slots > 1 ? (size_t)slots * T * Hq * 130 * sizeof(float) : 0;
}

void fq_launch_chunk(const fq_chunk_args& x, void* scratch, hipStream_t stream) {
    const fqc_plan p = fqc_choose(x);
    const float cap = x.cap < 0x1p100f ? x.cap : 0x1p100f;   // (no score comes near; a larger one's double or inverse would leave FP32's normal numbers)
    fqc_args a = {x.Q, x.q_scale, x.c, x.table, x.starts, x.lens, x.first, x.end, x.slopes, x.width, x.window, x.T, x.B, x.Hq, x.Hkv, x.max_len, p.slots, p.chunk,
                  x.out_scale, cap > 0.f ? 1.0f / cap : 0.f, {}, x.O};
    const double c[5] = {0x1.fffffcp-1, -0x1.5551b8p-2, 0x1.107a08p-3, -0x1.a88656p-5, 0x1.ed307ap-7}, k1 = 1.44269504088896340736 * cap;
    const double t[3] = {0x1.ffffcep-1, -0x1.550db4p-2, 0x1.0193e6p-3};
    for (int i = 0; i < 5; ++i) a.shape.k[i] = (float)(k1 * c[i]);
    for (int i = 0; i < 3; ++i) a.shape.t[i] = (float)(k1 * t[i]);
    a.shape.k1 = (float)k1;
    a.shape.k2 = (float)(2.0 * k1);
    const fqa_parts parts = {static_cast<float*>(scratch), static_cast<float*>(scratch) + (size_t)p.slots * x.T * x.Hq * 128, p.slots};
    if (p.few == 1) fqc_launch<1>(a, parts, stream);
    else if (p.few == 2) fqc_launch<2>(a, parts, stream);
    else fqc_launch<0>(a, parts, stream);
    if (p.slots > 1) fqa_join(parts, x.O, x.T * x.Hq, stream, x.starts, x.B, x.Hq);
}
