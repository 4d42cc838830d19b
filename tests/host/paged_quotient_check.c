// Host-side check of the short quotients of the paged append (csrc/fq_paged.hip), all FP32, IEEE.
//   scales      for every significand of a maximum m: fma(fma(-n, q, m), c, q) with c = fp32(1 / n), q = m * c, is the IEEE quotient m / n,
//               n = 448 and n = 7
//   INT4 codes  for every positive E4M3 sigma and every x within 64 units of a border (k + 1/2) * sigma or of a multiple of sigma, both
//               signs, and every estimate r0 of 1 / sigma within one unit: fma(fma(q, sigma, -x), -r0, q), q = x * r0, clamped to
//               -8 .. 7 and rounded by the addition of 1.5 * 2^23, is the code of the IEEE quotient
//   E4M3 codes  for maxima at every STRIDE-th significand, s = m / 448, r0 within one unit of 1 / s: x within 8 units of every border
//               between two codes times s: the same code
// Exit status 0 = no difference.  usage: paged_quotient_check [STRIDE]
#include <math.h>
#include <omp.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
static inline float from(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }
static inline uint32_t bits(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }
static uint8_t e4m3(float f) {                            // |f| < 464, nearest even
  const uint32_t u = bits(f);
  const uint8_t sign = (uint8_t)((u >> 24) & 0x80);
  const float a = fabsf(f);
  if (a < 0x1p-6f) return (uint8_t)(sign | (int)nearbyintf(a * 512.0f));
  const uint32_t m = u & 0x7FFFFFFFu, r = m + 0x7FFFFu + ((m >> 20) & 1u);
  return (uint8_t)(sign | ((r >> 20) - (120u << 3)));
}
static float value(int code) {
  const int e = code >> 3 & 15, m = code & 7;
  return e ? ldexpf(8 + m, e - 10) : ldexpf(m, -9);
}
static inline float quotient(float x, float s, float r) {
  const float q = x * r;
  return fmaf(fmaf(q, s, -x), -r, q);
}
static int int4_ieee(float x, float s) { return (int)fminf(fmaxf(nearbyintf(x / s), -8.f), 7.f) + 8; }
static int int4_short(float x, float s, float r) { return (int)(bits(fminf(fmaxf(quotient(x, s, r), -8.f), 7.f) + 12582920.0f) & 15u); }
int main(int argc, char** argv) {
  const int stride = argc > 1 ? atoi(argv[1]) : 1;
  long long bad = 0, total = 0;
  const float c448 = 1.0f / 448.0f, c7 = 1.0f / 7.0f;
  #pragma omp parallel for schedule(static) reduction(+ : bad, total)
  for (uint32_t f = 0; f < 1u << 24; ++f) {               // two binades: every significand at both parities of the exponent
    const float m = from(0x3F800000u + f), q = m * c448, p = m * c7;
    total += 2;
    if (bits(fmaf(fmaf(-448.0f, q, m), c448, q)) != bits(m / 448.0f)) ++bad;
    if (bits(fmaf(fmaf(-7.0f, p, m), c7, p)) != bits(m / 7.0f)) ++bad;
  }
  for (int code = 1; code < 127; ++code) {
    const float s = value(code), r = 1.0f / s;
    for (int d = -1; d <= 1; ++d) {
      const float r0 = from(bits(r) + (uint32_t)d);
      for (int h = 1; h <= 17; ++h)
        for (int u = -64; u <= 64; ++u) {
          const float x = from(bits(0.5f * (float)h * s) + (uint32_t)u);
          total += 2;
          if (int4_short(x, s, r0) != int4_ieee(x, s)) ++bad;
          if (int4_short(-x, s, r0) != int4_ieee(-x, s)) ++bad;
        }
      total += 1;
      if (int4_short(0.0f, s, r0) != 8) ++bad;
    }
  }
  #pragma omp parallel for schedule(dynamic, 4096) reduction(+ : bad, total)
  for (uint32_t f = 0; f < 1u << 23; f += (uint32_t)stride) {
    const float m = from(0x3F800000u + f), s = m / 448.0f, r = 1.0f / s;
    for (int d = -1; d <= 1; ++d) {
      const float r0 = from(bits(r) + (uint32_t)d);
      for (int code = 0; code < 126; ++code) {
        const float border = 0.5f * (value(code) + value(code + 1));
        for (int u = -8; u <= 8; ++u) {
          const float x = from(bits(border * s) + (uint32_t)u);
          ++total;
          if (e4m3(quotient(x, s, r0)) != e4m3(x / s)) ++bad;
        }
      }
    }
  }
  printf("total %lld  differences %lld\n", total, bad);
  return bad != 0;
}
