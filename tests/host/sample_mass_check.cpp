// csrc/fq_mass.h on the host: whole numbers for every kind of share, the largest among them, and shares that add up to one.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#define __device__
#define __forceinline__ inline
#include "fq_mass.h"

static long wrong, checked;

static void check(float e) {
    const double want = nearbyint((double)(float)((double)e * 4294967040.0));   // (the product has 48 bits: it is rounded to FP32 once, then to a whole number)
    wrong += (double)fqs_units(e) != want || want > 4294967295.0;
    ++checked;
}

int main() {
    for (uint32_t b = 0; b <= 0x3F800000u; b += 61) {     // 0 .. 1, subnormals too
        float e;
        memcpy(&e, &b, 4);
        check(e);
    }
    for (int k = 0; k < 160; ++k) {                       // about the powers of two
        const float p = ldexpf(1.0f, -k);
        check(p);
        check(nextafterf(p, 0.0f));
        if (k > 0) check(nextafterf(p, 2.0f));
    }
    for (int k = 0; k <= 8; ++k) wrong += (uint64_t)fqs_units(ldexpf(1.0f, -k)) << k != (uint64_t)fqs_units(1.0f);
    printf("checked %ld wrong %ld\n", checked, wrong);
    return wrong != 0;
}
