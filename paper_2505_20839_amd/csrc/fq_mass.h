// A token's mass: its share e (0 .. 1) of the best one's in whole numbers, the best's own being the largest FP32 number that 32 bits hold.  (2^32 does not
// fit, and with 2^32 - 1 for it alone two halves would be more than the whole.)
#pragma once

#define FQS_UNIT 4294967040.0f                            // 2^32 - 2^8

__device__ __forceinline__ unsigned fqs_units(float e) { return (unsigned)__builtin_rintf(e * FQS_UNIT); }
