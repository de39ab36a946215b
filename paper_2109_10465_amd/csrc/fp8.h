// The 8-bit format: blocks of 128 e4m3 values with a shared power of two.
#pragma once
#include "moe_common.h"

// Exponent byte b of a block from the bits of its largest magnitude: the smallest e >= -127 with top * 2^-e <= 448, as
// e + 127.  448 = 1.75 * 2^8, so e is top's exponent less 8, and one more where its mantissa is above 1.75; 127 for a
// block of zeros.  (A subnormal top gets -127 as well.)
__device__ __forceinline__ int scale_byte(uint32_t top) {
    const int b = (int)((min(top, 0x7f800000u) + 0x1fffffu) >> 23) - 8;
    return top == 0 ? 127 : max(b, 0);
}
// 2^-e.  e = -127 .. 120, so that this is 2^-120 .. 2^127
__device__ __forceinline__ float scale_inverse(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

static inline int fp8_blocks(int K) { return (K + 127) / 128; }
static inline int fp8_scale_stride(int K) { return (fp8_blocks(K) + 3) / 4 * 4; }

// Limits of one operand's extents and the type beside it
static inline int fp8_extent_status(int rows, int E, int K, int N, int dtype) {
    if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_DTYPE;
    if (rows < 1 || rows >= (1 << 30) || E < 1 || E > 256) return MOE_ERR_SHAPE;
    if (K < 8 || K > (1 << 20) || N < 8 || N > (1 << 20) || K % 8 || N % 8) return MOE_ERR_SHAPE;
    if ((int64_t)fp8_blocks(K) * fp8_blocks(N) >= (1 << 17)) return MOE_ERR_SHAPE;    // a matrix of fewer than 2^31 bytes
    return MOE_OK;
}
