// Quantisation to 8-bit integers, shared by the kernels of the int8 experts:
// a row (a token, a token's activations in an expert, a weight channel) has
// one fp32 scale s = amax / 127, and each element the code rint(x / s), the
// quotient rounded to 32 bits first, ties to even.  Codes lie in [-127, 127].
// A row of zeros has scale 0 and codes 0; a row that holds an infinity or a
// NaN has scale NaN and codes 0, so every result it reaches is NaN.
#pragma once

#include "common.h"

DEV uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
DEV uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// A row's scale from the bits of its largest magnitude (a NaN's bits are above
// an infinity's, which are above every number's).
struct I8Scale {
    float s, inv;
    bool far;    // s is out of the range where the short division below is exact
    DEV explicit I8Scale(uint32_t amax) {
        const float a = __uint_as_float(amax);
        s = amax >= 0x7f800000u ? __builtin_nanf("") : a / 127.0f;
        far = !(a > 1e-30f && a < 1e30f);
        inv = far ? 0.f : 1.0f / s;
    }
    // The correctly rounded quotient x / s from the correctly rounded 1 / s
    // (Markstein: the remainder x - q s is exact in a fused multiply-add, and
    // one correction by it rounds the quotient correctly), in 3 instructions
    // where the general division takes about ten.
    DEV int code(float x) const {
        float q;
        if (far) {
            if (!(s > 0.f)) return 0;
            q = x / s;
        } else {
            q = x * inv;
            q = __builtin_fmaf(__builtin_fmaf(-q, s, x), inv, q);
        }
        const int c = (int)rintf(q);
        return c > 127 ? 127 : c < -127 ? -127 : c;
    }
};

// Four codes in one word, the first in the low byte.
DEV uint32_t pack_i8(int a, int b, int c, int d) {
    return (uint32_t)(a & 255) | ((uint32_t)(b & 255) << 8) | ((uint32_t)(c & 255) << 16) | ((uint32_t)d << 24);
}
