// Sorting networks over packed (rank key, expert id) entries of 64 or 32 bits,
// shared by the routers' selections.  A larger entry ranks higher; 0 is padding.
#pragma once

#include "common.h"

// put the better of a, b first
DEV void order2(uint64_t &a, uint64_t &b) {
    const bool sw = b > a;
    const uint64_t x = a, y = b;
    a = sw ? y : x;
    b = sw ? x : y;
}
// 32-bit entries: one maximum and one minimum, where 64-bit ones take a compare
// and four selects
DEV void order2(uint32_t &a, uint32_t &b) {
    const uint32_t x = a, y = b;
    a = x > y ? x : y;
    b = x > y ? y : x;
}
DEV uint64_t shfl_xor_u64(uint64_t v, int m) {
    const int lo = __shfl_xor((int)(uint32_t)v, m, 64);
    const int hi = __shfl_xor((int)(uint32_t)(v >> 32), m, 64);
    return ((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo;
}
// Sort N entries best first (bitonic network, N a power of two).
template <int N, typename V>
DEV void sort_desc(V (&a)[N]) {
#pragma unroll
    for (int size = 2; size <= N; size <<= 1)
#pragma unroll
        for (int stride = size / 2; stride > 0; stride >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int j = i ^ stride;
                if (j > i) {
                    if ((i & size) == 0 || size == N) order2(a[i], a[j]);
                    else order2(a[j], a[i]);
                }
            }
}
// a, b sorted best first: a becomes the best N of both, sorted (the
// elementwise better of a and reversed b is bitonic; half-cleaners sort it).
// `b` is left with the others, in no order.
template <int N, typename V>
DEV void merge_best(V (&a)[N], V (&b)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) order2(a[j], b[N - 1 - j]);
#pragma unroll
    for (int len = N / 2; len >= 1; len >>= 1)
#pragma unroll
        for (int j = 0; j < N; ++j)
            if ((j & len) == 0) order2(a[j], a[j + len]);
}
