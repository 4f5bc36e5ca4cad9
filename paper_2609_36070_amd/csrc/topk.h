// Sorting networks over packed 64-bit (rank key, expert id) entries, shared by
// the routers' selections.  A larger entry ranks higher; 0 is padding.
#pragma once

#include "common.h"

// put the better of a, b first
DEV void order2(uint64_t &a, uint64_t &b) {
    const bool sw = b > a;
    const uint64_t x = a, y = b;
    a = sw ? y : x;
    b = sw ? x : y;
}
DEV uint64_t shfl_xor_u64(uint64_t v, int m) {
    const int lo = __shfl_xor((int)(uint32_t)v, m, 64);
    const int hi = __shfl_xor((int)(uint32_t)(v >> 32), m, 64);
    return ((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo;
}
// Sort N entries best first (bitonic network, N a power of two).
template <int N>
DEV void sort_desc(uint64_t (&a)[N]) {
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
template <int N>
DEV void merge_best(uint64_t (&a)[N], uint64_t (&b)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) order2(a[j], b[N - 1 - j]);
#pragma unroll
    for (int len = N / 2; len >= 1; len >>= 1)
#pragma unroll
        for (int j = 0; j < N; ++j)
            if ((j & len) == 0) order2(a[j], a[j + len]);
}
