// Sizes of the whole layer for a few tokens (few.hip): host and device code.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define FEW_FN __host__ __device__ inline
#else
#define FEW_FN inline
#endif

constexpr int FEW_MAX_T = 16;      // a column of the matrix products per token
constexpr int FEW_WGS = 512;       // workgroups, two to a CU
constexpr int FEW_UNIT = 256;      // rows of a weight that slices are counted in
constexpr int FEW_UP_COLS = 64, FEW_DOWN_COLS = 128;   // output columns of a tile
constexpr int FEW_LINE = 32;       // counters to a cache line
constexpr int FEW_ITEMS = 1024;    // slices of tiles that a product is cut into, about

// Slices of the d axis whose partial logits the router leaves; every workgroup of the
// second launch adds them all up.
constexpr int FEW_ROUTER_SLICES = 16;
FEW_FN int few_router_slices(int T, int d, int E) {
    int s = d / 64;
    const int most = 32768 / (T * E);
    if (s > most) s = most;
    return s < 1 ? 1 : s > FEW_ROUTER_SLICES ? FEW_ROUTER_SLICES : s;
}
// Slices of K that a product of `tiles` tiles and `units` units of K is cut into.
FEW_FN int few_slices(int tiles, int units) {
    if (tiles <= 0 || tiles >= FEW_ITEMS) return 1;
    const int s = (FEW_ITEMS + tiles - 1) / tiles;
    return s < units ? s : units;
}

struct FewLayout {
    long counters, part, up_part, h, y_part, total;    // byte offsets
    int ncounters, up_counters;
};
// counters: error word, items taken; tiles of H per expert slot (shared first),
// polled, so a line each; slices done per up tile, per down tile
FEW_FN FewLayout few_layout(long T, long d, long E, long k, long f, long fs) {
    const long slots = E < T * k ? E : T * k;
    const long up_tiles = slots * (f / FEW_UP_COLS) + fs / FEW_UP_COLS, down_tiles = d / FEW_DOWN_COLS;
    const long units = slots * (f / FEW_UNIT) + fs / FEW_UNIT;
    FewLayout L;
    long o = 0;
    auto take = [&](long bytes) {
        const long at = o;
        o += (bytes + 255) / 256 * 256;
        return at;
    };
    L.up_counters = (int)(up_tiles < FEW_ITEMS ? up_tiles : FEW_ITEMS);
    L.ncounters = (int)((2 + 257) * FEW_LINE + L.up_counters + down_tiles);
    L.counters = take(4l * L.ncounters);
    L.part = take(4l * FEW_ROUTER_SLICES * ((T * E + 3) / 4 * 4));
    // fewer than FEW_ITEMS tiles make fewer than twice as many slices
    L.up_part = take(2l * FEW_ITEMS * T * 2 * FEW_UP_COLS * 4);
    L.h = take(units * T * FEW_UNIT * 2 * 2);
    L.y_part = take((FEW_ITEMS + down_tiles) * T * FEW_DOWN_COLS * 4);
    L.total = o;
    return L;
}
