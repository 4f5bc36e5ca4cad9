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
constexpr int FEW_QUEUES = 8;
constexpr int FEW_LINE = 32;       // counters to a cache line

// Slices of the d axis whose partial logits the router leaves; every workgroup of the
// second launch adds them all up.
constexpr int FEW_ROUTER_SLICES = 16;
FEW_FN int few_router_slices(int T, int d, int E) {
    int s = d / 64;
    const int most = 32768 / (T * E);
    if (s > most) s = most;
    return s < 1 ? 1 : s > FEW_ROUTER_SLICES ? FEW_ROUTER_SLICES : s;
}
// Slices of K that a product of `tiles` tiles and `units` units of K is cut into: about
// FEW_UP_ITEMS or FEW_DOWN_ITEMS of them in all, of no fewer than 2 or 3 units each.
// Slices even out the CUs' shares, but each leaves its sums and the last one adds them
// up.  us by slices: up, 264 tiles of 28 units 1: 145, 2: 142, 4: 136, 7: 135, 14: 139; 288
// of 28 1: 207, 2: 171, 4: 164, 8: 168; 768 of 16 1: 250, 2: 273, 4: 277; 96 of 8 2: 35.4, 4: 33.6, 8:
// 37.7; down, 56 of 72 4: 187, 8: 170, 14: 165, 18: 164, 36: 168; 32 of 192 8: 268, 12: 281, 16: 253,
// 24: 250, 48: 267; 16 of 24 4: 35.6, 8: 33.6, 16: 35.0, 24: 37.9.
constexpr int FEW_UP_ITEMS = 1024, FEW_DOWN_ITEMS = 768;
FEW_FN int few_slices(int tiles, int units, int items, int least) {
    if (tiles <= 0) return 1;
    const int s = (items + tiles / 2) / tiles, most = units / least;
    return s < 2 || most < 2 ? 1 : s < most ? s : most;
}
// Sums that slices leave: tiles x slices (slices > 1) at most.
FEW_FN long few_sliced(long tiles, long items) { return items + (tiles < items ? tiles : items); }

struct FewLayout {
    long counters, part, up_part, h, y_part, total;    // byte offsets
    int ncounters, up_counters;
};
// counters: items taken, first items taken; tiles of H per expert slot (shared first),
// polled, so a line each; slices done per up tile, per down tile.
// All of it lies behind the workspace's first int32, the error word, from the next multiple
// of FEW_ALIGN bytes on: no cache line may hold what two tiles leave, or a workgroup that
// reads the one would go on reading the other as it was before it was there.
constexpr int FEW_ALIGN = 256;
FEW_FN FewLayout few_layout(long T, long d, long E, long k, long f, long fs) {
    const long slots = E < T * k ? E : T * k;
    const long up_tiles = slots * (f / FEW_UP_COLS) + fs / FEW_UP_COLS, down_tiles = d / FEW_DOWN_COLS;
    const long units = slots * (f / FEW_UNIT) + fs / FEW_UNIT;
    FewLayout L;
    long o = 0;                      // from the aligned address
    auto take = [&](long bytes) {
        const long at = o;
        o += (bytes + FEW_ALIGN - 1) / FEW_ALIGN * FEW_ALIGN;
        return at;
    };
    L.up_counters = (int)(up_tiles < FEW_UP_ITEMS ? up_tiles : FEW_UP_ITEMS);
    L.ncounters = (int)((1 + FEW_QUEUES + 257) * FEW_LINE + L.up_counters + down_tiles);
    L.counters = take(4l * L.ncounters);
    L.part = take(4l * FEW_ROUTER_SLICES * ((T * E + 3) / 4 * 4));
    L.up_part = take(few_sliced(up_tiles, FEW_UP_ITEMS) * T * 2 * FEW_UP_COLS * 4);
    L.h = take(units * T * FEW_UNIT * 2 * 2);
    L.y_part = take(few_sliced(down_tiles, FEW_DOWN_ITEMS) * T * FEW_DOWN_COLS * 4);
    L.total = o + FEW_ALIGN + 4;
    return L;
}
