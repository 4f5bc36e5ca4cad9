// Which path a forward takes: rules on sizes alone, host code without HIP.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstddef>

// Small batches (skinny.hip): 16-row tiles per workgroup, 0 for the tile GEMMs.
//
// 64-row tiles from 17 tokens up: more rows per pass over the weights beat
// the smaller tiles' higher occupancy at every mean row count (128 experts, us
// with 16 / 32 / 64 rows: 256 tokens 306 / 284 / 280, 512: 393 / 338 / 315);
// up to 16 tokens no expert has more than 16 rows.
//
// Up to 64 rows per expert on average: there more experts take a second tile
// and the tile GEMMs catch up.  (us here / there) 128 experts of 768, d 2048:
// 512 tokens 276 / 333, 1000 330 / 353; 32 of 1536, d 4096: 100 tokens with a
// hot expert 259 / 334, 250 336 / 341; 200 of 768, one expert per token: 8000
// tokens 466 / 545, 12800 549 / 580.  The host sees the mean only, and an uneven
// load moves the crossing down: with a router bias of std 2 it lies near 40 rows
// (128 experts: 32 rows 167 / 185, 64 rows 237 / 216; 200 experts: 20 rows 182 /
// 201, 64 rows 325 / 271), and a router collapsed onto 8 of 128 experts runs 512
// tokens in 117 / 95.
//
// The shared expert's rows are all T tokens, re-reading its weights per 64 of
// them: past the first 64 its products count up to the routed ones' bound, T f_s
// <= 64 E f.  200 experts of 768, one per token, and a shared one of 2048 (us
// here / there): 4000 tokens (T f_s = 53 E f) 506 / 615, 8000 (107) 745 / 739,
// 12800 (171) 1003 / 892; of 1024: 8000 (53) 616 / 649, 12800 (85) 784 / 756; 32 of
// 1536 and one of 2048: 1000 (42) 387 / 418, 2000 (83) 512 / 506.
inline int skinny_tiles(long T, long k, long E, long f, long fs) {
    if (T <= 0) return 0;
    if (T <= 16) return 1;
    return T * k <= 64 * E && (T <= 64 || T * fs <= 64 * E * f) ? 4 : 0;
}
// Tokens past which skinny_tiles is 0 for every f and fs.
inline long skinny_max_tokens(long E, long k) { return 64 * E / k > 16 ? 64 * E / k : 16; }

// Tiles of bm rows that R routes to E experts fill at most.
inline long skinny_slots(long R, long E, long bm) { return (R < E ? R : E) + R / bm; }

// K slices of a small batch's up/gate product: its workgroups (64 columns of f
// each) run in rounds of the 256 CUs, so 288 of them (8 experts and a shared one
// of 2048 columns) take as long as 512.  K is split over two or four where that
// ends the launch earlier, if each slice keeps 1024 rows; the SwiGLU then moves to
// a launch of its own (4 us), the slices are at most five rounds and their sums
// take at most SK_SLICE_BYTES.
//
// Workgroups are counted for the experts that T balanced tokens reach, with a
// tenth for the ones they reach beyond that (if there are any left).  Slices that just fit one round do
// so only where the launch has no spare workgroups: those end at once and leave
// their CU to a second one.
//
// Forward at 1 / 2 / 4 slices (us), by workgroups: 16, d 5120: 36 / - / 25; 64, d
// 4096: 56 / 45 / 41; 96, d 2048: 32.5 / 30.2; 112, d 4096: 60 / 50 / 52; 128, d 2048:
// 40 / 37, with spare ones 42 / 45; 148, d 4096: 62 / 65 / 56; 288, d 7168: 1 token
// 186 / 169 / 160, 61 tokens 242 / 214 / 206; 344, d 7168: 186 / 175; 592, d
// 6144: whole call 326 / 315.  As many rounds
// either way: 175, d 4096: 71 / 82 / 78; 210: 73 / 70 / 79; 256: 92 / 96 / 100; 444: 139 /
// 144; 493, d 2048: 73 / 78.
constexpr long SK_SPLIT_MAX = 4;
constexpr size_t SK_SLICE_BYTES = size_t(48) << 20;

inline long skinny_max_slices(long d) {
    long s = 1;
    while (s < SK_SPLIT_MAX && d / (2 * s) >= 1024) s *= 2;
    return s;
}

inline int skinny_kslices(long T, long k, long E, long d, long f, long fs, long tt) {
    const long R = T * k, bm = 16 * tt, shared = (T + bm - 1) / bm * (fs / 64);
    double reached = E * (1.0 - std::pow(1.0 - (double)k / E, (double)T));
    if (reached < R / bm) reached = (double)(R / bm);
    const long wgs = (long)std::ceil(reached * (f / 64) - 1e-6) + shared;
    const long grid = skinny_slots(R, E, bm) * (f / 64) + shared;
    const long most = T <= bm ? (R < E ? R : E) * (f / 64) + shared : grid;   // T rows: one tile per expert
    long best = 1, rounds = (wgs + 255) / 256;        // of `best` slices each
    for (long s = 2; s <= skinny_max_slices(d); s *= 2) {
        const long n = wgs * s;
        if (wgs >= (s == 2 ? 640 : 320) || 8 * (size_t)s * ((size_t)R * f + (size_t)T * fs) > SK_SLICE_BYTES) break;
        const long r = n <= 252 ? 1 : n <= 256 ? 1 + (grid * s > 256) : (std::min(n + n / 10, most * s) + 255) / 256;
        if (r * best < rounds * s) {
            best = s;
            rounds = r;
        }
    }
    return (int)best;
}

// Int8, one token (skinny_i8.hip): rows whose codes fit the workgroups' LDS.
// Two launches in place of five (us here / the streaming kernels): 128 experts,
// top 8, d 2048, f 768 14.1 / 26; 64, top 4, d 4096, f 256 11.3 / 27.6; 32, top 8, and a
// shared one, d 7168, f 2048 79 / 98; 16, top 2, d 1024, f 512 9.4 / 20.6.
constexpr long TOKEN_I8_K = 8192, TOKEN_I8_LDS = 56 * 1024;
inline bool token_i8(long T, long d, long k, long f, long fs) {
    const long routes = k + (fs > 0), waves = routes < 16 ? routes : 16;
    return T == 1 && d <= TOKEN_I8_K && waves * ((f > fs ? f : fs) + 16) <= TOKEN_I8_LDS;
}

// Int8: 16-row tiles of the streaming products, or 0 for the tile products.  The
// two cross where the bf16 ones do if the up product's 256 x 256 tiles fill the
// CUs (us here / there): 128 experts of 768, d 2048, 48 rows each 191 / 205, 64 216
// / 210; 32 of 1536, d 4096, 48 175 / 199, 64 202 / 199, 96 244 / 210; 16 of 2048, d 7168,
// 64 209 / 213, 96 266 / 220.  With fewer tiles a launch of them is one round,
// whatever their rows: 8 of 1536, d 4096, 96 rows 87 / 91, 128 95.5 / 94; 16 of 768, d
// 2048, 96 52 / 58, 128 60.5 / 60.3; later where every expert has the same rows: 8 and
// a shared one of 2048, d 7168, 128 172 / 239, 192 223 / 246, 256 303 / 254; 12 of
// 512, d 5120, 192 101 / 173; 8 of 768, d 2048, 256 48 / 56, 384 65 / 58.
inline int skinny_i8_tiles(long T, long k, long E, long f, long fs) {
    const int t = skinny_tiles(T, k, E, f, fs);
    if (t || (E * f + fs) / 128 >= 256) return t;
    const long rows = k == E ? 192 : 96;
    return T > 0 && T * k <= rows * E && T * fs <= rows * E * f ? 4 : 0;
}

// Tokens past which skinny_i8_tiles is 0 for every f and fs.
inline long skinny_i8_max_tokens(long E, long k) { return std::max((k == E ? 192L : 96L) * E / k, 16L); }

// Waves of a streaming workgroup, 8 columns of f (up product) or 16 of d each.
// Four, unless
// - dense routing: the columns of all experts are dealt in any parts, and a CU's
//   time is the lines it fetches, its waves' weights (16 rows) and the tile's bm
//   rows of activations, in whole rounds of the 256 CUs (8 experts and a shared
//   one, d 7168, f 2048, up to 64 tokens: 91-106 us so, 100-129 with four, 111-131
//   with eight);
// - the up product of 64-row tiles, at most six workgroups of four to a CU: eight
//   halve the activations' lines (us with eight / four, 40 tokens to 8 of 48 of 1024:
//   d 2048 79 / 88, d 5120 166 / 178; 28 of 1536: 74 / 82, 158 / 162; 48 of 768: 73 /
//   76, 146 / 140; past that, 64 of 1024: 102 / 97, 203 / 208; 128 of 768, d 2048, 64
//   tokens 148 / 140; 16-row tiles, 14 tokens to 48 of 768: 61 / 58, 130 / 120).
//   The down product with eight: 3 us slower to 3 faster over the same shapes.
constexpr long SX_MAX_WAVES = 15;
inline long skinny_i8_waves(long T, long k, long E, long N, long Ns, long bm, bool up, bool dense) {
    if (dense) {
        long best = 4, cost = 0;
        for (long nw = 4; nw <= SX_MAX_WAVES; ++nw) {
            const long units = (E * N + Ns + 8 * nw - 1) / (8 * nw);
            const long c = (units + 255) / 256 * (16 * nw + bm);
            if (cost == 0 || c < cost) {
                cost = c;
                best = nw;
            }
        }
        return best;
    }
    const long R = T * k, tiles = std::max(std::min(R, E), R / bm);
    const long units = tiles * (N / 32) + (T + bm - 1) / bm * (Ns / 32);
    return up && bm > 16 && units <= 6 * 256 ? 8 : 4;
}

// Dense routing on few token tiles: the folded down product has one workgroup
// per 256 x 256 tile of Y and a K loop over every expert, so a short batch
// leaves most CUs idle (200 tokens at d 7168: 28 workgroups of 288 K steps).
// The experts' products can run as tiles of their own into fp32 instead, with a
// small kernel that adds them in the same order of experts.  That shortens the
// chain of K steps from E f / 64 to `rounds` f / 64, rounds of the 256 CUs
// that E products of Y's tiles take, and costs a write and a read of fp32
// products, (E + shared) T d of them.  A K step of 64 takes about 1.4 us and
// the fp32 traffic runs at about 4.5 TB/s, so the two meet near 12000 values
// per column of f that the chain is shorter by.  Forward, folded / in parts
// (us): 8 experts and a shared one of 2048, d 7168: 200 tokens 706 / 387, 500
// 737 / 494; 8 of 1024, d 1024: 2048 tokens 253 / 128, 8192 450 / 481; 16 of
// 2048, d 256: 8192 tokens 1194 / 636; 8 of 256, d 1024: 2048 tokens 84 / 68,
// 8192 125 / 203; 2 of 256, d 256: 30000 tokens 49 / 71; over 306 shapes of 2
// to 16 experts the line is at most 10 % off the better side.
// Up to 64 tiles of Y a product of its own runs in quarter tiles, which the folded
// one cannot, in about two thirds of the time; that is all there is to gain with
// one expert, and for the shared expert's part of the chain: 1 expert of 2048, d
// 256: 300 tokens 62 / 34, 16000 138 / 122; of 512, d 1024: 2000 tokens 33.6 / 32.2,
// 4000 36 / 40; of 256, d 256, and a shared one of 1024: 2000 tokens 53 / 45, 16000
// 99 / 101; 2 of 512 and one of 1024, d 1024: 2000 tokens 85 / 70.
// Only up to half of the CUs' worth of Y tiles: past them the folded product
// fills the chip itself.
constexpr long DENSE_PARTS_MAX = 128, DENSE_PARTS_VALUES = 12000;
constexpr long DENSE_QUARTER_MAX = 64, DENSE_QUARTER_VALUES = 4500;

inline bool dense_parts(long T, long d, long E, long k, long f, long fs) {
    const long nt = (T + 255) / 256 * (d / 256);
    if (k != E || T <= 0 || nt > DENSE_PARTS_MAX) return false;
    const long rounds = (E * nt + 255) / 256;
    const long quarters = nt <= DENSE_QUARTER_MAX ? DENSE_QUARTER_VALUES * (fs + (E == 1 ? f : 0)) : 0;
    return (E + (fs > 0)) * T * d <= DENSE_PARTS_VALUES * f * (E - rounds) + quarters;
}

// Experts padded to the routers' tiles.
inline long route_padded(long E) {
    long p = 16;
    while (p < E) p *= 2;
    return p;
}

// The one-launch router: it re-reads W_r per 16 tokens, so up to 2048 tokens,
// and larger batches keep their logits' summation order.  Its loads of several
// expert columns need them aligned in every row.
//
// Up to 64 experts at every d (us here / the other routers): 32 experts, d
// 4096: 1 token 8.7 / 16.2, 1000 11.7 / 19.3, 2000 12.0 / 19.4; 64, d 16384:
// 1 token 37 / 74, 2048 50 / 83.  Past that a wave's chain of steps is long (8
// waves, 16 rows of W_r a lane in flight at 256) while the split router deals d
// to 8 blocks, and the two cross between d 3584 and 6144, later for more routes
// per token, which the split router's second launch selects on few CUs.
// 128 experts, top 1: d 4608 16 tokens 15.5 / 15.0, 2048 20 / 23; d 5120 16.6 / 15.4;
// top 8: d 5120 20 / 19, 500 tokens 22 / 24; d 7168 25 / 21, 29 / 26.  256 experts,
// top 1: d 3584 20 / 21, 28 / 29; d 4096 2048 tokens 32 / 30; d 4608 36 / 30; top 8:
// d 4608 30 / 30, 41 / 41; d 5120 740 tokens 34 / 40, 2048 45 / 41; d 7168 57 / 44;
// top 16, d 5120: 55 / 62.  W_r, re-read per 16 tokens, counts too: top 8, d 5120,
// 2048 tokens to 160 experts 38 / 42, 1600 to 200 40 / 42, to 256 44 / 43.  Over
// 3400 measured shapes at most 4 % (0.6 us) slower.
constexpr long ROUTE_DIRECT_MAX = 2048, ROUTE_DIRECT_ROWS = 160 * 2048;

inline bool route_direct(long T, long d, long E, long k) {
    const long ep = route_padded(E), cols = ep / 16 < 8 ? ep / 16 : 8;
    if (T <= 0 || T > ROUTE_DIRECT_MAX || E % cols) return false;
    if (ep <= 64) return true;
    if (ep == 128) return d <= (k >= 8 ? 5120 : 4608);
    const long top = k >= 8 ? 4608 : k >= 4 ? 4096 : 3584;
    return d <= top + (k >= 16 || (k >= 4 && T * E <= ROUTE_DIRECT_ROWS) ? 512 : 0);
}

// Logits for a selection by scores (score.hip), few tokens: the one-launch
// router's blocks on slices of the d axis, so that about all CUs read W_r; the
// selection adds the slices.  0: the other routers.
//
// A block reads its slice of W_r for 16 tokens, so the two cross by T d E (us with
// the selection, here / the others).  256 experts, d 7168: 1 token 11.5 / 22.4, 512
// 21.5 / 27, 1024 27.5 / 27.5, 1500 38 / 29; d 4096: 1024 20.7 / 21.1, 1500 26 / 22.5; d 2048:
// 2048 20.7 / 20.5, 3000 26 / 23.  128, d 7168: 1024 16.5 / 18.2, 1500 20.7 / 18.6; d 2048:
// 4096 16.4 / 19, 6000 23.6 / 20.  Up to 64 experts the others are slower: 64, d 7168:
// 1024 14.5 / 42, 4096 27 / 44, 6000 50 / 73, 8192 59 / 53; 32, d 4096: 1 token 8 / 15, 4096
// 15 / 20, 8192 22 / 28, 16384 49 / 41; 16, d 2048: 4096 14.3 / 16, 8192 19.4 / 18.5.
constexpr long ROUTE_SLICE_MAX = 8192, ROUTE_SLICE_BLOCKS = 256;

inline bool route_sliced(long T, long d, long E) {
    const long ep = route_padded(E), cols = ep / 16 < 8 ? ep / 16 : 8;
    if (T <= 0 || E % cols) return false;
    if (ep >= 128) return T <= 1024 || (T <= 4096 && T * d * ep <= 1L << 30);
    return T <= ROUTE_SLICE_MAX && T <= 256 * ep && T * d * ep <= 3L << 30;
}
inline long route_slice_steps(long d, long E) {      // slices of one step of 32 rows per wave
    const long nw = route_padded(E) <= 64 ? 16 : 8;
    const long s = d / 32 / nw;
    return s > 1 ? s : 1;
}
inline long route_slices(long T, long d, long E) {
    if (!route_sliced(T, d, E)) return 0;
    const long fill = ROUTE_SLICE_BLOCKS / ((T + 15) / 16), most = route_slice_steps(d, E);
    return std::max(std::min(fill, most), 1L);
}
// Rows of partial logits of any batch of up to T tokens.
inline long route_slice_rows(long T, long d, long E) {
    const long t = T < ROUTE_SLICE_MAX ? T : ROUTE_SLICE_MAX;
    return std::min(t * route_slice_steps(d, E), 16 * ROUTE_SLICE_BLOCKS);
}

// Larger batches of more than 64 experts: tiles of 128 tokens, their d axis in
// slices that divide its chunks of 64.  More slices fill the 256 CUs, or end the last
// round earlier, and cost a write and a read of their partial logits, which take
// the time of a chunk per 27 tiles; a tile's first loads and its epilogue take three
// chunks'.  Up to three rounds of tiles: past them a round is a small part, and the
// partial logits would be the larger part of a workspace.
//
// Router by 1 / 2 / 4 / 8 slices (us): 256 experts, d 512: 9000 tokens 31.5 / 29.7 / 37 /
// 43, 65536 92 / 114 / 157 / 276; d 1024: 8192 37 / 28 / 31 / 40; d 2048: 16384 54 / 45 / 54
// / 73; d 7168: 4200 109 / 64 / 45 / 51 (7: 38), 16384 121 / 89 / 99 / 119, 33000 263 / 225 /
// 221 / 264, 65536 323 / 363 / 402 / 492.  128 experts: d 256: 4200 16.8 / 15.7 / 17.5, 24000
// 23.8 / 29.8 / 35; d 2048: 16384 32 / 28 / 36 / 47, 20000 34 / 39 / 43 / 53; d 7168: 40000 181 /
// 164 / 171 / 201.  Over 480 shapes of 96 to 256 experts, d 256 to 7168 and 1100 to 65536
// tokens at most 14 % off the best count, 1 % on average (by rounds alone 180 and 23 %).
constexpr long ROUTE_TILE = 128, ROUTE_TILE_SLOTS = 768, ROUTE_TILE_MIN = 128;

// The slices for n tiles of d.
struct RouteTiles {
    double round[9];         // a round's time in chunks, by slices; 0: they do not divide
    explicit RouteTiles(long d) {
        const long chunks = d / 64;
        for (long s = 1; s <= 8; ++s) round[s] = chunks % s ? 0.0 : 3.0 + (double)(chunks / s);
    }
    long slices(long n) const {
        long best = 1;
        double least = (double)((n + 255) / 256) * round[1];
        for (long s = 2; s <= 8 && n * s <= ROUTE_TILE_SLOTS; ++s) {
            if (round[s] == 0.0) continue;
            const double c = (double)((n * s + 255) / 256) * round[s] + 0.037 * (double)(n * s);
            if (c < least) {
                least = c;
                best = s;
            }
        }
        return best;
    }
    // moe_route's, which selects in a launch of its own for partial logits alone:
    // doubled until the tiles fill the CUs
    long split_slices(long n) const {
        long s = 1;
        while (s < 8 && n * s < 256 && round[2 * s] != 0.0) s *= 2;
        return s;
    }
};
inline long route_tiles(long T) { return (T + ROUTE_TILE - 1) / ROUTE_TILE; }
// 0: no tiles for so few experts
inline long route_tile_slices(long T, long d, long E) {
    return route_padded(E) < ROUTE_TILE_MIN ? 0 : RouteTiles(d).slices(route_tiles(T));
}
inline long route_split_slices(long T, long d, long E) {
    return route_padded(E) < ROUTE_TILE_MIN ? 0 : RouteTiles(d).split_slices(route_tiles(T));
}
// Rows of partial logits of any batch of up to T tokens, for either router.
inline long route_part_rows(long T, long d, long E) {
    long rows = route_slice_rows(T, d, E);
    if (route_padded(E) < ROUTE_TILE_MIN) return rows;
    const RouteTiles r(d);
    // no slices past SLOTS / 2 tiles, and no more than 8 of fewer
    for (long n = std::min(route_tiles(T), ROUTE_TILE_SLOTS / 2); n > 0 && 8 * ROUTE_TILE * n > rows; --n) {
        const long s = std::max(r.slices(n), r.split_slices(n));
        if (s > 1) rows = std::max(rows, s * std::min(ROUTE_TILE * n, T));
    }
    return rows;
}

// The third LDS stage of B in a row product of `rows` rows over `groups` experts
// (DEEP in gemm.hip) pays while an expert's weights serve few m-tiles and costs
// a little where they serve many (its loads then hit in L2 either way, and more
// of them queue).  Forward, two / three stages (us), mean rows per expert: 125:
// 394 / 369, 512 (128 experts): 906 / 878, 1000: 1315 / 1291, 1024 (128 experts):
// 1570 / 1541, 2048: 2461 / 2453, 3000: 3580 / 3607, 4096: 4752 / 4777.
//
// Short products have no K steps to hide it in: with 4 or 8 of 64 the loads
// ahead are the whole product, and its tiles start later.  Forward that keeps
// its activations, d = f, two / three stages (us): K 256, 128 experts: 16 rows
// 34.3 / 35.3, 300 76.5 / 77.9; K 512: 16 rows 67.7 / 69.8, 100 79.4 / 81.1, 300
// 164 / 161, 900 378 / 368; K 768: 16 rows 149 / 151, 300 326 / 311; K 1024, 64
// experts: 16 rows 124 / 119, 300 267 / 253.
constexpr long DEEP_ROWS = 1024, DEEP_K = 768, DEEP_SHORT_K = 512, DEEP_SHORT_ROWS = 200;

inline bool deep_stages(long K, long rows, long groups) {
    const long n = groups > 0 ? groups : 1;
    if (rows > DEEP_ROWS * n) return false;
    return K >= DEEP_K || (K >= DEEP_SHORT_K && rows >= DEEP_SHORT_ROWS * n);
}

// The MXFP8 up/gate product's kept pre-activations (fp32, two values per element
// of H) go past the L2, as every other output (gemm_mx.hip).  Not where they fit
// the Infinity Cache beside little else: a short K loop then waits for these
// stores, and past the L2 they run at 2.4 TB/s instead of 3.5.  Forward that keeps
// them, past / through the L2 (us): d 256, 1500 rows of 8 experts, f 1024 (98 MB)
// 87 / 79, f 2048 (197 MB) 139 / 124; d 512, f 1536 125 / 113; d 1024, f 1024 116 / 106,
// f 2048 189 / 186; d 2048, f 1536 224 / 232.  Fewer rows (256 of 32 experts, d 1024,
// f 1536: 122 / 134), smaller (49 MB, d 256: 56 / 58) and larger (393 MB, d 512: 0.92
// of the time) are faster past it.
inline bool mx_keep_l2(long R, long E, long K, long N) {
    const long bytes = 8 * R * N;
    return K <= 1024 && R >= 1024 * E && bytes >= (64L << 20) && bytes <= (208L << 20);
}

// The whole layer for a few tokens (few.hip): weights that are more than the 256 MB of the
// memory's cache are loaded past it.  us through the caches / past them, the calls taking
// turns on 4 sets of weights: 76 MB 37.5 / 37.9, 152 MB 53.3 / 51.3, 353 MB 94 / 88, 500 MB 120
// / 114, 794 MB 177 / 167; on one set, which the cache holds up to there: 76 MB 32.8 / 36.6, 152
// MB 45.9 / 51.2, 202 MB 52 / 60, 353 MB 88 / 88.
inline bool few_past_caches(long T, long d, long E, long k, long f, long fs) {
    const double reached = E * (1.0 - std::pow(1.0 - (double)k / E, (double)T));
    return 6.0 * d * (reached * f + fs) > 256e6;
}

// Joining a block to the residual stream (join.hip): rows up to which a row gets
// as many threads as have something to load.
constexpr long JOIN_FEW_ROWS = 256;
// The forward: one workgroup of 1024 threads to a CU, with the weights in LDS, if it has 12
// rounds of rows (us, a workgroup per 1 to 4 rows / this: 16384 x 7168 211 / 189, in fp32 291 /
// 257; 8192 x 4096 66 / 61; 16384 x 2048 59 / 57; 6001 x 2048 31.7 / 32.8; 2100 x 7168 26 / 30).  A
// norm alone has little to read again: 4099 x 4096 13.7 / 17.2.
inline bool join_forward_rows(long T, long d, int weights, bool block) {
    const long rows = d <= 1024 ? 8 : d <= 2048 ? 4 : 2;     // of a workgroup at a time
    return block && d > 512 && d <= 8192 && T >= 12 * 256 * rows && weights * d * 4 <= 144 * 1024;
}
// Row lengths: what a workgroup's registers hold; with the sums over the rows beside it.
constexpr long JOIN_MAX_D = 16384, JOIN_SUMS_D = 8192;
// The backward: threads of a row (8 values each up to 4096), of a workgroup, and the
// workgroups, which leave a row of sums each.  Up to 512 of them (384 of longer rows) have rows
// for one round and read the weights where they lie (us, 256 with several rounds / these: 600 x
// 1000 15.3 / 13.6, 1024 x 1000 15.7 / 15.5, 512 x 2048 17.7 / 16.3, 300 x 4096 20.2 / 18.1, 512 x 4096 20.4
// / 22.9, 300 x 7168 39 / 29; 800 x 2048 20.7 / 20.7, 800 x 7168 60 / 64).  Beyond, one to a CU where a
// row takes 512 threads, else three, if each has 4 rounds of rows left (us with 256 / 768: 16384 x
// 2048 116 / 100, 20000 x 1024 75 / 66, 40000 x 512 80 / 67, 100000 x 64 114 / 29, 4000 x 2048 32 / 34).
// Two rounds of rows go to one workgroup up to 4096 columns: it writes the sums itself, without
// the launch that adds them up (us, 2 workgroups / one: 64 rows of 64 11 / 9.0, 2 of 2048
// 10.2 / 8.7, 2 of 4096 10.2 / 10.0, 2 of 7168 12 / 19).
inline long join_row_threads(long d) {
    long g = 8;
    while (g < 512 && 8 * g < d) g *= 2;
    return g;
}
inline long join_threads(long d) { return join_row_threads(d) < 256 ? 256 : join_row_threads(d); }
inline long join_rows(long d) { return join_threads(d) / join_row_threads(d); }   // of a workgroup
inline long join_workgroups(long T, long d) {
    const long n = (T + join_rows(d) - 1) / join_rows(d);
    if (n <= 2 && d <= 4096) return 1;
    if (n <= (d <= 2048 ? 512 : d <= JOIN_SUMS_D ? 384 : 256)) return n;
    return std::min(d <= 2048 ? 768L : 256L, std::max(256L, n / 4));
}
// At least as many, and never fewer for more rows: what the workspace is made for.
inline long join_part_rows(long T, long d) {
    return std::min((T + join_rows(d) - 1) / join_rows(d), d <= 2048 ? 768L : 384L);
}
