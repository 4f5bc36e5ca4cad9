// Int8 expert products of small batches (decoding): few rows per expert, so a
// product is a stream of the experts' codes from HBM, as in skinny.hip, at half
// the bytes.
//
// The codes are K-contiguous, one row per output channel, which is the row
// operand of v_mfma_i32_16x16x64_i8 as it lies: lane (g, r) takes 16 bytes of
// row r at k 16 g.  A workgroup owns up to 16 TT rows (tokens) of one expert and
// 16 NR channels (up product: half of them gate rows, half the up rows of the
// same f range); its 4 waves take every fourth 128-byte piece of K, so together
// they walk each row through neighbouring memory, whole 128-byte lines each.
// A wave keeps D pieces in flight (D 2 NR loads of 16 bytes per lane), straight
// into registers: no two waves need the same codes.  The tokens' codes are the
// column operand, 16 tokens each, from L2 or LDS.  The waves' 32-bit integer
// sums are added through LDS (in any order: they are exact), then come the
// scales and the SwiGLU.
//
// Up to 16 tokens the products quantise their own activations where they fit
// LDS (QF): the codes of the tile's rows, in every workgroup again, while the
// first pieces of the weights are on their way; two launches less, of the five
// that a call of one token would have.  The shared expert's tiles ride in the
// same launch.
#include "common.h"
#include "i8_common.h"
#include "kernels.h"
#include "rules.h"

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

enum { SI_UP = 0, SI_DOWN = 1 };
constexpr int SI_NW = 4;             // waves per workgroup, each 1/4 of K
constexpr int SI_PIECE = 128;        // bytes of a row per wave and step

DEV void barrier_no_fence() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
DEV void lds_barrier() {             // LDS writes visible, loads from memory still in flight
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier_no_fence();
}

// The expert of tile slot `slot` and the tile's number in it, -1 past the last
// tile: every wave scans the plan's offsets.
DEV int find_tile(const I8SkinnyArgs &a, int slot, int lane, int &within) {
    int found = -1, cum = 0;
    within = 0;
    for (int base = 0; base < a.E && found < 0; base += 64) {
        const int ee = base + lane;
        const int cnt = ee < a.E ? a.offsets[ee + 1] - a.offsets[ee] : 0;
        const int tiles = cnt > 0 ? (cnt + a.bm - 1) / a.bm : 0;
        int x = tiles;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int y = __shfl_up(x, off, 64);
            if (lane >= off) x += y;
        }
        const int excl = cum + x - tiles;
        const unsigned long long m = __ballot(slot >= excl && slot < excl + tiles);
        if (m) {
            const int src = __builtin_ctzll(m);
            found = base + src;
            within = slot - __shfl(excl, src, 64);
        }
        cum += __shfl(x, 63, 64);
    }
    within = __builtin_amdgcn_readfirstlane(within);
    return __builtin_amdgcn_readfirstlane(found);
}
// Whether lane group g4 of an accumulator holds up channels (the up product's
// second 8 rows).
DEV bool up_half(int g4) { return g4 >= 2; }

DEV void load8(const uint16_t *p, float (&v)[8]) {
    const u32x4_t w = ld_u32x4(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = bf_lo(w[j]);
        v[2 * j + 1] = bf_hi(w[j]);
    }
}
DEV void load8(const float *p, float (&v)[8]) {
    const f32x8 w = ld_f32x8(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = w[j];
}

// Codes and scales of `rows` rows of K values (row i at src + at(i)) into LDS,
// rows at pitch K + 16 (16 rows read side by side touch different banks).
template <typename S, typename F>
DEV void quantise_tile(const S *__restrict__ src, F at, int rows, int K, uint8_t *codes, float *scale,
                       uint32_t (*amax)[SI_NW]) {
    const int tid = threadIdx.x;
    for (int i = 0; i < rows; ++i) {
        const S *x = src + at(i);
        uint32_t m = 0;
        for (int c = tid; c < K / 8; c += 64 * SI_NW) {
            float v[8];
            load8(x + 8 * c, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) m = umax(m, abs_bits(v[j]));
        }
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) m = umax(m, (uint32_t)__shfl_xor((int)m, s, 64));
        if ((tid & 63) == 0) amax[i][tid >> 6] = m;
    }
    lds_barrier();
    for (int i = 0; i < rows; ++i) {
        const S *x = src + at(i);
        const I8Scale s(umax(umax(amax[i][0], amax[i][1]), umax(amax[i][2], amax[i][3])));
        if (tid == 0) scale[i] = s.s;
        for (int c = tid; c < K / 8; c += 64 * SI_NW) {
            float v[8];
            load8(x + 8 * c, v);
            *reinterpret_cast<u32x2_t *>(codes + i * (K + 16) + 8 * c) =
                u32x2_t{pack_i8(s.code(v[0]), s.code(v[1]), s.code(v[2]), s.code(v[3])),
                        pack_i8(s.code(v[4]), s.code(v[5]), s.code(v[6]), s.code(v[7]))};
        }
    }
    lds_barrier();
}

template <int MODE, int TT, int NR, int D, bool QF>
__global__ __launch_bounds__(64 * SI_NW, 2) void skinny_i8_kernel(I8SkinnyArgs a) {
    constexpr bool UP = MODE == SI_UP;
    constexpr int GR = UP ? NR / 2 : NR;               // groups of 16 output columns
    static_assert(!QF || TT == 1, "rows quantised in LDS: one tile of 16");
    __shared__ __attribute__((aligned(16))) i32x4_t red[SI_NW][TT * NR][64];
    __shared__ float row_scale[16];
    __shared__ uint32_t amax[16][SI_NW];
    extern __shared__ __attribute__((aligned(16))) uint8_t codes[];   // QF: [bm][K + 16]
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g4 = lane >> 4;

    // ---------------- which rows, which channels ----------------
    const int b = (int)blockIdx.x;
    const bool sh = b < a.nshared;   // the shared expert's tiles come first
    const I8Product &g = sh ? a.shared : a.routed;
    const int ncol = g.N / (16 * GR);
    int e = 0, row0, row_end, ntile;
    if (sh) {
        row0 = b / ncol * a.bm;
        row_end = a.T;
        ntile = b % ncol;
    } else {
        const int slot = (b - a.nshared) / ncol;
        ntile = (b - a.nshared) % ncol;
        int within = 0;
        e = find_tile(a, slot, lane, within);
        if (e < 0) return;
        row0 = a.offsets[e] + within * a.bm;
        row_end = a.offsets[e + 1];
    }
    row_end = min(row_end, row0 + a.bm);
    const int K = g.K, n0 = ntile * 16 * GR;
    // row of the activations that plan row p reads (rows past the tile repeat its last)
    auto source_row = [&](int p) {
        p = min(p, row_end - 1);
        if (UP && !sh) {
            const int j = a.perm[min(max(p, 0), a.routed.rows - 1)];
            p = (j >= 0 && j < a.routed.rows) ? j / a.k : 0;
        }
        return min(max(p, 0), g.a_nrows - 1);
    };

    // ---------------- operands ----------------
    const int pieces = K / SI_PIECE;
    const uint8_t *wp[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j) {
        const bool up = UP && j >= GR;
        wp[j] = (up ? g.B2 : g.B) + ((long)e * g.N + n0 + 16 * (up ? j - GR : j) + r) * K + 16 * g4;
    }
    uint32_t xo[TT];                 // element offsets (the rows span under 2^32)
    if constexpr (!QF) {
#pragma unroll
        for (int t = 0; t < TT; ++t) xo[t] = (uint32_t)source_row(row0 + 16 * t + r) * (uint32_t)K + 16u * g4;
    }
    u32x4_t w[D][NR][2], x[D][TT][2];
    auto load = [&](int s, int u) {
        const int k0 = SI_PIECE * u;
        if constexpr (!QF) {
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) x[s][t][h] = ld_u32x4(g.A + (xo[t] + (uint32_t)(k0 + 64 * h)));
        }
#pragma unroll
        for (int j = 0; j < NR; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) w[s][j][h] = ld_u32x4(wp[j] + k0 + 64 * h);
    };
    i32x4_t acc[TT][NR];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int j = 0; j < NR; ++j) acc[t][j] = i32x4_t{0, 0, 0, 0};

#pragma unroll
    for (int s = 0; s < D; ++s)
        if (wave + SI_NW * s < pieces) load(s, wave + SI_NW * s);
    __builtin_amdgcn_sched_barrier(0);
    const int rows = row_end - row0;
    if constexpr (QF) {
        if constexpr (UP) quantise_tile(a.X, [&](int i) { return (long)source_row(row0 + i) * K; }, rows, K, codes, row_scale, amax);
        else quantise_tile(g.Hin, [&](int i) { return (long)source_row(row0 + i) * K; }, rows, K, codes, row_scale, amax);
    }
    const uint8_t *cr = codes + min(r, rows - 1) * (K + 16) + 16 * g4;
    auto mul = [&](int s, int u) {
        if constexpr (QF) {
#pragma unroll
            for (int h = 0; h < 2; ++h) x[s][0][h] = ld_u32x4(cr + SI_PIECE * u + 64 * h);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < NR; ++j)
#pragma unroll
                for (int t = 0; t < TT; ++t)
                    acc[t][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
                        __builtin_bit_cast(i32x4_t, w[s][j][h]), __builtin_bit_cast(i32x4_t, x[s][t][h]),
                        acc[t][j], 0, 0, 0);
    };
    for (int u = wave; u < pieces;) {
#pragma unroll
        for (int s = 0; s < D; ++s) {
            if (u < pieces) {
                mul(s, u);
                __builtin_amdgcn_sched_barrier(0);
                if (u + SI_NW * D < pieces) load(s, u + SI_NW * D);
                __builtin_amdgcn_sched_barrier(0);
            }
            u += SI_NW;
        }
    }

    // ---------------- sum over the waves, epilogue ----------------
    // accumulator layout: lane (g4, r), register q holds channel 4 g4 + q of its
    // group, for row r
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int j = 0; j < NR; ++j) red[wave][t * NR + j][lane] = acc[t][j];
    __syncthreads();
    for (int o = wave; o < TT * GR; o += SI_NW) {
        const int t = o / GR, j = o % GR, p = row0 + 16 * t + r;
        auto total = [&](int i) {
            i32x4_t v = red[0][i][lane];
#pragma unroll
            for (int q = 1; q < SI_NW; ++q) v += red[q][i][lane];
            return v;
        };
        if (p >= row_end) continue;
        const float rs = QF ? row_scale[r] : g.As[source_row(p)];
        const long col = n0 + 16 * j + 4 * g4, ch = (long)e * g.N + col;
        const f32x4_t s1 = *reinterpret_cast<const f32x4_t *>(g.Bs + ch);
        const i32x4_t v = total(t * NR + j);
        if constexpr (UP) {
            const f32x4_t s2 = *reinterpret_cast<const f32x4_t *>(g.Bs2 + ch);
            const i32x4_t u = total(t * NR + GR + j);
            f32x4_t h;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                h[q] = silu_f(rs * ((float)v[q] * s1[q])) * (rs * ((float)u[q] * s2[q]));
            *reinterpret_cast<f32x4_t *>(g.H + (long)p * g.N + col) = h;
        } else {
            float y[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = rs * ((float)v[q] * s1[q]);
            *reinterpret_cast<u32x2_t *>(g.C + (long)p * g.N + col) =
                u32x2_t{pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3])};
        }
    }
}

template <int MODE, int TT, int NR, int D, bool QF>
hipError_t launch(I8SkinnyArgs a, hipStream_t st) {
    const int cols = 16 * (MODE == SI_UP ? NR / 2 : NR);
    a.bm = TT > 1 ? 16 * TT : (a.T < 16 ? a.T : 16);
    a.nshared = a.shared.N > 0 ? (a.T + a.bm - 1) / a.bm * (a.shared.N / cols) : 0;
    const long grid = a.nshared + skinny_slots(a.routed.rows, a.E, a.bm) * (a.routed.N / cols);
    if (grid <= 0) return hipSuccess;
    const size_t lds = QF ? (size_t)a.bm * ((a.shared.N > 0 && a.shared.K > a.routed.K ? a.shared.K : a.routed.K) + 16) : 0;
    skinny_i8_kernel<MODE, TT, NR, D, QF><<<dim3((unsigned)grid), dim3(64 * SI_NW), lds, st>>>(a);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The same products without a split of K, for calls with tiles enough: what
// bounds a CU is then the lines it can have on their way, of weights and of
// activations alike (7 TB/s in all, whatever the tile), so the activations are
// fetched once per workgroup and its channels are many.
//
// NW waves own 16 channels each (up product: 8 gate rows and the up rows of
// the same columns) over all of K, their codes straight into registers, D
// pieces of 128 bytes per row in flight.  One more wave fetches the rows'
// codes, a piece of 16 TT rows at a time, into a ring of SX_D pieces in LDS by
// direct loads (whole 128-byte lines, chunk XOR (row >> 1) & 7); it is a wave of
// its own because loads return in order, and the activations, from L2, would
// wait for weights asked for long before.  One barrier per piece.
//
// With dense routing every expert's rows are the tokens, so a workgroup's
// columns may belong to two experts, or to the shared one, and NW is what deals
// the columns evenly to the CUs (skinny_i8_waves).
constexpr int SX_D = 4, SX_WAVES = 15;

#define LDS_AS __attribute__((address_space(3)))
template <int N>
DEV void wait_vmcnt() {
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

DEV void load_lds16(const uint8_t *src, uint8_t *dst) {
    __builtin_amdgcn_global_load_lds(src, (LDS_AS void *)dst, 16, 0, 0);
}

template <int MODE, int TT, int D>
__global__ __launch_bounds__(64 * (SX_WAVES + 1)) void stream_i8_kernel(I8SkinnyArgs a) {
    constexpr bool UP = MODE == SI_UP;
    constexpr int STAGE = 16 * TT * SI_PIECE, NXL = STAGE / 1024;
    __shared__ __attribute__((aligned(16))) uint8_t ring[SX_D * STAGE];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), NW = a.nw;
    const int r = lane & 15, g4 = lane >> 4;
    constexpr int WC = UP ? 8 : 16;                    // output columns per wave

    // ---------------- which rows, which channels ----------------
    const int b = (int)blockIdx.x;
    bool sh = b < a.nshared;         // the shared expert's tiles come first
    int e = 0, row0, row_end, col;   // col: the wave's first output column
    bool idle = wave >= NW;
    if (UP && a.dense) {
        row0 = 0;
        row_end = a.T;
        const int c = (b * NW + min(wave, NW - 1)) * WC, routed = a.E * a.routed.N;
        sh = c >= routed;
        e = sh ? 0 : c / a.routed.N;
        col = sh ? c - routed : c - e * a.routed.N;
        if (sh && col >= a.shared.N) {   // past the last column: along for the barriers
            idle = true;
            sh = false;
            e = col = 0;
        }
    } else {
        const int ncol = (sh ? a.shared.N : a.routed.N) / (WC * NW);
        if (sh) {
            row0 = b / ncol * a.bm;
            row_end = a.T;
            col = b % ncol;
        } else {
            const int slot = (b - a.nshared) / ncol;
            col = (b - a.nshared) % ncol;
            int within = 0;
            e = find_tile(a, slot, lane, within);
            if (e < 0) return;
            row0 = a.offsets[e] + within * a.bm;
            row_end = a.offsets[e + 1];
        }
        col = (col * NW + min(wave, NW - 1)) * WC;
    }
    row_end = min(row_end, row0 + a.bm);
    const I8Product &g = sh ? a.shared : a.routed;
    const int K = g.K, pieces = K / SI_PIECE;
    const bool tokens = UP && (a.dense || sh);         // the rows are the tokens in order
    auto source_row = [&](int p) {
        p = min(p, row_end - 1);
        if (UP && !tokens) {
            const int j = a.perm[min(max(p, 0), a.routed.rows - 1)];
            p = (j >= 0 && j < a.routed.rows) ? j / a.k : 0;
        }
        return min(max(p, 0), g.a_nrows - 1);
    };

    if (wave == NW) {
        // ---------------- the activations ----------------
        const uint8_t *xp[NXL];
#pragma unroll
        for (int i = 0; i < NXL; ++i) {
            const int row = 8 * i + (lane >> 3);
            xp[i] = g.A + (long)source_row(row0 + row) * K + 16 * ((lane & 7) ^ ((row >> 1) & 7));
        }
        auto issue = [&](int st) {
#pragma unroll
            for (int i = 0; i < NXL; ++i) {
                load_lds16(xp[i], ring + st * STAGE + i * 1024);
                xp[i] += SI_PIECE;
            }
        };
        for (int u = 0; u < SX_D - 1 && u < pieces; ++u) issue(u);
        for (int u = 0; u < pieces; ++u) {
            // piece u has arrived; after the barrier nobody reads u - 1
            if (u + SX_D - 1 <= pieces) wait_vmcnt<NXL * (SX_D - 2)>();
            else wait_vmcnt<0>();
            barrier_no_fence();
            if (u + SX_D - 1 < pieces) issue((u + SX_D - 1) % SX_D);
        }
        return;
    }

    // ---------------- the weights ----------------
    const bool up = UP && r >= 8;
    const uint8_t *wp = (up ? g.B2 : g.B) + ((long)e * g.N + col + (UP ? r & 7 : r)) * K + 16 * g4;
    u32x4_t w[D][2];
    auto load = [&](int s, int u) {
#pragma unroll
        for (int h = 0; h < 2; ++h) w[s][h] = ld_u32x4(wp + SI_PIECE * u + 64 * h);
    };
    i32x4_t acc[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[t] = i32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < D; ++s)
        if (s < pieces) load(s, s);
    __builtin_amdgcn_sched_barrier(0);
    for (int u0 = 0; u0 < pieces; u0 += D) {
#pragma unroll
        for (int s = 0; s < D; ++s) {
            const int u = u0 + s;
            if (u < pieces) {
                barrier_no_fence();
                const uint8_t *x = ring + u % SX_D * STAGE;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int t = 0; t < TT; ++t) {
                        const int row = 16 * t + r;
                        const u32x4_t xv = ld_u32x4(x + row * SI_PIECE + 16 * ((4 * h + g4) ^ ((row >> 1) & 7)));
                        acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
                            __builtin_bit_cast(i32x4_t, w[s][h]), __builtin_bit_cast(i32x4_t, xv), acc[t], 0, 0, 0);
                    }
                __builtin_amdgcn_sched_barrier(0);
                if (u + D < pieces) load(s, u + D);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    if (idle) return;

    // ---------------- epilogue ----------------
    // lane (g4, r), register q: channel row 4 g4 + q of the wave (up product:
    // rows 0..7 gate, 8..15 up), for row r of the tile
    const long ch = (long)e * g.N + col;
    const int first = UP && a.dense && !sh ? a.offsets[e] : 0;   // dense: plan row of token 0
#pragma unroll
    for (int t = 0; t < TT; ++t) {
        const int row = row0 + 16 * t + r;
        const bool live = row < row_end;
        const float rs = g.As[source_row(row)];
        if constexpr (UP) {
            const f32x4_t sc = *reinterpret_cast<const f32x4_t *>((up_half(g4) ? g.Bs2 : g.Bs) + ch + 4 * (g4 & 1));
            float v[4];
            f32x4_t h;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = rs * ((float)acc[t][q] * sc[q]);
#pragma unroll
            for (int q = 0; q < 4; ++q) h[q] = silu_f(v[q]) * shfl_xor_f(v[q], 32);
            // a dense plan row that a malformed plan would push past the buffer is left out
            const int p = first + row;
            if (live && !up_half(g4) && p >= 0 && p < g.rows)
                *reinterpret_cast<f32x4_t *>(g.H + (long)p * g.N + col + 4 * g4) = h;
        } else if (live) {
            const f32x4_t sc = *reinterpret_cast<const f32x4_t *>(g.Bs + ch + 4 * g4);
            float y[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = rs * ((float)acc[t][q] * sc[q]);
            *reinterpret_cast<u32x2_t *>(g.C + (long)row * g.N + col + 4 * g4) =
                u32x2_t{pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3])};
        }
    }
}

template <int MODE, int TT, int D>
hipError_t launch_stream(I8SkinnyArgs a, hipStream_t st) {
    constexpr int WC = MODE == SI_UP ? 8 : 16;
    a.bm = 16 * TT;
    a.dense = MODE == SI_UP && a.k == a.E && a.T <= a.bm;
    a.nw = (int)skinny_i8_waves(a.T, a.k, a.E, a.routed.N, a.shared.N, a.bm, WC, a.dense);
    long grid;
    if (a.dense) {
        a.nshared = 0;
        grid = ((long)a.E * a.routed.N + a.shared.N + WC * a.nw - 1) / (WC * a.nw);
    } else {
        a.nshared = a.shared.N > 0 ? (a.T + a.bm - 1) / a.bm * (a.shared.N / (WC * a.nw)) : 0;
        grid = a.nshared + skinny_slots(a.routed.rows, a.E, a.bm) * (a.routed.N / (WC * a.nw));
    }
    if (grid <= 0) return hipSuccess;
    stream_i8_kernel<MODE, TT, D><<<dim3((unsigned)grid), dim3(64 * (a.nw + 1)), 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_skinny_i8_up(const I8SkinnyArgs &a, int tt, bool quantise, hipStream_t st) {
    if (quantise) return launch<SI_UP, 1, 2, 4, true>(a, st);
    return tt > 1 ? launch_stream<SI_UP, 4, 6>(a, st) : launch_stream<SI_UP, 1, 6>(a, st);
}
hipError_t launch_skinny_i8_down(const I8SkinnyArgs &a, int tt, bool quantise, hipStream_t st) {
    if (quantise) return launch<SI_DOWN, 1, 2, 4, true>(a, st);
    return tt > 1 ? launch_stream<SI_DOWN, 4, 6>(a, st) : launch_stream<SI_DOWN, 1, 6>(a, st);
}
