// Int8 expert products of small batches (decoding): few rows per expert, so a
// product is a stream of the experts' codes from HBM, as in skinny.hip, at half
// the bytes.  The codes are K-contiguous, one row per output channel, which is
// the row operand of v_mfma_i32_16x16x64_i8 as it lies: lane (g, r) takes 16
// bytes of row r at k 16 g.  The activations' codes are the column operand.
#include "common.h"
#include "i8_common.h"
#include "kernels.h"
#include "rules.h"

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

enum { SI_UP = 0, SI_DOWN = 1 };
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
DEV uint32_t max8(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = umax(m, abs_bits(v[j]));
    return m;
}
DEV uint32_t wave_max(uint32_t m) {
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) m = umax(m, (uint32_t)__shfl_xor((int)m, s, 64));
    return m;
}
DEV void put8(uint8_t *codes, const float (&v)[8], const I8Scale &s) {
    *reinterpret_cast<u32x2_t *>(codes) =
        u32x2_t{pack_i8(s.code(v[0]), s.code(v[1]), s.code(v[2]), s.code(v[3])),
                pack_i8(s.code(v[4]), s.code(v[5]), s.code(v[6]), s.code(v[7]))};
}

// ---------------------------------------------------------------------------
// One token: two launches in all, without the plan (the experts are the
// token's own list).  What counts is latency: every load that a wave will need
// goes out at once, and the workgroups quantise the activations for
// themselves, each the same row again, under the weights' round trip.  8 of 128
// experts of 768, d 2048, 25 and 13 MB of codes: 14.2 us together, 15.8 with the
// scales asked for where they are used and the activations behind the expert's id.
//
// Up product: a workgroup owns 8 columns of f of one of the token's experts (or
// of the shared one), 8 gate and 8 up rows in one operand; its 4 waves take every
// fourth 128-byte piece of K.  (16 columns: half as many workgroups, uneven over
// the CUs; with them one token to 8 of 128 experts of 768, d 2048, took 16.05 us in
// both launches, so 15.75.)
constexpr int TK_NW = 4, TK_D = 8;
constexpr int TK_HELD = TOKEN_I8_K / 8 / (64 * TK_NW);   // 8-value chunks of the token per thread

__global__ __launch_bounds__(64 * TK_NW) void token_up_kernel(I8SkinnyArgs a) {
    __shared__ __attribute__((aligned(16))) uint8_t codes[TOKEN_I8_K];
    __shared__ int red[TK_NW][16];
    __shared__ uint32_t amax[TK_NW];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g4 = lane >> 4;
    const int ns = a.shared.N / 8, b = (int)blockIdx.x - ns;
    const bool sh = b < 0;
    const I8Product &g = sh ? a.shared : a.routed;
    const int slot = sh ? 0 : b / (g.N / 8);
    const int n0 = 8 * (sh ? b + ns : b % (g.N / 8));
    const int K = g.K, pieces = K / SI_PIECE;

    // loads return in order: the token first, then the weights, then their scales
    int e = sh ? 0 : a.topk_idx[slot];
    float v[TK_HELD][8];
#pragma unroll
    for (int i = 0; i < TK_HELD; ++i) {
        const int c = tid + 64 * TK_NW * i;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        if (c < K / 8) load8(a.X + 8 * c, v[i]);
    }
    __builtin_amdgcn_sched_barrier(0);
    e = __builtin_amdgcn_readfirstlane(e);
    if (e < 0 || e >= a.E) return;   // routes outside the experts are left out
    const uint8_t *wp = (r < 8 ? g.B : g.B2) + ((long)e * g.N + n0 + (r & 7)) * K + 16 * g4;
    u32x4_t w[TK_D][2];
    auto load = [&](int s, int u) {
#pragma unroll
        for (int h = 0; h < 2; ++h) w[s][h] = ld_u32x4(wp + SI_PIECE * u + 64 * h);
    };
#pragma unroll
    for (int s = 0; s < TK_D; ++s)
        if (wave + TK_NW * s < pieces) load(s, wave + TK_NW * s);
    const long channel = (long)e * g.N + n0 + (tid & 7);
    const float gate_s = g.Bs[channel], up_s = g.Bs2[channel];
    __builtin_amdgcn_sched_barrier(0);

    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < TK_HELD; ++i) m = umax(m, max8(v[i]));
    m = wave_max(m);
    if (lane == 0) amax[wave] = m;
    lds_barrier();
    const I8Scale xs(umax(umax(amax[0], amax[1]), umax(amax[2], amax[3])));
#pragma unroll
    for (int i = 0; i < TK_HELD; ++i) {
        const int c = tid + 64 * TK_NW * i;
        if (c < K / 8) put8(codes + 8 * c, v[i], xs);
    }
    lds_barrier();

    i32x4_t acc = i32x4_t{0, 0, 0, 0};
    for (int u = wave; u < pieces;) {
#pragma unroll
        for (int s = 0; s < TK_D; ++s) {
            if (u < pieces) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // every column of the product is the token
                    const u32x4_t x = ld_u32x4(codes + SI_PIECE * u + 64 * h + 16 * g4);
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, w[s][h]),
                                                                __builtin_bit_cast(i32x4_t, x), acc, 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (u + TK_NW * TK_D < pieces) load(s, u + TK_NW * TK_D);
                __builtin_amdgcn_sched_barrier(0);
            }
            u += TK_NW;
        }
    }
    // lane (g4, r), register q: row 4 g4 + q, whatever r
    if (r == 0)
#pragma unroll
        for (int q = 0; q < 4; ++q) red[wave][4 * g4 + q] = acc[q];
    __syncthreads();
    if (tid < 8) {
        int gate = 0, up = 0;
#pragma unroll
        for (int q = 0; q < TK_NW; ++q) {
            gate += red[q][tid];
            up += red[q][8 + tid];
        }
        g.H[(long)slot * g.N + n0 + tid] =
            silu_f(xs.s * ((float)gate * gate_s)) * (xs.s * ((float)up * up_s));
    }
}

// Down product and the sum over the token's experts: a workgroup owns COLS
// columns of Y (8 where 16 would leave CUs without one), a wave of it one of the
// token's routes (the shared expert first): the route's row of H to LDS as
// codes, its channels over all of f, and the weighted result to LDS in fp32.  The
// sum runs in the routes' order and is rounded once.
constexpr int TK_DD = 6;
template <int COLS>
__global__ __launch_bounds__(1024) void token_down_kernel(I8SkinnyArgs a, const float *__restrict__ topk_w,
                                                          uint16_t *__restrict__ Y, int pitch) {
    extern __shared__ __attribute__((aligned(16))) uint8_t codes_all[];   // [waves][pitch]
    __shared__ float y[32][16];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
    const int r = lane & 15, g4 = lane >> 4;
    const int n0 = COLS * (int)blockIdx.x, nsh = a.shared.N > 0 ? 1 : 0, routes = a.k + nsh;
    uint8_t *codes = codes_all + wave * pitch;
    for (int s0 = wave; s0 < routes; s0 += nw) {
        const bool sh = s0 < nsh;
        const I8Product &g = sh ? a.shared : a.routed;
        const int slot = s0 - nsh, K = g.K, pieces = K / SI_PIECE;
        int e = sh ? 0 : a.topk_idx[slot];
        const float wt = sh ? 1.0f : topk_w[slot];
        const float *h = g.Hin + (sh ? 0 : (long)slot * K);
        // the row's largest value: the first 2048 values stay in registers
        float v[4][8];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = lane + 64 * i;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
            if (c < K / 8) load8(h + 8 * c, v[i]);
        }
        __builtin_amdgcn_sched_barrier(0);
        e = __builtin_amdgcn_readfirstlane(e);
        if (e < 0 || e >= a.E) {
            if (lane < 16) y[s0][lane] = 0.f;
            continue;
        }
        const uint8_t *wp = g.B + ((long)e * g.N + n0 + (r & (COLS - 1))) * K + 16 * g4;
        u32x4_t w[TK_DD][2];
        auto load = [&](int s, int u) {
#pragma unroll
            for (int q = 0; q < 2; ++q) w[s][q] = ld_u32x4(wp + SI_PIECE * u + 64 * q);
        };
#pragma unroll
        for (int s = 0; s < TK_DD; ++s)
            if (s < pieces) load(s, s);
        const f32x4_t sc = *reinterpret_cast<const f32x4_t *>(g.Bs + (long)e * g.N + n0 + (4 * g4 & (COLS - 1)));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) m = umax(m, max8(v[i]));
        for (int c = lane + 256; c < K / 8; c += 64) {
            float u[8];
            load8(h + 8 * c, u);
            m = umax(m, max8(u));
        }
        const I8Scale hs(wave_max(m));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = lane + 64 * i;
            if (c < K / 8) put8(codes + 8 * c, v[i], hs);
        }
        for (int c = lane + 256; c < K / 8; c += 64) {
            float u[8];
            load8(h + 8 * c, u);
            put8(codes + 8 * c, u, hs);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the wave's own codes
        i32x4_t acc = i32x4_t{0, 0, 0, 0};
        for (int u0 = 0; u0 < pieces; u0 += TK_DD) {
#pragma unroll
            for (int s = 0; s < TK_DD; ++s) {
                const int u = u0 + s;
                if (u < pieces) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const u32x4_t x = ld_u32x4(codes + SI_PIECE * u + 64 * q + 16 * g4);
                        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, w[s][q]),
                                                                    __builtin_bit_cast(i32x4_t, x), acc, 0, 0, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    if (u + TK_DD < pieces) load(s, u + TK_DD);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if (r == 0 && 4 * g4 < COLS) {
#pragma unroll
            for (int q = 0; q < 4; ++q) y[s0][4 * g4 + q] = wt * (hs.s * ((float)acc[q] * sc[q]));
        }
    }
    __syncthreads();
    if (tid < COLS) {
        float sum = 0.f;
        for (int s = 0; s < routes; ++s) sum = sum + y[s][tid];
        Y[n0 + tid] = f2bf(sum);
    }
}

// ---------------------------------------------------------------------------
// Several tokens: up to 16 TT rows of one expert per workgroup.  What bounds a CU
// here is the lines it can have on their way, of weights and of activations
// alike (7 TB/s in all, whatever the tile), so the activations are fetched once
// per workgroup and its channels are many.
//
// NW waves own 16 channels each (up product: 8 gate rows and the up rows of
// the same columns) over all of K, their codes straight into registers, D
// pieces of 128 bytes per row in flight.  One more wave fetches the rows'
// codes, a piece of 16 TT rows at a time, into a ring of SX_D pieces in LDS by
// direct loads (whole 128-byte lines, chunk XOR (row >> 1) & 7); it is a wave of
// its own because loads return in order, and the activations, from L2, would
// wait for weights asked for long before.  One barrier per piece.  16 tokens to 8 of
// 32 experts of 1536, d 4096: up 79 us for 403 MB of codes, down 39 for 201 (5 TB/s;
// a large copy reaches 5.2); 61 tokens, 8 experts and a shared one of 2048, d 7168:
// up 55 us for 264 MB, down 36 for 132.
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
            // fp32 for the sum over a token's experts, as for one token: few rows, 0 to 3 %
            // of a call (16 tokens to 8 of 32 experts 136.3 -> 137.8 us, 61 to 8 and a
            // shared one 105.8 -> 107.1, 512 to 8 of 128 165 -> 170)
            f32x4_t y;
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = rs * ((float)acc[t][q] * sc[q]);
            *reinterpret_cast<f32x4_t *>(g.Cf + (long)row * g.N + col + 4 * g4) = y;
        }
    }
}

template <int MODE, int TT, int D>
hipError_t launch_stream(I8SkinnyArgs a, hipStream_t st) {
    constexpr int WC = MODE == SI_UP ? 8 : 16;
    a.bm = 16 * TT;
    a.dense = MODE == SI_UP && a.k == a.E && a.T <= a.bm;
    a.nw = (int)skinny_i8_waves(a.T, a.k, a.E, a.routed.N, a.shared.N, a.bm, MODE == SI_UP, a.dense);
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

hipError_t launch_skinny_i8_up(const I8SkinnyArgs &a, int tt, hipStream_t st) {
    return tt > 1 ? launch_stream<SI_UP, 4, 4>(a, st) : launch_stream<SI_UP, 1, 4>(a, st);
}
hipError_t launch_skinny_i8_down(const I8SkinnyArgs &a, int tt, hipStream_t st) {
    return tt > 1 ? launch_stream<SI_DOWN, 4, 4>(a, st) : launch_stream<SI_DOWN, 1, 4>(a, st);
}

hipError_t launch_token_i8_up(const I8SkinnyArgs &a, hipStream_t st) {
    const int grid = a.shared.N / 8 + a.k * (a.routed.N / 8);
    token_up_kernel<<<dim3((unsigned)grid), dim3(64 * TK_NW), 0, st>>>(a);
    return hipGetLastError();
}
hipError_t launch_token_i8_down(const I8SkinnyArgs &a, const float *topk_w, uint16_t *Y, hipStream_t st) {
    const int routes = a.k + (a.shared.N > 0), nw = routes < 16 ? routes : 16;
    const int pitch = (a.shared.K > a.routed.K ? a.shared.K : a.routed.K) + 16;
    const dim3 block(64 * nw);
    const size_t lds = (size_t)nw * pitch;
    if (a.routed.N / 16 < 256)
        token_down_kernel<8><<<dim3((unsigned)(a.routed.N / 8)), block, lds, st>>>(a, topk_w, Y, pitch);
    else
        token_down_kernel<16><<<dim3((unsigned)(a.routed.N / 16)), block, lds, st>>>(a, topk_w, Y, pitch);
    return hipGetLastError();
}
