// Grouped int8 products of the experts on v_mfma_i32_32x32x32_i8.  Per expert
// e and buffer positions p of e's region (the shared expert: the tokens as
// they are, in the same launch):
//
//   I8_UP    g = sx sg[n] (Xq[tok(p)] . Wg_q[e][n]), u likewise;
//            H = silu(g) u in fp32, for the row quantiser
//   I8_DOWN  Yexp = sh sd[n] (Hq[p] . Wd_q[e][n]) -> bf16
//
// Every operand is a matrix of K-contiguous byte rows with one fp32 scale per
// row.  The dot products are exact in 32-bit integers (K <= 131072: 127^2 K
// stays below 2^31) and rounded once, to fp32, when the scales are applied.
//
// 256 x 256 block tile, K step 128 bytes, two LDS stages filled by direct
// global->LDS loads (128-byte rows, chunk XOR (row >> 1) & 7), 8 waves of 128 x 64
// (two per SIMD), tiles rastered XCD-aware.  The MFMA takes 16 consecutive
// bytes of row l % 32 from lane l, at k 16 (l / 32) of its 32.
#include "common.h"
#include "i8_common.h"
#include "kernels.h"
#include "rules.h"

#define LDSP __attribute__((address_space(3)))

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));

constexpr int BM = 256, BN = 256, BK = 128;
constexpr int WAVES_M = 2, WAVES_N = 4, NWAVES = WAVES_M * WAVES_N;
constexpr int NTHREADS = 64 * NWAVES;
constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 32, TN = WN / 32;
constexpr int TILE = BM * BK;                      // bytes per operand per stage
constexpr int LD_PER_OP = TILE / 1024 / NWAVES;    // 1 KB direct loads per operand per wave per step

enum I8Mode { I8_UP = 0, I8_DOWN = 1 };

DEV int swz(int r, int c) { return c ^ ((r >> 1) & 7); }
DEV int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Raw buffer resource over [p, p + bytes) (gfx9 word 3: 32-bit data format).
DEV __amdgpu_buffer_rsrc_t make_rsrc(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, (int)bytes, 0x00020000);
}
DEV void barrier_no_fence() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
template <int N>
DEV void wait_vmcnt() {
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

// MFMA operand for rows [r0, r0 + 32) at k sub-step ks (32 wide) of a stage tile.
DEV i32x4_t frag(const uint8_t *t, int r0, int ks, int lane) {
    const int r = r0 + (lane & 31), h = lane >> 5;
    return __builtin_bit_cast(i32x4_t, ld_u32x4(t + r * BK + 16 * swz(r, 2 * ks + h)));
}

template <int MODE>
__global__ __launch_bounds__(NTHREADS, 1) void gemm_i8_kernel(I8GemmArgs args) {
    __shared__ __attribute__((aligned(16))) uint8_t lds_all[4 * TILE];
    __shared__ float sc_a[BM], sc_b[BN];     // scales of the tile's rows and columns
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = uniform(tid >> 6);
    const int wm = wave / WAVES_N, wn = wave % WAVES_N;

    // ---------------- tile: expert region and rows ----------------
    const bool sh = (int)blockIdx.x < args.shared_grid;   // the shared expert's tiles come first
    const I8Product &g = sh ? args.shared : args.routed;
    int e = 0, row0 = 0, row_end = 0, ntile = 0;
    const int ntn = (MODE == I8_UP) ? g.N / (BN / 2) : g.N / BN;
    if (sh) {
        int mt = 0;
        if (!map_tile(blockIdx.x, (g.rows + BM - 1) / BM, ntn, mt, ntile)) return;
        row0 = mt * BM;
        row_end = g.rows;
    } else {
        int within = 0;
        if (!place_tile<BM>(args.offsets, args.E, (int)blockIdx.x - args.shared_grid, ntn, lane, e, within, ntile))
            return;
        row0 = uniform(args.offsets[e]) + within * BM;
        row_end = uniform(args.offsets[e + 1]);
    }
    const int n0 = ntile * ((MODE == I8_UP) ? BN / 2 : BN);
    const bool gather = MODE == I8_UP && !sh;

    // physical A row of tile row r (rows past the region's end repeat its last
    // row; their results are never stored)
    auto a_phys = [&](int r) {
        const int p = min(row0 + r, row_end - 1);
        const int phys = gather ? args.rowidx[min(max(p, 0), args.routed.rows - 1)] : p;
        return min(max(phys, 0), g.a_nrows - 1);
    };
    // MODE I8_UP: tile columns 64 c + 0..31 are gate, 64 c + 32..63 the up columns of the same f
    auto b_col = [&](int c) { return (MODE == I8_UP) ? n0 + (c >> 6) * 32 + (c & 31) : n0 + c; };
    if (tid < BM) {
        sc_a[tid] = g.As[a_phys(tid)];
    } else {
        const int c = tid - BM;
        const float *s = (MODE == I8_UP) && (c & 32) ? g.Bs2 : g.Bs;
        sc_b[c] = s[(long)e * g.N + b_col(c)];
    }

    // ---------------- direct-load set-up ----------------
    // Tile load i of wave w is wave instruction q = LD_PER_OP w + i: 1 KB = 8
    // rows of 128 bytes; lane -> row 8 q + lane / 8, physical chunk
    // (lane & 7) ^ ((4 (q & 1) + lane / 16) & 7).
    const int l8 = lane >> 3;
    const uint32_t col_even = 16u * (uint32_t)((lane & 7) ^ ((l8 >> 1) & 7));
    const uint32_t col_odd = 16u * (uint32_t)((lane & 7) ^ ((4 + (l8 >> 1)) & 7));
    const uint32_t K = (uint32_t)g.K;
    const uint32_t b_lane_even = (uint32_t)l8 * K + col_even, b_lane_odd = (uint32_t)l8 * K + col_odd;
    uint32_t a_off[LD_PER_OP];
#pragma unroll
    for (int i = 0; i < LD_PER_OP; ++i) {
        const int q = LD_PER_OP * wave + i;
        a_off[i] = (uint32_t)a_phys(8 * q + l8) * K + ((q & 1) ? col_odd : col_even);
    }
    const int nk = g.K / BK;
    auto issue_a = [&](int kt, uint8_t *la) {
#pragma unroll
        for (int i = 0; i < LD_PER_OP; ++i) {
            const int q = LD_PER_OP * wave + i;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(g.A, g.a_bytes), (LDSP void *)(la + q * 1024),
                                                     16, a_off[i], (uint32_t)kt * BK, 0, 0);
        }
    };
    auto issue_b = [&](int kt, uint8_t *lb) {
#pragma unroll
        for (int i = 0; i < LD_PER_OP; ++i) {
            const int q = LD_PER_OP * wave + i;
            const bool up = (MODE == I8_UP) && ((q >> 2) & 1);
            const uint32_t brow = (uint32_t)(e * g.N + b_col(8 * q));
            __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(up ? g.B2 : g.B, g.b_bytes),
                                                     (LDSP void *)(lb + q * 1024), 16,
                                                     (q & 1) ? b_lane_odd : b_lane_even,
                                                     brow * K + (uint32_t)kt * BK, 0, 0);
        }
    };

    i32x16_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0;

    // Fragments one step ahead of their MFMAs.
    constexpr int KS = BK / 32;
    i32x4_t bfr[TN], a_cur;
    auto compute_ks = [&](const uint8_t *la, const uint8_t *lb, int ks) {
        if (ks == 0) {
#pragma unroll
            for (int j = 0; j < TN; ++j) bfr[j] = frag(lb, wn * WN + 32 * j, 0, lane);
            a_cur = frag(la, wm * WM, 0, lane);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            i32x4_t a_nxt = a_cur;
            if (i + 1 < TM) a_nxt = frag(la, wm * WM + 32 * (i + 1), ks, lane);
            else if (ks + 1 < KS) a_nxt = frag(la, wm * WM, ks + 1, lane);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a_cur, bfr[j], acc[i][j], 0, 0, 0);
                if (i == TM - 1 && ks + 1 < KS) bfr[j] = frag(lb, wn * WN + 32 * j, ks + 1, lane);
            }
            a_cur = a_nxt;
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    issue_a(0, lds_all);
    issue_b(0, lds_all + 2 * TILE);
    int cur = 0;
#pragma clang loop unroll(disable)
    for (int kt = 0; kt < nk; ++kt) {
        wait_vmcnt<0>();
        barrier_no_fence();
        const int nxt = uniform(cur ^ 1);
        const uint8_t *la = lds_all + cur * TILE, *lb = lds_all + (2 + cur) * TILE;
        if (kt + 1 < nk) issue_b(kt + 1, lds_all + (2 + nxt) * TILE);
        asm volatile("" ::: "memory");
        compute_ks(la, lb, 0);
        compute_ks(la, lb, 1);
        if (kt + 1 < nk) {
            asm volatile("" ::: "memory");
            issue_a(kt + 1, lds_all + nxt * TILE);
            asm volatile("" ::: "memory");
        }
        compute_ks(la, lb, 2);
        compute_ks(la, lb, 3);
        cur = nxt;
    }
    __syncthreads();

    // ---------------- epilogue ----------------
    // accumulator layout: lane l, register q -> row 8 (q / 4) + 4 (l / 32) + q % 4,
    // column l % 32; rows go through a per-wave LDS scratch (32 x WN fp32)
    const int lrow = lane & 31, lhalf = lane >> 5;
    constexpr int SP = WN + 4;
    static_assert(NWAVES * 32 * SP * 4 <= 4 * TILE, "epilogue scratch fits the stages");
    float *scr = reinterpret_cast<float *>(lds_all) + wave * 32 * SP;
    float sb[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] = sc_b[wn * WN + 32 * j + lrow];
    auto stage = [&](int i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const int row = 8 * (q >> 2) + 4 * lhalf + (q & 3);
                scr[row * SP + 32 * j + lrow] = (float)acc[i][j][q] * sb[j];
            }
    };
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        stage(i);
        if constexpr (MODE == I8_UP) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int row = (lane >> 2) + 16 * t, c = 8 * (lane & 3);
                const int rl = wm * WM + 32 * i + row, p = row0 + rl;
                const float sr = sc_a[rl];
                const f32x8 ga = ld_f32x8(scr + row * SP + c), ub = ld_f32x8(scr + row * SP + 32 + c);
                f32x8 h;
#pragma unroll
                for (int k = 0; k < 8; ++k) h[k] = silu_f(sr * ga[k]) * (sr * ub[k]);
                if (p < row_end) st_f32x8(g.H + (long)p * g.N + n0 + wn * 32 + c, h);
            }
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int row = (lane >> 3) + 8 * t, c = 8 * (lane & 7);
                const int rl = wm * WM + 32 * i + row, p = row0 + rl;
                const float sr = sc_a[rl];
                f32x8 v = ld_f32x8(scr + row * SP + c);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = sr * v[k];
                if (p < row_end)
                    __builtin_nontemporal_store(pack_bf8(v), reinterpret_cast<u32x4_t *>(
                                                                 g.C + (long)p * g.N + n0 + wn * WN + c));
            }
        }
    }
}

template <int MODE>
hipError_t launch_i8_mode(I8GemmArgs a, hipStream_t st) {
    const int cols = MODE == I8_UP ? BN / 2 : BN;
    const long sh = a.shared.rows > 0 && a.shared.N > 0
                        ? raster_grid((a.shared.rows + BM - 1) / BM, a.shared.N / cols) : 0;
    const long rt = a.routed.rows > 0 ? raster_grid(a.routed.rows / BM + a.E, a.routed.N / cols) : 0;
    if (sh + rt <= 0) return hipSuccess;
    a.shared_grid = (int)sh;
    gemm_i8_kernel<MODE><<<dim3((unsigned)(sh + rt)), dim3(NTHREADS), 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_i8_up(const I8GemmArgs &a, hipStream_t st) { return launch_i8_mode<I8_UP>(a, st); }
hipError_t launch_gemm_i8_down(const I8GemmArgs &a, hipStream_t st) { return launch_i8_mode<I8_DOWN>(a, st); }
