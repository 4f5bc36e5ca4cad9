// Grouped int8 products of the experts on v_mfma_i32_32x32x32_i8.  Per expert
// e and buffer positions p of e's region (the shared expert: the tokens as
// they are, in the same launch):
//
//   I8_UP    g = sx sg[n] (Xq[tok(p)] . Wg_q[e][n]), u likewise;
//            H = silu(g) u in fp32, for the row quantiser
//   I8_DOWN  Yexp = sd[n] (Hq[p] . Wd_q[e][n]) / u[e] -> fp16
//
// The route's weight in the sum over a token's experts holds the rest, the row's
// scale times u[e], a power of two that fits the expert's largest possible value to
// fp16: half a step is 2^-11 of a value, an eighth of bf16's, and for the smallest
// values at most 2^-8 of one unit of the integer sum in the expert's largest channel
// (K 768: 2^-15).  (bf16, as in moe_forward, was off by 1.4 times as much as one
// rounding of Y.)
//
// Every operand is a matrix of K-contiguous byte rows with one fp32 scale per
// row.  The dot products are exact in 32-bit integers (K <= 131072: 127^2 K
// stays below 2^31) and rounded once, to fp32, when the scales are applied.
//
// 256 x 256 block tile, K step 128 bytes, two LDS stages filled by direct
// global->LDS loads (128-byte rows, chunk XOR (row >> 1) & 7), 8 waves of 128 x 64
// (two per SIMD), tiles rastered XCD-aware.  The MFMA takes 16 consecutive
// bytes of row l % 32 from lane l, at k 16 (l / 32) of its 32.
//
// One workgroup per CU runs tile after tile.  A tile of K = 768 is six steps, and
// its first loads and its epilogue's stores together take as long: the next
// tile's first step is asked for before the epilogue, whose stores then drain
// behind the next tile's products.
//
// 16384 tokens to 8 of 32 experts of 1536, d 4096: up 1470 us, 2.24 POP/s, down 920,
// 1.79 (a tile of 12 steps has the epilogue of one of 32); a large library
// product reaches 2.12.  The matrix units are busy 58 and 46 % of the time, at 1.88
// GHz (2.1 to 2.3 in launches of 0.1 to 0.2 ms); waves wait half of theirs, next to
// none of it for LDS.
#include "common.h"
#include "i8_common.h"
#include "kernels.h"
#include "rules.h"

#define LDSP __attribute__((address_space(3)))

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x16_t __attribute__((ext_vector_type(16)));

constexpr int BM = 256, BN = 256, BK = 128;
constexpr int WAVES_M = 2, WAVES_N = 4, NWAVES = WAVES_M * WAVES_N;   // XW
constexpr int NTHREADS = 64 * NWAVES;
constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 32, TN = WN / 32;
constexpr int TILE = BM * BK;                      // bytes per operand per stage
constexpr int LD_PER_OP = TILE / 1024 / NWAVES;    // 1 KB direct loads per operand per wave per step

constexpr int SP = WN + 4;                         // pitch of an epilogue scratch row
// stores per lane and tile: up product one per value of H, down product 8 rows at a time
template <int MODE> constexpr int STORES = MODE == 0 ? 16 * TM : 4 * TM;
constexpr int NT = 2;                              // buffer stores past the L2 (non-temporal)
static_assert(TN == 2, "a gate and an up group of 32 columns per wave");

enum I8Mode { I8_UP = 0, I8_DOWN = 1 };

DEV int swz(int r, int c) { return c ^ ((r >> 1) & 7); }
DEV int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Raw buffer resource over [p, p + bytes) (gfx9 word 3: 32-bit data format).
DEV __amdgpu_buffer_rsrc_t make_rsrc(const void *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), (short)0, (int)bytes, 0x00020000);
}
// 16 bytes per lane from [p, p + bytes) at voff + soff (zeros past the end) to
// LDS, consecutive lanes to consecutive places from dst
DEV void load_lds16(const uint8_t *p, uint32_t bytes, uint8_t *dst, uint32_t voff, uint32_t soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(p, bytes), (LDSP void *)dst, 16, voff, soff, 0, 0);
}
// 16 or 4 bytes per lane to [p, p + bytes), dropped past the end; the first past
// the L2, which holds the operand panels
DEV void store_b128(u32x4_t v, void *p, uint32_t bytes, uint32_t off) {
    __builtin_amdgcn_raw_buffer_store_b128(v, make_rsrc(p, bytes), off, 0, NT);
}
DEV void store_b32(float v, void *p, uint32_t bytes, uint32_t voff, uint32_t soff) {
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), make_rsrc(p, bytes), voff, soff, 0);
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

// One tile: its expert's region and place in it.
struct I8Tile {
    int sh, e, row0, row_end, ntile;
};

template <int MODE>
__global__ __launch_bounds__(NTHREADS, 1) void gemm_i8_kernel(I8GemmArgs args) {
    // An array per stage and operand, named where it is used: the compiler lets
    // direct loads into one of them pass reads of another.  With one array for
    // all stages it waits for every load in flight before any read of it, so
    // the loads of step k + 1 had to arrive before step k began (16384 tokens,
    // 32 experts of 1536, d 4096: up 1770 us, down 1107, now 1470 and 920).
    __shared__ __attribute__((aligned(16))) uint8_t lds_a0[TILE], lds_b0[TILE], lds_a1[TILE], lds_b1[TILE];
    // scales of a tile's rows and columns, by parity of the tile, and the waves'
    // epilogue scratch
    __shared__ __attribute__((aligned(16))) float epi[2 * (BM + BN) + NWAVES * 8 * SP];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = uniform(tid >> 6);
    const int wm = wave / WAVES_N, wn = wave % WAVES_N;
    constexpr int COLS = (MODE == I8_UP) ? BN / 2 : BN;     // output columns per tile

    // ---------------- tiles of this workgroup ----------------
    // slots blockIdx, blockIdx + 256, ... of the raster (the shared expert's
    // come first), some of them empty; the experts' tile counts stay in registers
    ExpertTiles<BM> ex;
    ex.scan(args.offsets, args.E, lane);
    const int slots = args.shared_grid + args.routed_grid;
    int slot = (int)blockIdx.x - (int)gridDim.x;
    auto next_tile = [&](I8Tile &t) {        // leaves t alone where there is none
        for (slot += (int)gridDim.x; slot < slots; slot += (int)gridDim.x) {
            const int sh = slot < args.shared_grid;
            const I8Product &g = sh ? args.shared : args.routed;
            const int mtiles = sh ? (g.rows + BM - 1) / BM : ex.total;
            int mt = 0, n = 0;
            if (!map_tile(sh ? slot : slot - args.shared_grid, mtiles, g.N / COLS, mt, n)) continue;
            int e = 0, within = mt;
            if (!sh) e = ex.find(mt, within);
            const int first = sh ? 0 : uniform(args.offsets[e]);
            t = I8Tile{sh, e, first + within * BM, sh ? g.rows : uniform(args.offsets[e + 1]), n};
            return true;
        }
        return false;
    };
    // physical A row of a tile's row r (rows past the region's end repeat its
    // last row; their results are never stored), in two parts: the plan's
    // entry, then the row's number
    auto a_entry = [&](const I8Tile &t, int r) {
        const int p = min(t.row0 + r, t.row_end - 1);
        return MODE == I8_UP && !t.sh ? args.rowidx[min(max(p, 0), args.routed.rows - 1)] : p;
    };
    auto a_row = [&](const I8Tile &t, int entry) {
        return min(max(entry, 0), (t.sh ? args.shared.a_nrows : args.routed.a_nrows) - 1);
    };
    // MODE I8_UP: tile columns 64 c + 0..31 are gate, 64 c + 32..63 the up columns of the same f
    auto b_col = [&](const I8Tile &t, int c) {
        return t.ntile * COLS + ((MODE == I8_UP) ? (c >> 6) * 32 + (c & 31) : c);
    };

    // ---------------- loads ----------------
    // Tile load i of wave w is wave instruction q = LD_PER_OP w + i: 1 KB = 8
    // rows of 128 bytes; lane -> row 8 q + lane / 8, physical chunk
    // (lane & 7) ^ ((4 (q & 1) + lane / 16) & 7).
    const int l8 = lane >> 3;
    const uint32_t col_even = 16u * (uint32_t)((lane & 7) ^ ((l8 >> 1) & 7));
    const uint32_t col_odd = 16u * (uint32_t)((lane & 7) ^ ((4 + (l8 >> 1)) & 7));
    struct Loads {
        uint32_t a[LD_PER_OP];               // lane offsets of A's loads
        uint32_t scale;                      // row of this thread's scale
    };
    auto ask_loads = [&](const I8Tile &t, Loads &l) {
#pragma unroll
        for (int i = 0; i < LD_PER_OP; ++i) l.a[i] = (uint32_t)a_entry(t, 8 * (LD_PER_OP * wave + i) + l8);
        l.scale = (uint32_t)a_entry(t, tid & (BM - 1));
    };
    auto set_loads = [&](const I8Tile &t, Loads &l) {
        const uint32_t K = (uint32_t)(t.sh ? args.shared.K : args.routed.K);
#pragma unroll
        for (int i = 0; i < LD_PER_OP; ++i)
            l.a[i] = (uint32_t)a_row(t, (int)l.a[i]) * K + (((LD_PER_OP * wave + i) & 1) ? col_odd : col_even);
        l.scale = (uint32_t)a_row(t, (int)l.scale);
    };
    auto issue_a = [&](const I8Tile &t, const Loads &l, int kt, uint8_t *la) {
        const I8Product &g = t.sh ? args.shared : args.routed;
#pragma unroll
        for (int i = 0; i < LD_PER_OP; ++i)
            load_lds16(g.A, g.a_bytes, la + (LD_PER_OP * wave + i) * 1024, l.a[i], (uint32_t)kt * BK);
    };
    auto issue_b = [&](const I8Tile &t, int kt, uint8_t *lb) {
        const I8Product &g = t.sh ? args.shared : args.routed;
        const uint32_t K = (uint32_t)g.K;
#pragma unroll
        for (int i = 0; i < LD_PER_OP; ++i) {
            const int q = LD_PER_OP * wave + i;
            const bool up = (MODE == I8_UP) && ((q >> 2) & 1);
            const uint32_t brow = (uint32_t)(t.e * g.N + b_col(t, 8 * q));
            load_lds16(up ? g.B2 : g.B, g.b_bytes, lb + q * 1024, (uint32_t)l8 * K + ((q & 1) ? col_odd : col_even),
                       brow * K + (uint32_t)kt * BK);
        }
    };
    // thread tid's scale of a tile: row tid, or column tid - BM
    static_assert(NTHREADS == BM + BN && BM % 64 == 0, "a scale per thread, rows and columns in waves of their own");
    // (gate and up channels alternate by 32 lanes: a wave of columns reads both arrays)
    // (down product: its columns' alone, with the expert's unit)
    struct Scale {
        float s, unit;
    };
    auto scale_of = [&](const I8Tile &t, const Loads &l) {
        const I8Product &g = t.sh ? args.shared : args.routed;
        const int c = (tid - BM) & (BN - 1);
        const float *at = MODE == I8_UP && tid < BM ? g.As + l.scale
                        : ((MODE == I8_UP) && (c & 32) ? g.Bs2 : g.Bs) + ((long)t.e * g.N + b_col(t, c));
        return Scale{*at, MODE == I8_UP ? 1.f : args.unit[2 * (t.sh ? args.E : t.e)]};
    };

    I8Tile t, nt;
    Loads ld, nld;
    if (!next_tile(t)) return;
    nt = t;
    ask_loads(t, ld);
    set_loads(t, ld);
    nld = ld;
    Scale scale = scale_of(t, ld);
    issue_b(t, 0, lds_b0);
    issue_a(t, ld, 0, lds_a0);
    issue_a(t, ld, 1, lds_a1);               // K is a multiple of 256: steps come in pairs
    issue_b(t, 1, lds_b1);
    constexpr int KS = BK / 32, LPS = 2 * LD_PER_OP;
    wait_vmcnt<LPS>();
    const int lrow = lane & 31, lhalf = lane >> 5;
    float *const scr = epi + 2 * (BM + BN) + wave * 8 * SP;
    for (int parity = 0;; parity ^= 1) {
        epi[parity * (BM + BN) + tid] = scale.s * scale.unit;
        i32x16_t acc[TM][TN];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) acc[i][j][q] = 0;
        // Fragments one step ahead of their MFMAs.  Waves whose rows are all past the
        // region's end leave the products out, but not the stores, whose number the
        // waits count on (8192 tokens to 128 experts of 768, d 2048: 557 -> 541 us; 3000
        // to 64 of 1024: 207 -> 196).
        const bool busy = t.row0 + wm * WM < t.row_end;
        i32x4_t bfr[TN], a_cur;
        auto compute_ks = [&](const uint8_t *la, const uint8_t *lb, int ks) {
            if (!busy) return;
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

        // Step 0 of a tile is asked for at the last step of the tile before (the
        // last tile's own again where there is none after it: one sequence of loads
        // and stores, whose waits are known counts), ahead of that tile's stores,
        // step 1 behind them, step kt + 1 at step kt from then on.  What the next
        // tile is, is asked three steps before the end; its rows' numbers are there
        // a step later.
        const int nk = (t.sh ? args.shared.K : args.routed.K) / BK;
        bool more = false;
        auto ask_next = [&] {
            more = next_tile(nt);
            if (more) ask_loads(nt, nld);
        };
        auto set_next = [&] {
            if (more) {
                set_loads(nt, nld);
                scale = scale_of(nt, nld);
            }
        };
        // the second step of a pair, and the loads of the step after it
        auto odd_step = [&](int kt) {
            const bool last = kt + 1 == nk;
            const I8Tile &lt = last ? nt : t;
            const Loads &ll = last ? nld : ld;
            const int lk = last ? 0 : kt + 1;
            issue_b(lt, lk, lds_b0);
            asm volatile("" ::: "memory");
            compute_ks(lds_a1, lds_b1, 0);
            compute_ks(lds_a1, lds_b1, 1);
            asm volatile("" ::: "memory");
            issue_a(lt, ll, lk, lds_a0);
            asm volatile("" ::: "memory");
            compute_ks(lds_a1, lds_b1, 2);
            compute_ks(lds_a1, lds_b1, 3);
        };
        // (the counter ends at 63: with more behind them, the first stores too)
        wait_vmcnt<LPS + STORES<MODE> < 63 ? LPS + STORES<MODE> : 63>();
        // the scale, which other waves read: one that is not busy waits for no LDS
        // access of its own before then
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        barrier_no_fence();
        if (nk == 2) {
            ask_next();
            set_next();
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) compute_ks(lds_a0, lds_b0, ks);
        wait_vmcnt<0>();
        barrier_no_fence();
        if (nk == 4) ask_next();
        odd_step(1);
#pragma clang loop unroll(disable)
        for (int kt = 2; kt < nk; kt += 2) {
            wait_vmcnt<0>();
            barrier_no_fence();
            if (kt + 2 == nk) set_next();
            issue_b(t, kt + 1, lds_b1);
            asm volatile("" ::: "memory");
            compute_ks(lds_a0, lds_b0, 0);
            compute_ks(lds_a0, lds_b0, 1);
            asm volatile("" ::: "memory");
            issue_a(t, ld, kt + 1, lds_a1);
            asm volatile("" ::: "memory");
            compute_ks(lds_a0, lds_b0, 2);
            compute_ks(lds_a0, lds_b0, 3);
            wait_vmcnt<0>();
            barrier_no_fence();
            if (kt + 4 == nk) ask_next();
            odd_step(kt + 1);
        }
        // ---------------- epilogue ----------------
        // accumulator layout: lane l, register q -> row 8 (q / 4) + 4 (l / 32) + q % 4,
        // column l % 32.  Rows past the region lie past the end of the stores'
        // resource and are dropped there, so that every tile has the same number
        // of stores.
        const I8Product &g = t.sh ? args.shared : args.routed;
        const float *sc = epi + parity * (BM + BN);
        float sb[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) sb[j] = sc[BM + wn * WN + 32 * j + lrow];
        const int rows = min(t.row_end - t.row0, BM), n0 = t.ntile * COLS;
        if constexpr (MODE == I8_UP) {
            // a lane has gate and up of the same column: H needs no exchange, and
            // the 32 lanes of a row store a whole line
            float *const out = g.H + (long)t.row0 * g.N;
            const uint32_t bytes = (uint32_t)rows * (uint32_t)g.N * 4u, pitch = (uint32_t)g.N * 4u;
            const uint32_t lane_off = (uint32_t)(4 * lhalf) * pitch + (uint32_t)(n0 + wn * 32 + lrow) * 4u;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int qg = 0; qg < 4; ++qg) {
                    const int rl = wm * WM + 32 * i + 8 * qg;
                    const f32x4_t sr = *reinterpret_cast<const f32x4_t *>(sc + rl + 4 * lhalf);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float ga = sr[q] * ((float)acc[i][0][4 * qg + q] * sb[0]);
                        const float ub = sr[q] * ((float)acc[i][1][4 * qg + q] * sb[1]);
                        store_b32(silu_f(ga) * ub, out, bytes, lane_off, (uint32_t)(rl + q) * pitch);
                    }
                }
        } else {
            // 16 bits: these outputs are the largest arrays of a large batch, and fp32
            // for them took 1000 tokens to 32 experts from 246 to 262 us, 8192 to 128 535 ->
            // 652, 4099 dense 1703 -> 1895, 16384 2808 -> 3247.  (Small batches hold fp32:
            // skinny_i8.hip.)
            // 8 rows at a time through a scratch of the wave's own (8 x WN fp32),
            // one 16-byte store per lane, whole lines.  (Weights as the MFMA's row
            // operand give a lane 8 channels without the scratch, but stores of 32
            // bytes per row: 8192 tokens to 128 experts of 768 163 -> 179 us, past the
            // L2 299.)
            const int er = lane >> 3, ec = lane & 7;
            uint16_t *const out = g.C + (long)t.row0 * g.N;
            const uint32_t bytes = (uint32_t)rows * (uint32_t)g.N * 2u;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int qg = 0; qg < 4; ++qg) {
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            scr[(4 * lhalf + q) * SP + 32 * j + lrow] = (float)acc[i][j][4 * qg + q] * sb[j];
                    const int rl = wm * WM + 32 * i + 8 * qg + er;
                    const f16x8_t v = __builtin_convertvector(ld_f32x8(scr + er * SP + 8 * ec), f16x8_t);
                    store_b128(__builtin_bit_cast(u32x4_t, v), out, bytes, (uint32_t)(rl * g.N + n0 + wn * WN + 8 * ec) * 2u);
                }
        }
        // every wave is done with the last step's stage by now
        barrier_no_fence();
        if (!more) break;
        t = nt;
        ld = nld;
        issue_a(t, ld, 1, lds_a1);
        issue_b(t, 1, lds_b1);
    }
    wait_vmcnt<0>();                         // no load into LDS outlives the workgroup
}

template <int MODE>
hipError_t launch_i8_mode(I8GemmArgs a, hipStream_t st) {
    const int cols = MODE == I8_UP ? BN / 2 : BN;
    const long sh = a.shared.rows > 0 && a.shared.N > 0
                        ? raster_grid((a.shared.rows + BM - 1) / BM, a.shared.N / cols) : 0;
    const long rt = a.routed.rows > 0 ? raster_grid(a.routed.rows / BM + a.E, a.routed.N / cols) : 0;
    if (sh + rt <= 0) return hipSuccess;
    a.shared_grid = (int)sh;
    a.routed_grid = (int)rt;
    // one workgroup per CU (the rasters' grids are multiples of 256)
    gemm_i8_kernel<MODE><<<dim3(256), dim3(NTHREADS), 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_gemm_i8_up(const I8GemmArgs &a, hipStream_t st) { return launch_i8_mode<I8_UP>(a, st); }
hipError_t launch_gemm_i8_down(const I8GemmArgs &a, hipStream_t st) { return launch_i8_mode<I8_DOWN>(a, st); }
