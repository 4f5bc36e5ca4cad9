// The whole layer for up to 16 tokens (decoding) in two launches: the router's
// partial logits, and everything else -- selection by scores, both products of
// the experts and the sum.
//
// The work is a stream of the weights of the reached experts.  Workgroups take
// items from one queue: tiles of the up product (64 gate and 64 up columns, the
// shared expert's first), then tiles of the down product (128 columns, over the
// rows of all reached experts one after the other), each cut along K so that there
// are enough of them.  A tile of the down product waits for the H of its rows.  No
// wait needs a workgroup that has not started, or one that waits itself: first items
// come from counters of their own, out of the queue's order, so before its first wait
// a workgroup sees every first item of the up product taken, and does those that are
// not; the others are taken in order; and a workgroup that waits holds no item but the
// one it waits for, since it asks for the next one afterwards.
//
// A tile's arithmetic: 4 waves take every fourth 32-row slice of K; a wave's step
// is 32 rows x 128 columns, 8 loads of 16 bytes per lane straight into registers, 8
// columns of 8 rows, which are transposed there (v_perm_b32) into the row operands
// of 8 v_mfma_f32_16x16x32_bf16; the 16 tokens are the column operand.  The next
// step's loads, and the next item's first, are under way meanwhile.
//
// H is held as two bf16 parts, high and low (16 significant bits), and an expert's
// part of the down product is scaled by the token's weight, or left out, in fp32:
// an expert's infinities reach the tokens that chose it and no others, and Y is
// rounded once.  Both parts cost a second product per operand; the matrix units are
// under 10 % busy.
//
// Measured: 16 tokens to 32 experts of 1536, d 4096 (1.2 GB) 227 us, 5.3 TB/s, where a copy
// of 2 GiB has 4.9; 7 tokens, 8 experts of 2048 and a shared one, d 7168 (0.8 GB) 154; one
// token to 128 experts of 768, d 2048 (76 MB) 34 (moe_route_scored, moe_plan and
// moe_forward 47): router 4.7, selection 6, up product 12, the wait for its sums 1, down
// product 4, the last sums 2, and the launches.  What it took, us for those three: waits by
// whole-cache write-backs and invalidations 494 / 375 / 131, stores through the L2 331 / 261 / 64, selection by
// compares of a whole workgroup 300 / 197 / 39, by candidates 289 / 188 / 37, first items from 8
// counters and slices by size 266 / 177 / 34, past the caches 246 / 168 / 34.  Tried and slower: three
// workgroups to a CU (168 registers; 328 / 221 / 47), all items from 8 queues (313 / 195 / 46: the
// search for the next queue delays a tile's sums).
#include <cfloat>

#include "common.h"
#include "few.h"
#include "kernels.h"
#include "rules.h"

namespace {

constexpr float MASKED = -1e38f;

// ---------------------------------------------------------------- router
// Partial logits of a slice of the d axis and 16 V experts: part [S][T][E] (slices at a
// pitch of g.pitch).  As the layer's tiles below: a wave's step is 32 rows, a lane
// loads V experts of 8 rows as they lie, the tokens are the column operand; the
// 8 waves' sums meet in LDS in order.  Clears the counters, too.
constexpr int RW = 8;
template <int V>
__global__ __launch_bounds__(64 * RW) void few_router_kernel(FewArgs g) {
    constexpr int NB = 4, COLS = 16 * V;     // steps under way, experts
    __shared__ float red[RW][FEW_MAX_T][COLS + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g4 = lane >> 4;
    const int steps = g.d / 32, S = gridDim.x, eb = COLS * blockIdx.y;
    const int s0 = (int)((long)steps * blockIdx.x / S), s1 = (int)((long)steps * (blockIdx.x + 1) / S);
    const uint16_t *Wr = g.W_r + (eb + V * r < g.E ? eb + V * r : 0);
    const uint16_t *X = g.X + (long)(r < g.T ? r : g.T - 1) * g.d + 8 * g4;
    f32x4_t acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int b = s0 + wave; b < s1; b += NB * RW) {
        u32x4_t x[NB];
        uint32_t w[NB][8][(V + 1) / 2];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const int st = min(b + n * RW, s1 - 1);
            x[n] = ld_u32x4(X + 32l * st);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint16_t *p = Wr + (32l * st + 8 * g4 + j) * g.E;
                if constexpr (V == 4) {
                    const u32x2_t q = ld_u32x2(p);
                    w[n][j][0] = q[0];
                    w[n][j][1] = q[1];
                } else {
                    w[n][j][0] = *p;
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            if (b + n * RW >= s1) break;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                u32x4_t a;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    a[q] = __builtin_amdgcn_perm(w[n][2 * q + 1][i >> 1], w[n][2 * q][i >> 1],
                                                 (i & 1) ? 0x07060302u : 0x05040100u);
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                                 __builtin_bit_cast(bf16x8_t, x[n]), acc[i], 0, 0, 0);
            }
        }
    }
    if (blockIdx.x == 0 && blockIdx.y == 0) {
        if (tid == 0) *g.err = 0;
        for (int i = tid; i < g.ncounters; i += 64 * RW) g.counters[i] = 0;
    }
    // accumulators: lane (g4, r), register p of product i: expert V (4 g4 + p) + i, token r
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int p = 0; p < 4; ++p) red[wave][r][V * (4 * g4 + p) + i] = acc[i][p];
    __syncthreads();
    for (int i = tid; i < g.T * COLS; i += 64 * RW) {
        const int t = i / COLS, c = i % COLS;
        if (eb + c >= g.E) continue;
        float s = red[0][t][c];
#pragma unroll
        for (int w = 1; w < RW; ++w) s = s + red[w][t][c];
        g.part[(long)blockIdx.x * g.pitch + t * g.E + eb + c] = s;
    }
}

// ---------------------------------------------------------------- selection
// Within rows of 16 lanes, the same for each of them: DPP moves within quads, then
// mirrored half rows and rows.
template <typename F>
DEV float row16(float v, F f) {
#define STEP(CTRL)                                                                              \
    v = f(v, __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xF, 0xF, true)))
    STEP(0xB1);
    STEP(0x4E);
    STEP(0x141);
    STEP(0x140);
#undef STEP
    return v;
}
DEV double shfl_xor_d(double v, int m) {
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)b, m, 64);
    const uint32_t hi = (uint32_t)__shfl_xor((int)(uint32_t)(b >> 32), m, 64);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
// Unsigned key with the order of the double, above 1, and back.
DEV uint64_t rank_key(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);   // -0 and 0 are one
    return (b >> 63) ? ~b : (b | (1ull << 63));
}
DEV double key_value(uint64_t k) {
    return k <= 1 ? -INFINITY : __longlong_as_double((long long)((k >> 63) ? k & ~(1ull << 63) : ~k));
}
// a / b for 0 <= a < 2^24, rb = 1 / b rounded
DEV int div24(int a, int b, float rb) {
    int q = (int)((float)a * rb);
    const int r = a - q * b;
    q += r >= b ? 1 : 0;
    q -= r < 0 ? 1 : 0;
    return q;
}

constexpr int NW = 4, NT = 64 * NW, PITCH = 128 + 4;

// The largest of the wave's values, the same for every lane: DPP moves within rows and to
// the next rows, then the last lane's.
DEV uint32_t wave_max(uint32_t v) {
    auto step = [&](int o) { v = (uint32_t)o > v ? (uint32_t)o : v; };
    step(__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));
    step(__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));
    step(__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));
    step(__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true));
    step(__builtin_amdgcn_update_dpp((int)v, (int)v, 0x142, 0xA, 0xF, false));   // lane 15 to the next row
    step(__builtin_amdgcn_update_dpp((int)v, (int)v, 0x143, 0xC, 0xF, false));   // lane 31 to the upper half
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
// LDS written by a wave and read by its other lanes
DEV void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

struct Select {                      // scratch of the start
    __attribute__((aligned(16))) float z[FEW_MAX_T * 256];         // [T][E]
    float bal[256], w[FEW_MAX_T][16], zmax[FEW_MAX_T], sum[FEW_MAX_T];
    uint32_t mask[256];
    int ids[FEW_MAX_T][16], slot_of[256], cnt[NW];
    __attribute__((aligned(16))) struct {
        uint64_t key[256];           // then the candidates
        uint32_t top[64];
        double gs[64];
    } wave[NW];
};

// One token's experts, as moe_route_scored defines them, by one wave: from its logits z
// to k ascending ids, each also in s.mask.  Lane l holds experts l, 64 + l, ...  Experts
// are ranked by 64-bit keys; only those can be chosen whose key's upper half is not
// below the k-th largest of the lanes' best ones, mostly few more than k, and where
// these are more than k they are ranked by whole keys and ids.  Loops stay compact:
// every call fetches this code from memory.
DEV void select_experts(const FewArgs &g, Select &s, int t, int wave, int lane) {
    const ScoreArgs &a = g.score;
    const int E = g.E, k = g.k, G = a.groups, n = E / G;
    const float *z = s.z + t * E;
    auto &m = s.wave[wave];
    const bool by_score = g.balance || (G > 1 && a.pair);
    auto live = [&](int e) { return z[e] >= MASKED && s.bal[e] >= MASKED; };
    float zmax = -INFINITY;
    double sum = 0.0;
    if (!a.sigmoid && (by_score || !a.renorm)) {     // the softmax's sum
        for (int e = lane; e < E; e += 64) zmax = fmaxf(zmax, live(e) ? fminf(z[e], FLT_MAX) : -INFINITY);
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) zmax = fmaxf(zmax, shfl_xor_f(zmax, x));
#pragma unroll 1
        for (int e = lane; e < E; e += 64)
            if (live(e)) sum += exp((double)fminf(z[e], FLT_MAX) - (double)zmax);
#pragma unroll 1
        for (int x = 1; x < 64; x <<= 1) sum += shfl_xor_d(sum, x);
        if (lane == 0) {
            s.zmax[t] = zmax;
            s.sum[t] = (float)sum;
        }
    }
#pragma unroll 1
    for (int e = lane; e < E; e += 64) {
        double v = (double)fminf(z[e], FLT_MAX);
        if (by_score) {
            const double x = exp(a.sigmoid ? -v : v - (double)zmax);
            v = (a.sigmoid ? 1.0 / (1.0 + x) : x / sum) + (double)s.bal[e];
        }
        m.key[e] = live(e) ? rank_key(v) : 1;        // a key of 0 is no expert
    }
    wave_sync();
    uint64_t kept = ~0ull;                           // by group
    if (G > 1) {
        int lpg = 32;                                // lanes to a group
        while (lpg * G > 64) lpg >>= 1;
        const int o = lane / lpg;
        double b1 = -INFINITY, b2 = -INFINITY;
        if (o < G)
#pragma unroll 1
            for (int e = lane % lpg; e < n; e += lpg) {
                const double v = key_value(m.key[o * n + e]);
                b2 = fmax(b2, fmin(b1, v));
                b1 = fmax(b1, v);
            }
#pragma unroll 1
        for (int x = 1; x < lpg; x <<= 1) {
            const double o1 = shfl_xor_d(b1, x), o2 = shfl_xor_d(b2, x);
            b2 = fmax(fmin(b1, o1), fmax(b2, o2));
            b1 = fmax(b1, o1);
        }
        if (o < G && lane % lpg == 0) m.gs[o] = a.pair && b2 > -INFINITY ? b1 + b2 : b1;
        wave_sync();
        const double mine = m.gs[lane < G ? lane : 0];
        int better = 0;
#pragma unroll 4
        for (int q = 0; q < G; ++q) {
            const double v = m.gs[q];
            better += v > mine || (v == mine && q < lane) ? 1 : 0;
        }
        kept = __ballot(lane < G && better < a.top_groups);
    }
    const float rn = 1.0f / (float)n;
    uint64_t key[4];
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int e = lane + 64 * q;
        key[q] = 0;
        if (e < E && ((kept >> (G > 1 ? div24(e, n, rn) : 0)) & 1)) key[q] = m.key[e];
        top = max(top, (uint32_t)(key[q] >> 32));
    }
    m.top[lane] = top;
    wave_sync();
    int above = 0;
    {
        u32x4_t v[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) v[q] = *reinterpret_cast<const u32x4_t *>(&m.top[4 * q]);
#pragma unroll
        for (int q = 0; q < 16; ++q)
#pragma unroll
            for (int p = 0; p < 4; ++p) above += v[q][p] > top ? 1 : 0;
    }
    const uint32_t least = ~wave_max(above < k ? ~top : 0u);
    unsigned long long cand[4];
    int count = 0;
    const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        cand[q] = __ballot(key[q] != 0 && (uint32_t)(key[q] >> 32) >= least);
        count += __popcll(cand[q]);
    }
    if (count > k) {
        // the candidates in ascending id: of equal keys, the one before is better
        int at[4], first = 0;
        wave_sync();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            at[q] = first + __popcll(cand[q] & below);
            if ((cand[q] >> lane) & 1) m.key[at[q]] = key[q];
            first += __popcll(cand[q]);
        }
        wave_sync();
        int better[4] = {0, 0, 0, 0};
#pragma unroll 4
        for (int o = 0; o < count; ++o) {
            const uint64_t v = m.key[o];
#pragma unroll
            for (int q = 0; q < 4; ++q) better[q] += v > key[q] || (v == key[q] && o < at[q]) ? 1 : 0;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) cand[q] &= __ballot(better[q] < k);
    }
    int first = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if ((cand[q] >> lane) & 1) {
            s.ids[t][first + __popcll(cand[q] & below)] = lane + 64 * q;
            atomicOr(&s.mask[lane + 64 * q], 1u << t);
        }
        first += __popcll(cand[q]);
    }
    wave_sync();                                     // m is free again
}

// The weights of the tokens' experts, 16 lanes to a token: renormalised ones are ratios
// of scores, taken to the largest of them, so that scores that underflow together
// keep theirs.
DEV void weigh_experts(const FewArgs &g, Select &s, int tid) {
    const ScoreArgs &a = g.score;
    const int t = tid / 16, j = tid % 16;
    const bool route = t < g.T && j < g.k;
    const int id = route ? s.ids[t][j] : 0;
    const float z = route ? s.z[t * g.E + id] : 0.f;
    const bool on = route && z >= MASKED && s.bal[id] >= MASKED;
    const float zc = on ? fminf(z, FLT_MAX) : 0.f;
    float u = 0.f, total = 1.f;
    if (a.renorm) {
        const float c = a.sigmoid ? fminf(zc, 0.f) : zc;
        const float m = row16(on ? c : -INFINITY, [](float x, float y) { return fmaxf(x, y); });
        const float x = expf(c - m);
        if (on) u = a.sigmoid ? x / (1.0f + expf(-fabsf(zc))) : x;
        total = row16(u, [](float x, float y) { return x + y; });
    } else if (on) {
        const float x = expf(a.sigmoid ? -zc : zc - s.zmax[t]);
        u = a.sigmoid ? 1.0f / (1.0f + x) : x / s.sum[t];
    }
    if (route) s.w[t][j] = u > 0.f ? a.scale * (u / total) : 0.f;
}

// ---------------------------------------------------------------- the layer
// Waits between workgroups.  What one workgroup writes for others goes through
// its XCD's L2 to memory (agent-scope stores); its waves wait for that, meet at a
// barrier, and one thread adds to a counter.  A consumer's thread polls the counter
// and its workgroup passes a barrier; what it then loads, whole lines, was never read
// before in this launch, so no cache holds an older copy.  A release and an acquire
// instead write back and invalidate whole caches: 2 to 5 us for each tile.  Waits
// end after 2 s in any case (wall clock of 100 MHz), with the error word set.
constexpr unsigned long long WAIT_TICKS = 200000000ull;
DEV void poll(const int *ctr, int need, int *err) {
    const unsigned long long t0 = wall_clock64();
    while (__hip_atomic_load(ctr, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < need) {
        if (wall_clock64() - t0 > WAIT_TICKS) {
            __hip_atomic_store(err, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            return;
        }
        __builtin_amdgcn_s_sleep(4);
    }
}
DEV void st_agent(void *p, f32x4_t v) {
    const u32x4_t u = __builtin_bit_cast(u32x4_t, v);
    uint64_t *q = reinterpret_cast<uint64_t *>(p);
    __hip_atomic_store(q, (uint64_t)u[1] << 32 | u[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(q + 1, (uint64_t)u[3] << 32 | u[2], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
DEV void st_agent(void *p, uint32_t lo, uint32_t hi) {
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), (uint64_t)hi << 32 | lo, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}
// This wave's stores have arrived, but for the LATER loads that followed them.
template <int LATER>
DEV void stores_done() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LATER) : "memory");
}
DEV int add(int *ctr) { return __hip_atomic_fetch_add(ctr, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// PAST: weights are loaded past the caches (few_past_caches).
template <bool PAST>
__global__ __launch_bounds__(NT, 2) void few_kernel(FewArgs g) {
    __shared__ __attribute__((aligned(16))) union {
        float red[NW][16][PITCH];
        Select sel;
    } sh;
    __shared__ float s_w[256][FEW_MAX_T];     // weight of a slot's expert for a token
    __shared__ int s_list[256], s_mask[256];  // expert of a slot, tokens that chose it
    __shared__ int s_next, s_last;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g4 = lane >> 4;
    const int T = g.T, d = g.d, f = g.f, fs = g.fs;
    int *err = g.err, *queue = g.counters, *h_done = queue + (1 + FEW_QUEUES) * FEW_LINE;
    int *up_done = h_done + 257 * FEW_LINE, *down_done = up_done + g.up_counters;

    // A workgroup's first item comes from one of FEW_QUEUES counters (item FEW_QUEUES i +
    // q for the i-th that asks counter q: adds to one counter take 12 ns each, 6 us for
    // all workgroups), the others in order from `queue`.
    int *firsts = queue + FEW_LINE;
    int next = 0;
    // ---------------- routing: every workgroup for itself ----------------
    {
        Select &s = sh.sel;
        const float my_bias = g.bias && tid < g.E ? g.bias[tid] : 0.f;
        const float my_bal = g.balance && tid < g.E ? g.balance[tid] : 0.f;
        // slices added in order, all of them under way at once
        for (int i = 4 * tid; i < T * g.E; i += 4 * NT) {
            f32x4_t v = f32x4_t{0.f, 0.f, 0.f, 0.f}, u[FEW_ROUTER_SLICES];
#pragma unroll
            for (int q = 0; q < FEW_ROUTER_SLICES; ++q)
                u[q] = *reinterpret_cast<const f32x4_t *>(g.part + (long)(q < g.S ? q : 0) * g.pitch + i);
#pragma unroll
            for (int q = 0; q < FEW_ROUTER_SLICES; ++q)
                if (q < g.S)
#pragma unroll
                    for (int p = 0; p < 4; ++p) v[p] = v[p] + u[q][p];
            *reinterpret_cast<f32x4_t *>(s.z + i) = v;
        }
        if (tid == 0) next = add(firsts + blockIdx.x % FEW_QUEUES * FEW_LINE);   // after the loads: they return in order
        s.bal[tid] = my_bal;
        s.mask[tid] = 0;
        __syncthreads();
        if (g.bias) {
            if (tid < g.E)
                for (int t = 0; t < T; ++t) s.z[t * g.E + tid] = s.z[t * g.E + tid] + my_bias;
            __syncthreads();
        }
#pragma unroll 1
        for (int t = wave; t < T; t += NW) select_experts(g, s, t, wave, lane);
        __syncthreads();
        weigh_experts(g, s, tid);
        // slots: the experts that some token chose
        const uint32_t m = s.mask[tid];
        const unsigned long long b = __ballot(m != 0);
        if (lane == 0) s.cnt[wave] = __popcll(b);
        __syncthreads();
        int at = __popcll(b & ((1ull << lane) - 1));
        for (int w = 0; w < wave; ++w) at += s.cnt[w];
        if (m) {
            s_list[at] = tid;
            s_mask[at] = (int)m;
            s.slot_of[tid] = at;
        }
        if (tid == 0) {
            s_last = s.cnt[0] + s.cnt[1] + s.cnt[2] + s.cnt[3];
            s_next = FEW_QUEUES * next + blockIdx.x % FEW_QUEUES;
            // others have done this workgroup's first item: it goes on where they are
            if (s_next >= (int)gridDim.x) s_next = add(queue) + gridDim.x;
        }
        __syncthreads();
        const int t = tid / 16, j = tid % 16;
        if (t < T && j < g.k) {
            s_w[s.slot_of[s.ids[t][j]]][t] = s.w[t][j];
            if (blockIdx.x == 0) {
                g.topk_idx[t * g.k + j] = s.ids[t][j];
                g.topk_w[t * g.k + j] = s.w[t][j];
            }
        }
        if (blockIdx.x == 0)
            for (int i = tid; i < T * g.E; i += NT) g.logits[i] = s.z[i];
        __syncthreads();
    }
    const int slots = __builtin_amdgcn_readfirstlane(s_last);
    const int fu = f / FEW_UNIT, su = fs / FEW_UNIT, units = su + slots * fu;
    const int up_sh = fs / FEW_UP_COLS, up_e = f / FEW_UP_COLS, up_tiles = up_sh + slots * up_e;
    const int ks = few_slices(up_tiles, d / FEW_UNIT, FEW_UP_ITEMS, 2);
    const int cols = d / FEW_DOWN_COLS, ds = few_slices(cols, units, FEW_DOWN_ITEMS, 3);
    const int up_items = up_tiles * ks, items = up_items + cols * ds;
    // units of a slice; the first ones have one more
    const int up_q = d / FEW_UNIT / ks, up_r = d / FEW_UNIT % ks, down_q = units / ds, down_r = units % ds;
    const float r_ks = 1.0f / (float)ks, r_up = 1.0f / (float)up_e, r_cols = 1.0f / (float)cols,
                r_fu = 1.0f / (float)fu;

    // ---------------- items ----------------
    struct Item {
        int n0, slot, u0, u1;        // columns from n0; up: expert slot (-1: shared), both: units of K
        int tile, s;                 // slice of the tile's K
        bool up;
    };
    auto decode = [&](int q) {
        Item it;
        it.up = q < up_items;
        if (it.up) {
            it.tile = div24(q, ks, r_ks);
            it.s = q - it.tile * ks;
            it.u0 = it.s * up_q + min(it.s, up_r);
            it.u1 = it.u0 + up_q + (it.s < up_r ? 1 : 0);
            if (it.tile < up_sh) {
                it.slot = -1;
                it.n0 = it.tile * FEW_UP_COLS;
            } else {
                it.slot = div24(it.tile - up_sh, up_e, r_up);
                it.n0 = (it.tile - up_sh - it.slot * up_e) * FEW_UP_COLS;
            }
        } else {
            it.s = div24(q - up_items, cols, r_cols);
            it.tile = q - up_items - it.s * cols;
            it.n0 = it.tile * FEW_DOWN_COLS;
            it.u0 = it.s * down_q + min(it.s, down_r);
            it.u1 = it.u0 + down_q + (it.s < down_r ? 1 : 0);
            it.slot = 0;
        }
        return it;
    };
    // slot of a unit of the down product's K, -1 for the shared expert's
    auto slot_of = [&](int u) { return u < su ? -1 : div24(u - su, fu, r_fu); };
    const int kw = 32 * wave + 8 * g4;          // the lane's first row of a step
    auto down_ptr = [&](int u, int n0) {
        const int s = slot_of(u);
        const uint16_t *m = s < 0 ? g.Wd_s + (long)u * FEW_UNIT * d
                                  : g.Wd + ((long)s_list[s] * f + (long)(u - su - s * fu) * FEW_UNIT) * d;
        return m + (long)kw * d + n0 + 8 * r;
    };
    auto up_ptr = [&](const Item &it) {
        const long ld = it.slot < 0 ? fs : f;
        const uint16_t *m = it.slot < 0 ? (r < 8 ? g.Wg_s : g.Wu_s)
                                        : (r < 8 ? g.Wg : g.Wu) + (long)s_list[it.slot] * d * f;
        return m + ((long)it.u0 * FEW_UNIT + kw) * ld + it.n0 + 8 * (r & 7);
    };

    u32x4_t w0[8], w1[8];
    auto load = [&](u32x4_t (&w)[8], const uint16_t *p, long ld) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const u32x4_t *q = reinterpret_cast<const u32x4_t *>(p + j * ld);
            w[j] = PAST ? __builtin_nontemporal_load(q) : *q;
        }
    };
    f32x4_t acc[8];
    auto operand = [&](const u32x4_t (&w)[8], int i) {
        u32x4_t a;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            a[q] = __builtin_amdgcn_perm(w[2 * q + 1][i >> 1], w[2 * q][i >> 1],
                                         (i & 1) ? 0x07060302u : 0x05040100u);
        return __builtin_bit_cast(bf16x8_t, a);
    };
    auto mul = [&](const u32x4_t (&w)[8], u32x4_t x) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(operand(w, i), __builtin_bit_cast(bf16x8_t, x),
                                                             acc[i], 0, 0, 0);
    };
    auto mul2 = [&](const u32x4_t (&w)[8], u32x4_t xh, u32x4_t xl) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bf16x8_t a = operand(w, i);
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, xh), acc[i], 0, 0, 0);
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8_t, xl), acc[i], 0, 0, 0);
        }
    };
    auto clear = [&](f32x4_t (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    };
    const int tok = r < T ? r : T - 1;          // columns past T repeat the last token; nothing reads them
    const long plane = (long)units * T * FEW_UNIT;          // H: high parts, then low
    const uint16_t *H = g.H;

    int q = __builtin_amdgcn_readfirstlane(s_next);
    __syncthreads();                            // the search below and the first item's end write s_next again
    Item it = decode(q);
    const uint16_t *np = it.up ? up_ptr(it) : g.X;
    long nld = it.up ? (it.slot < 0 ? fs : f) : 0;
    if (q < items && !it.up) {
        np = down_ptr(it.u0, it.n0);
        nld = d;
    }
    load(w0, np, nld);
    // Before its first wait a workgroup looks whether all first items of the up product
    // are taken; one that is not belongs to a workgroup which has not started, and it
    // does that item itself, its own one (`held`) after it.
    const int first_ups = min((int)gridDim.x, up_items);
    bool waits = false;
    int held = -1;
    while (q < items) {
        if (!it.up && !waits) {
            if (wave == 0) {
                int i = -1;
                for (;;) {
                    const int c = __hip_atomic_load(firsts + lane % FEW_QUEUES * FEW_LINE, __ATOMIC_RELAXED,
                                                    __HIP_MEMORY_SCOPE_AGENT);
                    const unsigned long long left =
                        __ballot(lane < FEW_QUEUES && FEW_QUEUES * c + lane < first_ups);
                    if (!left) break;
                    const int from = __builtin_ctzll(left);
                    // (no add: behind the last up item are items that nobody else would do)
                    int n = c;
                    const bool won = lane == from && __hip_atomic_compare_exchange_strong(
                        firsts + from * FEW_LINE, &n, c + 1, __ATOMIC_RELAXED, __ATOMIC_RELAXED,
                        __HIP_MEMORY_SCOPE_AGENT);
                    if (__ballot(won)) {
                        i = FEW_QUEUES * __builtin_amdgcn_readlane(c, from) + from;
                        break;
                    }
                }
                if (lane == 0) s_next = i;
            }
            __syncthreads();
            const int i = __builtin_amdgcn_readfirstlane(s_next);
            __syncthreads();
            waits = i < 0;
            if (i >= 0) {
                held = q;
                q = i;
                it = decode(q);
                np = up_ptr(it);
                nld = it.slot < 0 ? fs : f;
                load(w0, np, nld);
            }
        }
        // the next item is asked for early, but by an item that waits not before it has
        // what it waited for: others would have nothing
        if (tid == 0 && held < 0 && it.up) next = add(queue) + gridDim.x;
        clear(acc);
        f32x4_t total[8];
        if (it.up) {
            const long ld = it.slot < 0 ? fs : f;
            const uint16_t *wp = np;
            const uint16_t *xp = g.X + (long)tok * d + (long)it.u0 * FEW_UNIT + kw;
            u32x4_t x0 = ld_u32x4(xp), x1;
#pragma unroll 1
            for (int u = it.u0; u < it.u1; ++u) {
                x1 = ld_u32x4(xp + 128);
                load(w1, wp + 128 * ld, ld);
                __builtin_amdgcn_sched_barrier(0);
                mul(w0, x0);
                __builtin_amdgcn_sched_barrier(0);
                xp += 256;
                wp += 256 * ld;
                if (u + 1 < it.u1) {
                    x0 = ld_u32x4(xp);
                    load(w0, wp, ld);
                }
                __builtin_amdgcn_sched_barrier(0);
                mul(w1, x1);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            clear(total);
            // the H of the item's rows
            const int sa = slot_of(it.u0), sb = slot_of(it.u1 - 1);
            if (tid <= sb - sa) {
                const int s = sa + tid;
                poll(h_done + FEW_LINE * (1 + s), s < 0 ? up_sh : up_e, err);
            }
            if (tid == 0 && sb - sa == 256) poll(h_done + FEW_LINE * (1 + sb), up_e, err);
            __syncthreads();
            if (tid == 0) next = add(queue) + gridDim.x;
            // A token that did not choose an expert takes the H of one that did: its
            // column is dropped, and the loads fetch no lines of their own.
            auto h_at = [&](int q) {
                const int chose = q < 0 ? 0 : s_mask[q], t = (chose >> r) & 1 ? r : __builtin_ctz(chose | 0x10000);
                return (q < 0 ? tok : t) * FEW_UNIT + kw;
            };
            int s = sa, left = s < 0 ? su - it.u0 : fu - (it.u0 - su - s * fu);    // units of it
            const uint16_t *hu = H + (long)it.u0 * T * FEW_UNIT, *wp = np;
            int at = h_at(s);
            u32x4_t h0 = ld_u32x4(hu + at), l0 = ld_u32x4(hu + plane + at), h1, l1;
#pragma unroll 1
            for (int u = it.u0; u < it.u1; ++u) {
                h1 = ld_u32x4(hu + at + 128);
                l1 = ld_u32x4(hu + plane + at + 128);
                load(w1, wp + 128l * d, d);
                __builtin_amdgcn_sched_barrier(0);
                mul2(w0, h0, l0);
                __builtin_amdgcn_sched_barrier(0);
                int sn = s;
                if (u + 1 < it.u1) {
                    hu += (long)T * FEW_UNIT;
                    wp += 256l * d;
                    if (--left == 0) {
                        sn = s + 1;
                        left = fu;
                        at = h_at(sn);
                        wp = down_ptr(u + 1, it.n0);
                    }
                    h0 = ld_u32x4(hu + at);
                    l0 = ld_u32x4(hu + plane + at);
                    load(w0, wp, d);
                }
                __builtin_amdgcn_sched_barrier(0);
                mul2(w1, h1, l1);
                __builtin_amdgcn_sched_barrier(0);
                if (u + 1 == it.u1 || sn != s) {
                    // an expert's part: its weight, or nothing, for this lane's token
                    const bool on = s < 0 || ((s_mask[s] >> r) & 1);
                    const float wt = s < 0 ? 1.f : on ? s_w[s][r] : 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int p = 0; p < 4; ++p) total[i][p] = total[i][p] + (on ? wt * acc[i][p] : 0.f);
                    clear(acc);
                    s = sn;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = total[i];
        }
        // ---------------- the waves' sums meet; the next item's loads leave ----------------
        // accumulators: lane (g4, r), register p of product i: column 8 (4 g4 + p) + i, token r
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<f32x4_t *>(&sh.red[wave][r][8 * (4 * g4 + p) + 4 * h]) =
                    f32x4_t{acc[4 * h][p], acc[4 * h + 1][p], acc[4 * h + 2][p], acc[4 * h + 3][p]};
        if (tid == 0) s_next = held < 0 ? next : held;
        held = -1;
        __syncthreads();
        const Item cur = it;
        q = __builtin_amdgcn_readfirstlane(s_next);
        it = decode(q);
        np = g.X;                            // none left: anything, once
        nld = 0;
        if (q < items) {
            np = it.up ? up_ptr(it) : down_ptr(it.u0, it.n0);
            nld = it.up ? (it.slot < 0 ? fs : f) : d;
        }
        // a thread finishes 4 columns of tokens et and et + 8
        const int en = 4 * (tid & 31);
        f32x4_t v[2];
#pragma unroll
        for (int eh = 0; eh < 2; ++eh) {
            const int et = (tid >> 5) + 8 * eh;
            v[eh] = *reinterpret_cast<const f32x4_t *>(&sh.red[0][et][en]);
#pragma unroll
            for (int w = 1; w < NW; ++w) {
                const f32x4_t u = *reinterpret_cast<const f32x4_t *>(&sh.red[w][et][en]);
#pragma unroll
                for (int p = 0; p < 4; ++p) v[eh][p] = v[eh][p] + u[p];
            }
        }
        // the sums of the whole K: H of an up tile, Y of a down tile
        auto finish = [&]() {
#pragma unroll
            for (int eh = 0; eh < 2; ++eh) {
                const int et = (tid >> 5) + 8 * eh;
                if (!cur.up) {
                    if (et < T)
                        *reinterpret_cast<u32x2_t *>(g.Y + (long)et * d + cur.n0 + en) =
                            u32x2_t{pack_bf2(v[eh][0], v[eh][1]), pack_bf2(v[eh][2], v[eh][3])};
                    continue;
                }
                // the first half of a token's threads hold the gate, the second the up columns
                const int unit = (cur.slot < 0 ? 0 : su + cur.slot * fu) + cur.n0 / FEW_UNIT;
                float h[4], l[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const float u = shfl_xor_f(v[eh][p], 16);
                    const float x = silu_f(v[eh][p]) * u;
                    h[p] = bf2f(f2bf(x));
                    // an infinite (or NaN) high part stands alone
                    l[p] = fabsf(h[p]) <= FLT_MAX ? x - h[p] : 0.f;
                }
                if (et < T && en < FEW_UP_COLS) {
                    uint16_t *p = g.H + ((long)unit * T + et) * FEW_UNIT + cur.n0 % FEW_UNIT + en;
                    st_agent(p, pack_bf2(h[0], h[1]), pack_bf2(h[2], h[3]));
                    st_agent(p + plane, pack_bf2(l[0], l[1]), pack_bf2(l[2], l[3]));
                }
            }
        };
        // Slices of K: each leaves its sums, [tile][slice][T][128], and the last one
        // to come adds all of them in order.
        const int slices = cur.up ? ks : ds;
        float *base = (cur.up ? g.up_part : g.y_part) + (long)cur.tile * slices * T * 128;
        if (slices > 1) {
#pragma unroll
            for (int eh = 0; eh < 2; ++eh) {
                const int et = (tid >> 5) + 8 * eh;
                if (et < T) st_agent(base + ((long)cur.s * T + et) * 128 + en, v[eh]);
            }
        } else {
            finish();
        }
        // the next item's first loads follow the stores
        asm volatile("" ::: "memory");
        load(w0, np, nld);
        stores_done<8>();
        __syncthreads();
        int *h_ctr = h_done + FEW_LINE * (1 + cur.slot);
        if (slices == 1) {
            if (tid == 0 && cur.up) add(h_ctr);
            continue;
        }
        if (tid == 0) s_last = add((cur.up ? up_done : down_done) + cur.tile) == slices - 1;
        __syncthreads();
        if (s_last) {
#pragma unroll
            for (int eh = 0; eh < 2; ++eh) {
                const int et = (tid >> 5) + 8 * eh;
                v[eh] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if (et < T)
#pragma unroll 8
                    for (int i = 0; i < slices; ++i) {
                        const f32x4_t u = *reinterpret_cast<const f32x4_t *>(base + ((long)i * T + et) * 128 + en);
#pragma unroll
                        for (int p = 0; p < 4; ++p) v[eh][p] = v[eh][p] + u[p];
                    }
            }
            finish();
            if (cur.up) {
                stores_done<0>();
                __syncthreads();
                if (tid == 0) add(h_ctr);
            }
        }
    }
}

}  // namespace

hipError_t launch_few(const FewArgs &g, hipStream_t st) {
    if (g.T <= 0) return hipSuccess;
    if (g.E % 4 == 0)
        few_router_kernel<4><<<dim3((unsigned)g.S, (unsigned)((g.E + 63) / 64)), dim3(64 * RW), 0, st>>>(g);
    else
        few_router_kernel<1><<<dim3((unsigned)g.S, (unsigned)((g.E + 15) / 16)), dim3(64 * RW), 0, st>>>(g);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (few_past_caches(g.T, g.d, g.E, g.k, g.f, g.fs)) few_kernel<true><<<dim3(FEW_WGS), dim3(NT), 0, st>>>(g);
    else few_kernel<false><<<dim3(FEW_WGS), dim3(NT), 0, st>>>(g);
    return hipGetLastError();
}
