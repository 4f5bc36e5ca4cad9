// The whole layer for up to 16 tokens (decoding) in two launches: the router's
// partial logits, and everything else -- selection by scores, both products of
// the experts and the sum.
//
// The work is a stream of the weights of the reached experts.  Workgroups take
// items from one queue: tiles of the up product (64 gate and 64 up columns, the
// shared expert's first), then tiles of the down product (128 columns, over the
// rows of all reached experts one after the other), each cut along K so that there
// are enough of them.  A tile of the down product waits for the H of its rows.  An
// item depends on items before it in the queue alone, which running workgroups have
// taken, so no wait needs a workgroup that has not started.
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
// rounded once.
#include <cfloat>

#include "common.h"
#include "few.h"
#include "kernels.h"

namespace {

constexpr float MASKED = -1e38f;

// ---------------------------------------------------------------- router
// Partial logits of a slice of the d axis: part [S][T][E].  W_r's rows go to RT
// threads, V experts each; 1024 / RT rows at a time.  Clears the counters, too.
template <int V, int TT>
__global__ __launch_bounds__(1024) void few_router_kernel(FewArgs g, int RT) {
    constexpr int CHUNK = 128, TC = TT < 4 ? TT : 4;
    __shared__ float xs[TT][CHUNK];
    __shared__ float red[TC][16][64 * V];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (blockIdx.x == 0)
        for (int i = tid; i < g.ncounters; i += 1024) g.counters[i] = 0;
    const int units = g.d / CHUNK, S = gridDim.x;
    const int u0 = (int)((long)units * blockIdx.x / S), u1 = (int)((long)units * (blockIdx.x + 1) / S);
    const int c = tid % RT, RG = 1024 / RT, rg = tid / RT, e0 = c * V;
    float acc[TT][V];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int v = 0; v < V; ++v) acc[t][v] = 0.f;
    for (int u = u0; u < u1; ++u) {
        const long k0 = (long)u * CHUNK;
        for (int i = tid; i < TT * CHUNK; i += 1024) {
            const int t = i / CHUNK;
            xs[t][i % CHUNK] = t < g.T ? bf2f(g.X[(long)t * g.d + k0 + i % CHUNK]) : 0.f;
        }
        __syncthreads();
        if (e0 < g.E)
            for (int r0 = rg; r0 < CHUNK; r0 += 8 * RG) {
                uint16_t w[8][V];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int r = r0 + j * RG;
                    const uint16_t *p = g.W_r + (k0 + (r < CHUNK ? r : r0)) * g.E + e0;
                    if constexpr (V == 4) {
                        const u32x2_t q = ld_u32x2(p);
                        w[j][0] = (uint16_t)q[0]; w[j][1] = (uint16_t)(q[0] >> 16);
                        w[j][2] = (uint16_t)q[1]; w[j][3] = (uint16_t)(q[1] >> 16);
                    } else {
                        w[j][0] = *p;
                    }
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int r = r0 + j * RG;
                    if (r >= CHUNK) break;
#pragma unroll
                    for (int t = 0; t < TT; ++t)
#pragma unroll
                        for (int v = 0; v < V; ++v) acc[t][v] = acc[t][v] + xs[t][r] * bf2f(w[j][v]);
                }
            }
        __syncthreads();
    }
    // rows of one wave, then the waves in order
    for (int m = RT; m < 64; m <<= 1)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int v = 0; v < V; ++v) acc[t][v] = acc[t][v] + shfl_xor_f(acc[t][v], m);
    const int span = RT < 64 ? 1 : RT / 64;          // waves side by side in a row
#pragma unroll
    for (int t0 = 0; t0 < TT; t0 += TC) {
        if (t0 >= g.T) break;
#pragma unroll
        for (int t = 0; t < TC; ++t)
#pragma unroll
            for (int v = 0; v < V; ++v) red[t][wave][lane * V + v] = acc[t0 + t][v];
        __syncthreads();
        for (int i = tid; i < TC * g.E; i += 1024) {
            const int t = i / g.E, e = i % g.E;
            if (t0 + t >= g.T) break;
            const int cc = e / V, w0 = cc / 64, at = (cc % 64) * V + e % V;
            float s = red[t][w0][at];
            for (int w = w0 + span; w < 16; w += span) s = s + red[t][w][at];
            g.part[((long)blockIdx.x * g.T + t0 + t) * g.E + e] = s;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- selection
// The same for every lane: largest of the wave's values.
DEV uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)v, m, 64);
        v = o > v ? o : v;
    }
    return v;
}
DEV double wave_sum_d(double v) {
#pragma unroll 1
    for (int m = 1; m < 64; m <<= 1) {
        const uint64_t b = (uint64_t)__double_as_longlong(v);
        const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)b, m, 64);
        const uint32_t hi = (uint32_t)__shfl_xor((int)(uint32_t)(b >> 32), m, 64);
        v += __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
    }
    return v;
}
DEV double shfl_d(double v, int src) {
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)b, src, 64);
    const uint32_t hi = (uint32_t)__shfl((int)(uint32_t)(b >> 32), src, 64);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
// Unsigned key with the order of the double, above 1.
DEV uint64_t rank_key(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);   // -0 and 0 are one
    return (b >> 63) ? ~b : (b | (1ull << 63));
}

// One token's experts, by one wave, ranked by 64-bit values as moe_route_scored
// defines them; compact loops, since a call fetches this code from memory once.
// z: its logits (LDS); val: room for E doubles; ids and w: its k places.
DEV void select_token(const FewArgs &g, const float *z, double *val, int *ids, float *w, int lane) {
    const ScoreArgs &a = g.score;
    const int E = g.E, n = E / a.groups, k = g.k;
    const bool by_score = g.balance || (a.groups > 1 && a.pair);
    const bool row_sum = !a.sigmoid && (by_score || !a.renorm);
    auto live = [&](int e) { return z[e] >= MASKED && (!g.balance || g.balance[e] >= MASKED); };
    float zmax = -INFINITY;
    double sum = 0.0;
    if (row_sum) {
        for (int e = lane; e < E; e += 64) zmax = fmaxf(zmax, live(e) ? fminf(z[e], FLT_MAX) : -INFINITY);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) zmax = fmaxf(zmax, shfl_xor_f(zmax, m));
    }
#pragma unroll 1
    for (int e = lane; e < E; e += 64) {
        double v = (double)fminf(z[e], FLT_MAX);
        if (by_score || row_sum) {
            const double x = exp(a.sigmoid ? -v : v - (double)zmax);
            if (live(e)) sum += x;
            if (by_score) v = a.sigmoid ? 1.0 / (1.0 + x) : x;
        }
        val[e] = v;
    }
    if (row_sum) sum = wave_sum_d(sum);
#pragma unroll 1
    for (int e = lane; e < E; e += 64) {
        double v = val[e];
        if (by_score) {
            if (!a.sigmoid) v = v / sum;
            if (g.balance) v += (double)g.balance[e];
        }
        val[e] = live(e) ? v : -INFINITY;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // groups: lpg lanes each
    uint64_t kept = ~0ull;
    int lpg = 64;
    if (a.groups > 1) {
        while (lpg * a.groups > 64) lpg >>= 1;
        const int grp = lane / lpg;
        double b1 = -INFINITY, b2 = -INFINITY;
        if (grp < a.groups)
#pragma unroll 1
            for (int i = lane % lpg; i < n; i += lpg) {
                const double v = val[grp * n + i];
                b2 = fmax(b2, fmin(b1, v));
                b1 = fmax(b1, v);
            }
#pragma unroll 1
        for (int m = 1; m < lpg; m <<= 1) {
            const double o1 = shfl_d(b1, lane ^ m), o2 = shfl_d(b2, lane ^ m);
            b2 = fmax(fmin(b1, o1), fmax(b2, o2));
            b1 = fmax(b1, o1);
        }
        const double gs = a.pair && b2 > -INFINITY ? b1 + b2 : b1;
        int better = 0;
#pragma unroll 1
        for (int o = 0; o < a.groups; ++o) {
            const double og = shfl_d(gs, o * lpg);
            better += og > gs || (og == gs && o < grp) ? 1 : 0;
        }
        kept = __ballot(better < a.top_groups);
    }
    // the lane's experts: `per` consecutive ones, so that lower lanes hold lower ids
    const int per = (E + 63) / 64;
    uint64_t key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = lane * per + i;
        key[i] = 0;
        if (i < per && e < E && (a.groups == 1 || ((kept >> (e / n * lpg)) & 1)))
            key[i] = val[e] > -INFINITY ? rank_key(val[e]) : 1;
    }
    uint32_t chosen = 0;
#pragma unroll 1
    for (int r = 0; r < k; ++r) {
        uint64_t best = key[0];
        int at = 0;
#pragma unroll
        for (int i = 1; i < 4; ++i)
            if (key[i] > best) {
                best = key[i];
                at = i;
            }
        const uint32_t hi = (uint32_t)(best >> 32), lo = (uint32_t)best;
        uint32_t m = wave_max(hi);
        unsigned long long c = __ballot(hi == m);
        if (c & (c - 1)) {
            const uint32_t l = wave_max(hi == m ? lo : 0u);
            c = __ballot(hi == m && lo == l);
        }
        if (lane == __builtin_ctzll(c)) {
            chosen |= 1u << at;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i == at) key[i] = 0;
        }
    }
    // places in ascending id
    int before = 0;
    const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < 4; ++i) before += __popcll(__ballot((chosen >> i) & 1) & below);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((chosen >> i) & 1) ids[before++] = lane * per + i;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // weights: lane j takes place j; renormalised ones are ratios of scores, taken
    // to the largest of them, so that scores that underflow together keep theirs
    const int id = lane < k ? ids[lane] : 0;
    const bool on = lane < k && live(id);
    const float zc = on ? fminf(z[id], FLT_MAX) : 0.f;
    float u = 0.f, total = 1.f;
    if (a.renorm) {
        float m = on ? (a.sigmoid ? fminf(zc, 0.f) : zc) : -INFINITY;
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) m = fmaxf(m, shfl_xor_f(m, x));
        const float x = expf((a.sigmoid ? fminf(zc, 0.f) : zc) - m);
        if (on) u = a.sigmoid ? x / (1.0f + expf(-fabsf(zc))) : x;
        total = u;
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) total = total + shfl_xor_f(total, x);
    } else if (on) {
        const float x = expf(a.sigmoid ? -zc : zc - zmax);
        u = a.sigmoid ? 1.0f / (1.0f + x) : x / (float)sum;
    }
    if (lane < k) w[lane] = u > 0.f ? a.scale * (u / total) : 0.f;
}

// ---------------------------------------------------------------- the layer
// Waits between workgroups.  A producer's waves have stored, wait for that
// (vmcnt), meet at a barrier, and one thread adds to a counter with release; a
// consumer's thread polls, and its workgroup acquires behind a barrier.  Waits end
// after 0.2 s in any case (wall clock of 100 MHz), with the error word set.
constexpr unsigned long long WAIT_TICKS = 20000000ull;
DEV void poll(const int *ctr, int need, int *err) {
    const unsigned long long t0 = wall_clock64();
    while (__hip_atomic_load(ctr, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < need) {
        if (__hip_atomic_load(err, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) return;
        if (wall_clock64() - t0 > WAIT_TICKS) {
            __hip_atomic_store(err, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            return;
        }
        __builtin_amdgcn_s_sleep(1);
    }
}
DEV void acquire() { __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent"); }
DEV void stores_done() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}
DEV int add_release(int *ctr) {
    return __hip_atomic_fetch_add(ctr, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
}

constexpr int NW = 4, PITCH = 128 + 4;

struct Select {                      // scratch of the start
    float z[FEW_MAX_T * 256];
    double val[NW][256];
    int ids[FEW_MAX_T][16];
    float w[FEW_MAX_T][16];
    uint32_t mask[256];
    int slot_of[256];
    int cnt[NW];
};

__global__ __launch_bounds__(64 * NW, 2) void few_kernel(FewArgs g) {
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
    int *err = g.counters, *queue = g.counters + 1, *h_done = g.counters + 4;
    int *up_done = h_done + 257, *down_done = up_done + g.up_counters;

    if (tid == 0) s_next = __hip_atomic_fetch_add(queue, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // ---------------- routing: every workgroup for itself ----------------
    {
        Select &s = sh.sel;
        for (int i = tid; i < T * g.E; i += 64 * NW) {
            float v = 0.f;
#pragma unroll 4
            for (int q = 0; q < g.S; ++q) v = v + g.part[(long)q * T * g.E + i];
            if (g.bias) v = v + g.bias[i % g.E];
            s.z[i] = v;
        }
        s.mask[tid] = 0;
        __syncthreads();
#pragma unroll 1
        for (int t = wave; t < T; t += NW)
            select_token(g, s.z + t * g.E, s.val[wave], s.ids[t], s.w[t], lane);
        __syncthreads();
        const int t = tid / 16, j = tid % 16;
        const bool route = t < T && j < g.k;
        if (route) atomicOr(&s.mask[s.ids[t][j]], 1u << t);
        __syncthreads();
        const unsigned long long b = __ballot(s.mask[tid] != 0);
        if (lane == 0) s.cnt[wave] = __popcll(b);
        __syncthreads();
        int at = __popcll(b & ((1ull << lane) - 1));
        for (int w = 0; w < wave; ++w) at += s.cnt[w];
        if (s.mask[tid]) {
            s_list[at] = tid;
            s_mask[at] = (int)s.mask[tid];
            s.slot_of[tid] = at;
        }
        __syncthreads();
        if (route) s_w[s.slot_of[s.ids[t][j]]][t] = s.w[t][j];
        if (blockIdx.x == 0) {
            if (route) {
                g.topk_idx[t * g.k + j] = s.ids[t][j];
                g.topk_w[t * g.k + j] = s.w[t][j];
            }
            for (int i = tid; i < T * g.E; i += 64 * NW) g.logits[i] = s.z[i];
        }
        if (tid == 0) s_last = s.cnt[0] + s.cnt[1] + s.cnt[2] + s.cnt[3];
        __syncthreads();
    }
    const int slots = __builtin_amdgcn_readfirstlane(s_last);
    const int fu = f / FEW_UNIT, su = fs / FEW_UNIT, units = su + slots * fu;
    const int up_sh = fs / FEW_UP_COLS, up_e = f / FEW_UP_COLS, up_tiles = up_sh + slots * up_e;
    const int ks = few_slices(up_tiles, d / FEW_UNIT);
    const int cols = d / FEW_DOWN_COLS, ds = few_slices(cols, units);
    const int up_items = up_tiles * ks, items = up_items + cols * ds;

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
            it.tile = q / ks;
            it.s = q - it.tile * ks;
            const int n = d / FEW_UNIT;
            it.u0 = (int)((long)n * it.s / ks);
            it.u1 = (int)((long)n * (it.s + 1) / ks);
            if (it.tile < up_sh) {
                it.slot = -1;
                it.n0 = it.tile * FEW_UP_COLS;
            } else {
                it.slot = (it.tile - up_sh) / up_e;
                it.n0 = (it.tile - up_sh - it.slot * up_e) * FEW_UP_COLS;
            }
        } else {
            it.s = (q - up_items) / cols;
            it.tile = q - up_items - it.s * cols;
            it.n0 = it.tile * FEW_DOWN_COLS;
            it.u0 = (int)((long)units * it.s / ds);
            it.u1 = (int)((long)units * (it.s + 1) / ds);
            it.slot = 0;
        }
        return it;
    };
    // slot of a unit of the down product's K, -1 for the shared expert's
    auto slot_of = [&](int u) { return u < su ? -1 : (u - su) / fu; };
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
        for (int j = 0; j < 8; ++j) w[j] = ld_u32x4(p + j * ld);
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
    Item it = decode(q);
    if (q < items) {
        if (it.up) load(w0, up_ptr(it), it.slot < 0 ? fs : f);
        else load(w0, down_ptr(it.u0, it.n0), d);
    }
    while (q < items) {
        int next = 0;
        if (tid == 0) next = __hip_atomic_fetch_add(queue, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        clear(acc);
        f32x4_t total[8];
        if (it.up) {
            const long ld = it.slot < 0 ? fs : f;
            const uint16_t *wp = up_ptr(it);
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
                poll(h_done + 1 + s, s < 0 ? up_sh : up_e, err);
            }
            if (tid == 0 && sb - sa == 256) poll(h_done + 1 + sb, up_e, err);
            __syncthreads();
            acquire();
            const uint16_t *hp = H + ((long)it.u0 * T + tok) * FEW_UNIT + kw;
            u32x4_t h0 = ld_u32x4(hp), l0 = ld_u32x4(hp + plane), h1, l1;
            int s = sa;
            const uint16_t *wp = down_ptr(it.u0, it.n0);
#pragma unroll 1
            for (int u = it.u0; u < it.u1; ++u) {
                h1 = ld_u32x4(hp + 128);
                l1 = ld_u32x4(hp + plane + 128);
                load(w1, wp + 128l * d, d);
                __builtin_amdgcn_sched_barrier(0);
                mul2(w0, h0, l0);
                __builtin_amdgcn_sched_barrier(0);
                hp += (long)T * FEW_UNIT;
                int sn = s;
                if (u + 1 < it.u1) {
                    h0 = ld_u32x4(hp);
                    l0 = ld_u32x4(hp + plane);
                    wp = down_ptr(u + 1, it.n0);
                    load(w0, wp, d);
                    sn = slot_of(u + 1);
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
        if (tid == 0) s_next = next;
        __syncthreads();
        const Item cur = it;
        q = __builtin_amdgcn_readfirstlane(s_next);
        it = decode(q);
        if (q < items) {
            if (it.up) load(w0, up_ptr(it), it.slot < 0 ? fs : f);
            else load(w0, down_ptr(it.u0, it.n0), d);
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
        // Slices of K: each leaves its sums, the last one to come adds all of them in order.
        const int slices = cur.up ? ks : ds;
        bool finish = true;
        if (slices > 1) {
            // [tile][slice][T][128]
            float *base = (cur.up ? g.up_part : g.y_part) + (long)cur.tile * slices * T * 128;
#pragma unroll
            for (int eh = 0; eh < 2; ++eh) {
                const int et = (tid >> 5) + 8 * eh;
                if (et < T) *reinterpret_cast<f32x4_t *>(base + ((long)cur.s * T + et) * 128 + en) = v[eh];
            }
            stores_done();
            if (tid == 0) s_last = add_release((cur.up ? up_done : down_done) + cur.tile) == slices - 1;
            __syncthreads();
            finish = s_last != 0;
            if (finish) {
                acquire();
#pragma unroll
                for (int eh = 0; eh < 2; ++eh) {
                    const int et = (tid >> 5) + 8 * eh;
                    v[eh] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                    if (et < T)
#pragma unroll 4
                        for (int i = 0; i < slices; ++i) {
                            const f32x4_t u = *reinterpret_cast<const f32x4_t *>(base + ((long)i * T + et) * 128 + en);
#pragma unroll
                            for (int p = 0; p < 4; ++p) v[eh][p] = v[eh][p] + u[p];
                        }
                }
            }
        }
        if (finish && cur.up) {
            // the first half of a token's threads hold the gate, the second the up columns
            const int unit = (cur.slot < 0 ? 0 : su + cur.slot * fu) + cur.n0 / FEW_UNIT;
#pragma unroll
            for (int eh = 0; eh < 2; ++eh) {
                const int et = (tid >> 5) + 8 * eh;
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
                    *reinterpret_cast<u32x2_t *>(p) = u32x2_t{pack_bf2(h[0], h[1]), pack_bf2(h[2], h[3])};
                    *reinterpret_cast<u32x2_t *>(p + plane) = u32x2_t{pack_bf2(l[0], l[1]), pack_bf2(l[2], l[3])};
                }
            }
            stores_done();
            if (tid == 0) add_release(h_done + 1 + cur.slot);
        } else if (finish) {
#pragma unroll
            for (int eh = 0; eh < 2; ++eh) {
                const int et = (tid >> 5) + 8 * eh;
                if (et < T)
                    *reinterpret_cast<u32x2_t *>(g.Y + (long)et * d + cur.n0 + en) =
                        u32x2_t{pack_bf2(v[eh][0], v[eh][1]), pack_bf2(v[eh][2], v[eh][3])};
            }
        }
        __syncthreads();                     // red and s_last are free again
    }
}

}  // namespace

hipError_t launch_few(const FewArgs &g, hipStream_t st) {
    if (g.T <= 0) return hipSuccess;
    int RT = 1;
    const int V = g.E % 4 ? 1 : 4;
    while (RT * V < g.E) RT *= 2;
#define FEW_ROUTER(V, TT) few_router_kernel<V, TT><<<dim3(g.S), dim3(1024), 0, st>>>(g, RT)
    if (V == 4) {
        if (g.T == 1) FEW_ROUTER(4, 1);
        else if (g.T <= 4) FEW_ROUTER(4, 4);
        else FEW_ROUTER(4, 16);
    } else {
        if (g.T == 1) FEW_ROUTER(1, 1);
        else if (g.T <= 4) FEW_ROUTER(1, 4);
        else FEW_ROUTER(1, 16);
    }
#undef FEW_ROUTER
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    few_kernel<<<dim3(FEW_WGS), dim3(64 * NW), 0, st>>>(g);
    return hipGetLastError();
}
