// What stands between two blocks of a model: a block's output y goes back into
// the residual stream x, and the next block's input h is made from the sum r.
//
//   n = N_y(y)                        none, RMS or layer norm, with weight and bias
//   v = n / (1 - drop) where kept, else 0
//   r = x + scale gate[c] token_gate[t] v     rounded to the stream's type
//   h = N_r(r)                        of the stored r
//
// and the gradient, D being the whole gradient of r:
//   D  = dr + N_r^T dh                dx = D
//   dv = scale gate token_gate D      dn = dv / (1 - drop) where kept, else 0
//   dy = N_y^T dn                     N^T g = s (g w - u mean(g w u) - mean(g w)),
// u the row without mean and divided by its deviation 1 / s (an RMS norm has no
// mean and no last term).  Weights, biases and the gate get sums over the rows,
// the token gates sums over the columns.
//
// Both are one pass over memory: a row lies in the registers of G threads, 8 CH
// values each, from its load to its store, and its sums meet through DPP and LDS.
// The mask of the dropout is computed again where it is needed (Philox4x32-10:
// Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011;
// 8 elements per block of the generator).
//
// Statistics, sums and everything between load and store are fp32.  r is rounded
// where it is stored, and h is made from that value, which is what the backward and
// the next block find; h and dy are bf16, as the layer's inputs and outputs.
//
// Bound by memory: 16384 x 7168 in bf16 162 us (0.94 GB, 5.8 TB/s), its gradient 312 (1.41
// GB, 4.5; a copy of 2 GiB 4.9).  The gradient has 40 vector instructions for an element
// and those of the generator, 55 % of the SIMDs' time, between two sums over the row, so
// what counts is that a row's loads are on their way during the row before it, and that
// nothing waits behind them: weights from memory instead of LDS return after them (367
// us), and so do registers that are spilt: sums that neither three of RMS norms (SUMS 13) nor
// three of the sum's norm and the gate (7) cover take the form with room for all five, which
// spills 38 of them at 4096 to 8192 columns, 88 with an fp32 stream.  The same size takes 690
// (RMS, then layer norm) to 754 us (two layer norms) there, in fp32 999 to 1040; with three
// sums in fp32, 11 spilt, 535.
// Tried and slower: 1024 threads of 8 values for such a row (128 registers; 378 us), rows
// of two workgroups on a CU, each with its own sums (390).
#include <algorithm>
#include <cfloat>

#include "common.h"
#include "kernels.h"
#include "rules.h"

namespace {

// ---------------------------------------------------------------- dropout
// 16 bits per element of a chunk of 8: the chunk's four words
struct Words { uint32_t w[4]; };

DEV Words philox(uint64_t seed, uint64_t offset, uint32_t chunk, uint32_t row) {
    uint32_t c0 = chunk, c1 = row, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}
// n where kept, else 0; out: what an element's 16 bits must reach
DEV f32x8 drop8(const f32x8 &n, const Words &w, uint32_t out) {
    f32x8 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = (uint16_t)w.w[i] >= (uint16_t)out ? n[2 * i] : 0.f;
        v[2 * i + 1] = w.w[i] >= out << 16 ? n[2 * i + 1] : 0.f;
    }
    return v;
}

// ---------------------------------------------------------------- rows
// PAST: past the caches, which hold none of what is that large.
template <bool PAST>
DEV u32x4_t ld16(const void *p) {
    const u32x4_t *q = reinterpret_cast<const u32x4_t *>(p);
    return PAST ? __builtin_nontemporal_load(q) : *q;
}
template <bool PAST>
DEV void st16(void *p, u32x4_t v) {
    u32x4_t *q = reinterpret_cast<u32x4_t *>(p);
    if constexpr (PAST) __builtin_nontemporal_store(v, q);
    else *q = v;
}
// 8 consecutive values as they lie in memory
template <bool F32> struct Raw;
template <> struct Raw<false> {
    u32x4_t a;
    template <bool PAST = false>
    DEV void load(const void *p, int i) { a = ld16<PAST>((const uint16_t *)p + i); }
    DEV void clear() { a = u32x4_t{0u, 0u, 0u, 0u}; }
    DEV f32x8 get() const {
        return f32x8{bf_lo(a[0]), bf_hi(a[0]), bf_lo(a[1]), bf_hi(a[1]),
                     bf_lo(a[2]), bf_hi(a[2]), bf_lo(a[3]), bf_hi(a[3])};
    }
};
template <> struct Raw<true> {
    u32x4_t a, b;
    template <bool PAST = false>
    DEV void load(const void *p, int i) {
        a = ld16<PAST>((const float *)p + i);
        b = ld16<PAST>((const float *)p + i + 4);
    }
    DEV void clear() { a = b = u32x4_t{0u, 0u, 0u, 0u}; }
    DEV f32x8 get() const {
        f32x8 v;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            v[q] = __uint_as_float(a[q]);
            v[4 + q] = __uint_as_float(b[q]);
        }
        return v;
    }
};
template <bool F32, bool PAST = false>
DEV void put(void *p, int i, const f32x8 &v) {
    if constexpr (F32) {
        u32x4_t lo, hi;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            lo[q] = __float_as_uint(v[q]);
            hi[q] = __float_as_uint(v[4 + q]);
        }
        st16<PAST>((float *)p + i, lo);
        st16<PAST>((float *)p + i + 4, hi);
    } else {
        st16<PAST>((uint16_t *)p + i, pack_bf8(v));
    }
}

// ---------------------------------------------------------------- sums over a row
template <int CTRL>
DEV float add_peer(float v) {
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
template <int CTRL, int ROWS>
DEV float add_before(float v) {
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, ROWS, 0xF, false));
}
// Over N = 1, 2, 4, 8 or 16 neighbouring lanes, the same in each: quads, then
// mirrored half rows and rows.
template <int N>
DEV float lanes_sum(float v) {
    if constexpr (N > 1) v = add_peer<0xB1>(v);
    if constexpr (N > 2) v = add_peer<0x4E>(v);
    if constexpr (N > 4) v = add_peer<0x141>(v);
    if constexpr (N > 8) v = add_peer<0x140>(v);
    return v;
}
// Over the wave, in its last lane.
DEV float wave_sum_last(float v) {
    v = lanes_sum<16>(v);
    v = add_before<0x142, 0xA>(v);           // lane 15 of the row before
    return add_before<0x143, 0xC>(v);        // lane 31
}
// N sums over the G threads of a row, the same in each of them.  Rows of more
// than a wave meet in `red` (a slot per wave), which must not be written again
// before every thread has passed another barrier: callers alternate.
template <int G, int N>
DEV void row_sums(float (&v)[N], float (*red)[4]) {
    if constexpr (G < 64) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = lanes_sum<(G < 16 ? G : 16)>(v[i]);
            if constexpr (G == 32) v[i] = v[i] + shfl_xor_f(v[i], 16);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum_last(v[i]);
    if constexpr (G == 64) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v[i]), 63));
    } else {
        constexpr int W = G < 64 ? 1 : G / 64;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if (lane == 63)
#pragma unroll
            for (int i = 0; i < N; ++i) red[wave][i] = v[i];
        __syncthreads();
        const float *from = red[wave / W * W + lane % W];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lanes_sum<W>(from[i]);
    }
}
DEV float sum8(const f32x8 &v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
// Which of its workgroup's rows a thread has: of whole waves, so that addresses are scalar
template <int G>
DEV int row_of_thread() {
    return G >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : (int)threadIdx.x / G;
}
DEV float dot8(const f32x8 &a, const f32x8 &b) {
    float x = a[0] * b[0], y = a[1] * b[1];
#pragma unroll
    for (int i = 2; i < 8; i += 2) {
        x = fmaf(a[i], b[i], x);
        y = fmaf(a[i + 1], b[i + 1], y);
    }
    return x + y;
}
DEV f32x8 zero8() { return f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }

// The pointer, for loads that are to stay where they are: weights that the compiler
// moves out of the loop over the rows take registers that the sums need.
DEV const float *again(const float *p) {
    asm volatile("" : "+s"(p));
    return p;
}

DEV float dev_inv(float var, float eps) { return 1.0f / sqrtf(var + eps); }

// ---------------------------------------------------------------- forward
// Values past the row's end are loaded as zeros.  ROWS: a workgroup takes rows in
// steps of the whole grid, with the weights in LDS and each row asked for while the
// one before is worked on, past the caches (16384 x 7168: 162 us, through them 173); otherwise
// NT / G rows.
template <bool F32, bool ROWS, int NT, int G, int CH>
__global__ __launch_bounds__(NT) void join_forward_kernel(JoinArgs g) {
    constexpr int NG = NT / G, SZ = F32 ? 4 : 2;
    __shared__ float red[ROWS ? 8 : 4][NT / 64][4];
    extern __shared__ __attribute__((aligned(16))) float w_lds[];
    const int lane = threadIdx.x % G;
    const float inv_d = 1.0f / (float)g.d;
    bool ok[CH];
    int col[CH];
    Raw<F32> xr[CH];
    Raw<false> yr[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        col[c] = 8 * (lane + G * c);
        ok[c] = col[c] < g.d;
        if (!ok[c]) col[c] = 0;
        xr[c].clear();
        yr[c].clear();
    }
    enum { YW, YB, GATE, RW, RB };
    const float *weights[5] = {g.y_weight, g.y_bias, g.gate, g.r_weight, g.r_bias};
    int at[5], n_w = 0;
#pragma unroll
    for (int a = 0; a < 5; ++a) at[a] = weights[a] ? n_w++ * g.d : 0;
    auto weight = [&](int a, int c) {
        if constexpr (!ROWS) return ld_f32x8(weights[a] + col[c]);
        const float *p = w_lds + at[a] + col[c] / 2;
        const f32x4_t lo = *reinterpret_cast<const f32x4_t *>(p);
        const f32x4_t hi = *reinterpret_cast<const f32x4_t *>(p + g.d / 2);
        return f32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    uint64_t seed = 0, offset = 0;
    if (g.rng) {
        seed = (uint64_t)g.rng[0];
        offset = (uint64_t)g.rng[1];
    }
    const long step = (long)gridDim.x * NG, rounds = ROWS ? (g.T + step - 1) / step : 1;
    long row = g.row0 + (long)blockIdx.x * NG + row_of_thread<G>();
    if (!ROWS && G <= 64 && row >= g.T) return;      // no barriers then
    // (a row past the last is the last one again, and not stored)
    auto load_x = [&](long t) {
        const size_t i = (size_t)((t < g.T ? t : g.T - 1) * g.d);
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (ok[c]) xr[c].template load<ROWS>((const char *)g.x + i * SZ, col[c]);
    };
    auto load_y = [&](long t) {
        const size_t i = (size_t)((t < g.T ? t : g.T - 1) * g.d);
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (ok[c] && g.y) yr[c].template load<ROWS>(g.y + i, col[c]);
    };
    load_x(row);
    load_y(row);
    if constexpr (ROWS) {                    // two planes of 4 columns of 8 each
#pragma unroll
        for (int a = 0; a < 5; ++a)
            if (weights[a])
                for (int j = threadIdx.x; j < g.d / 4; j += NT)
                    *reinterpret_cast<f32x4_t *>(w_lds + at[a] + (j & 1) * (g.d / 2) + 4 * (j >> 1)) =
                        *reinterpret_cast<const f32x4_t *>(weights[a] + 4 * j);
        __syncthreads();
    }
    for (long k = 0; k < rounds; ++k, row += step) {
        const bool on = row < g.T;
        const long t = on ? row : g.T - 1;
        const size_t i = (size_t)(t * g.d);
        float (*slots)[NT / 64][4] = red + (ROWS ? 4 * (k & 1) : 0);
        float ym = 0.f, ys = 0.f, rm = 0.f, rs = 0.f;
        // mean and 1 / deviation of the row in v
        auto stats = [&](const f32x8 (&v)[CH], int kind, float eps, float &m, float &s, int slot) {
            float sum[1] = {0.f};
            if (kind == JOIN_LAYER) {
#pragma unroll
                for (int c = 0; c < CH; ++c) sum[0] = sum[0] + sum8(v[c]);
                row_sums<G>(sum, slots[slot]);
                m = sum[0] * inv_d;
                sum[0] = 0.f;
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const f32x8 u = v[c] - m;
                    const float q = dot8(u, u);
                    sum[0] = sum[0] + (ok[c] ? q : 0.f);
                }
            } else {
#pragma unroll
                for (int c = 0; c < CH; ++c) sum[0] = sum[0] + dot8(v[c], v[c]);
            }
            row_sums<G>(sum, slots[slot + 1]);
            s = dev_inv(sum[0] * inv_d, eps);
        };
        auto normed = [&](const f32x8 &v, int kind, float m, float s, int w, int b, int c) {
            f32x8 n = kind == JOIN_LAYER ? (v - m) * s : v * s;
            if (weights[w]) n = n * weight(w, c);
            if (weights[b]) n = n + weight(b, c);
            return n;
        };
        f32x8 r[CH];
        if (g.y) {
#pragma unroll
            for (int c = 0; c < CH; ++c) r[c] = yr[c].get();
            if constexpr (ROWS) load_y(row + step);
            if (g.y_norm) {
                stats(r, g.y_norm, g.y_eps, ym, ys, 0);
#pragma unroll
                for (int c = 0; c < CH; ++c) r[c] = normed(r[c], g.y_norm, ym, ys, YW, YB, c);
            }
            const float a = g.scale * g.keep * (g.token_gate ? g.token_gate[t] : 1.f);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                f32x8 v = r[c];
                if (g.gate) v = v * weight(GATE, c);
                v = v * a;
                if (g.rng) v = drop8(v, philox(seed, offset, (uint32_t)col[c] / 8, (uint32_t)t), g.out);
                r[c] = xr[c].get() + v;
                if constexpr (!F32) {
                    Raw<false> q;
                    q.a = pack_bf8(r[c]);
                    r[c] = q.get();
                    if (on && ok[c]) st16<ROWS>((uint16_t *)g.r + i + col[c], q.a);
                } else {
                    if (on && ok[c]) put<true, ROWS>((float *)g.r + i, col[c], r[c]);
                }
                if (!ok[c]) r[c] = zero8();          // what a bias has left there
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) r[c] = xr[c].get();
        }
        if constexpr (ROWS) load_x(row + step);
        if (g.r_norm) stats(r, g.r_norm, g.r_eps, rm, rs, 2);
        if (g.h)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (g.r_norm) r[c] = normed(r[c], g.r_norm, rm, rs, RW, RB, c);
                if (on && ok[c]) put<false, ROWS>(g.h + i, col[c], r[c]);
            }
        if (g.stats && on && lane == 0)
            *reinterpret_cast<f32x4_t *>(g.stats + 4 * t) = f32x4_t{ym, ys, rm, rs};
    }
}

// ---------------------------------------------------------------- backward
// A workgroup takes rows in steps of the whole grid, G threads to a row, and keeps its
// sums over them in registers; each row is loaded one step ahead.  What lies past
// a row's end, and rows past the last, are zeros.  SUMS: the sums it has room for;
// LAYER: the norms may be layer norms.  ONCE: there is one round of rows, and nothing to
// hold over rounds (1 x 7168 13.4 -> 7.6 us, 256 x 7168 32 -> 22, 256 x 2048 15.1 -> 14).  (All five sums and both means take 40 more
// registers than a thread of 1024 has.)
template <bool F32, int SUMS, bool LAYER, int NT, int G, int CH, bool ONCE = false>
__global__ __launch_bounds__(NT) void join_backward_kernel(JoinArgs g) {
    constexpr int NG = NT / G;
    __shared__ float red[4][NT / 64][4];
    // weights, where they fit; in the end [d] sums if NG > 1
    extern __shared__ __attribute__((aligned(16))) float cols[];
    constexpr bool LDS_W = CH <= 2 && !ONCE;          // (beyond, they would take up to 256 KB)
    const int lane = threadIdx.x % G, group = row_of_thread<G>();
    const float inv_d = 1.0f / (float)g.d;
    bool ok[CH];
    int col[CH];
    f32x8 sum[5][CH];        // weight and bias of r's norm, gate, weight and bias of y's
    const int sums = g.sums & SUMS;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        col[c] = 8 * (lane + G * c);
        ok[c] = col[c] < g.d;
        if (!ok[c]) col[c] = 0;
#pragma unroll
        for (int a = 0; a < 5; ++a) sum[a][c] = zero8();
    }
    // Weights come from LDS: a load from memory would return after the next row's,
    // which are asked for before it.  Two planes of 4 columns of 8 each.
    const float *weights[4] = {g.r_weight, g.y_weight, g.y_bias, g.gate};
    int at[4], n_w = 0;
#pragma unroll
    for (int a = 0; a < 4; ++a) at[a] = weights[a] ? n_w++ * g.d : 0;
    auto weight = [&](int a, int c) {
        if constexpr (!LDS_W) return ld_f32x8((ONCE ? weights[a] : again(weights[a])) + col[c]);
        const float *p = cols + at[a] + col[c] / 2;
        const f32x4_t lo = *reinterpret_cast<const f32x4_t *>(p);
        const f32x4_t hi = *reinterpret_cast<const f32x4_t *>(p + g.d / 2);
        return f32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    enum { RW, YW, YB, GATE };
    uint64_t seed = 0, offset = 0;
    if (g.rng) {
        seed = (uint64_t)g.rng[0];
        offset = (uint64_t)g.rng[1];
    }
    Raw<F32> rr[CH], dr[CH];
    Raw<false> yr[CH], hr[CH];
    f32x4_t st = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const long step = (long)gridDim.x * NG, rounds = ONCE ? 1 : (g.T + step - 1) / step;
    long row = (long)blockIdx.x * NG + group;
#pragma unroll
    for (int c = 0; c < CH; ++c) {           // lanes past the row's end keep the zeros
        rr[c].clear();
        dr[c].clear();
        yr[c].clear();
        hr[c].clear();
    }
    constexpr int SZ = F32 ? 4 : 2;
    auto load_r = [&](long t) {
        const size_t i = (size_t)(t * g.d);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (t >= g.T) {
                rr[c].clear();
                hr[c].clear();
            } else if (ok[c]) {
                if (g.dh && g.r_norm) rr[c].load((const char *)g.r_in + i * SZ, col[c]);
                if (g.dh) hr[c].load(g.dh + i, col[c]);
            }
        }
    };
    auto load_dr = [&](long t) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (t >= g.T) dr[c].clear();
            else if (g.dr && ok[c]) dr[c].load((const char *)g.dr + (size_t)(t * g.d) * SZ, col[c]);
        }
    };
    auto load_y = [&](long t) {
        st = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (t < g.T) st = *reinterpret_cast<const f32x4_t *>(g.stats_in + 4 * t);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (t >= g.T) yr[c].clear();
            else if (g.y && ok[c]) yr[c].load(g.y + t * g.d, col[c]);
        }
    };
    load_r(row);
    load_dr(row);
    load_y(row);
    // Weights of y's norm that can make a finite row infinite, NaN ones too (true where nobody asks):
    // its values are within sqrt(d) < 2^7 deviations, so 2^119 leaves all of them below 2^127.
    bool odd_weights = true;
    if constexpr (LDS_W) {
        bool odd = false;
#pragma unroll
        for (int a = 0; a < 4; ++a)
            if (weights[a])
                for (int j = threadIdx.x; j < g.d / 4; j += NT) {
                    const f32x4_t v = *reinterpret_cast<const f32x4_t *>(weights[a] + 4 * j);
                    *reinterpret_cast<f32x4_t *>(cols + at[a] + (j & 1) * (g.d / 2) + 4 * (j >> 1)) = v;
                    if (CH > 1 && (a == YW || a == YB))
                        for (int q = 0; q < 4; ++q) odd = odd || !(fabsf(v[q]) <= 0x1p119f);
                }
        if constexpr (CH > 1) odd_weights = __syncthreads_or(odd);
        else __syncthreads();
    }
    for (long k = 0; k < rounds; ++k, row += step) {
        const bool on = row < g.T;
        const long t = on ? row : g.T - 1;
        const float ym = st[0], ys = st[1], rm = st[2], rs = st[3];
        // ---- D = dr + N_r^T dh
        f32x8 D[CH];
        if (g.dh && g.r_norm) {
            f32x8 u[CH];
            float s[LAYER ? 2 : 1] = {};
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                f32x8 gw = hr[c].get();
                u[c] = LAYER ? (rr[c].get() - rm) * rs : rr[c].get() * rs;
                if (SUMS & 1 && sums & 1) sum[0][c] = sum[0][c] + gw * u[c];
                if (SUMS & 2 && sums & 2) sum[1][c] = sum[1][c] + gw;
                if (g.r_weight) gw = gw * weight(RW, c);
                s[0] = s[0] + dot8(gw, u[c]);
                if constexpr (LAYER) s[1] = s[1] + sum8(gw);
                D[c] = gw;
            }
            load_r(row + step);
            row_sums<G>(s, red[2 * (k & 1)]);
            const float a = s[0] * inv_d;
            float b = 0.f;
            if constexpr (LAYER) b = g.r_norm == JOIN_LAYER ? s[1] * inv_d : 0.f;
            if constexpr (SUMS == 0) {
                if (g.means && on && lane == 0) {
                    g.means[2 * t] = a;
                    g.means[2 * t + 1] = b;
                }
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                D[c] = D[c] - u[c] * a;
                if constexpr (LAYER) D[c] = D[c] - b;
                D[c] = dr[c].get() + rs * D[c];
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) D[c] = dr[c].get() + hr[c].get();
            load_r(row + step);
        }
        load_dr(row + step);
        if constexpr (SUMS == 0) {
            if (!g.dx) {                     // the means alone
                load_y(row + step);
                continue;
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (!ok[c]) D[c] = zero8();
            else if (on) put<F32>((char *)g.dx + (size_t)(t * g.d) * SZ, col[c], D[c]);
        }
        if (!g.y) {
            load_y(row + step);
            continue;
        }
        // ---- through the gates, the dropout and y's norm
        f32x8 y[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) y[c] = yr[c].get();
        load_y(row + step);
        const float tg = g.token_gate ? g.token_gate[t] : 1.f;
        // the token's gate comes last where its own gradient is wanted
        const float f = g.dtoken_gate ? g.scale * g.keep : g.scale * g.keep * tg;
        // What dropout has taken out is 0 for the gates too, also where it is infinite or NaN.
        // Longer rows have no registers for the words that long (16384 x 7168: 339 us, 311 this way)
        // and make them again if a row needs it: one with such values has no finite deviation, or large weights.
        constexpr bool WORDS = CH == 1;
        bool odd = false;
        if constexpr (!WORDS) odd = g.rng && __ballot(!g.y_norm || odd_weights || !(ys > 0.f && ys <= FLT_MAX));
        float s[LAYER ? 3 : 2] = {};                     // the last one: of the token's gate
        constexpr int TG = LAYER ? 2 : 1;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (g.y_norm) y[c] = LAYER ? (y[c] - ym) * ys : y[c] * ys;
            f32x8 n = y[c], w, e = D[c] * f;             // e: of the kept elements, without gates
            Words bits;
            if (g.rng) {
                bits = philox(seed, offset, (uint32_t)col[c] / 8, (uint32_t)t);
                e = drop8(e, bits, g.out);
            }
            if (g.y_weight) {
                w = weight(YW, c);
                n = n * w;
            }
            if (g.y_bias) n = n + weight(YB, c);
            if constexpr (WORDS) {
                if (g.rng) n = drop8(n, bits, g.out);
            } else if (odd) {
                uint32_t j = (uint32_t)col[c] / 8;
                asm volatile("" : "+v"(j));
                n = drop8(n, philox(seed, offset, j, (uint32_t)t), g.out);
            }
            if (g.dtoken_gate) {
                f32x8 ge = e;
                if (g.gate) ge = ge * weight(GATE, c);
                s[TG] = s[TG] + dot8(n, ge);
                e = e * tg;
            }
            if (SUMS & 4 && sums & 4) sum[2][c] = sum[2][c] + n * e;
            if (g.gate) e = e * weight(GATE, c);
            if (SUMS & 8 && sums & 8) sum[3][c] = sum[3][c] + e * y[c];
            if (SUMS & 16 && sums & 16) sum[4][c] = sum[4][c] + e;
            if (g.y_weight) e = e * w;
            s[0] = s[0] + dot8(e, y[c]);
            if constexpr (LAYER) s[1] = s[1] + sum8(e);
            D[c] = e;
        }
        if (g.y_norm || g.dtoken_gate) row_sums<G>(s, red[2 * (k & 1) + 1]);
        if (g.dtoken_gate && on && lane == 0) g.dtoken_gate[t] = s[TG];
        const float a = s[0] * inv_d;
        float b = 0.f;
        if constexpr (LAYER) b = g.y_norm == JOIN_LAYER ? s[1] * inv_d : 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (g.y_norm) {
                D[c] = D[c] - y[c] * a;
                if constexpr (LAYER) D[c] = D[c] - b;
                D[c] = ys * D[c];
            }
            if (on && ok[c]) st_u32x4(g.dy + t * g.d + col[c], pack_bf8(D[c]));
        }
    }
    // ---- the workgroup's sums over its rows: the rows of a wave, then the others' in
    // order, to `part`, or where they belong if it is the only one
    constexpr int STEP = G < 64 ? 64 : G, TURNS = NT / STEP;
    int n = 0;
#pragma unroll
    for (int a = 0; a < 5; ++a) {
        if (!(SUMS >> a & 1) || !(sums >> a & 1)) continue;
        float *to = gridDim.x == 1 ? g.out_sums[n] : g.part + ((long)blockIdx.x * g.nsums + n) * g.d;
#pragma unroll
        for (int m = G; m < 64; m <<= 1)
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[a][c][i] = sum[a][c][i] + shfl_xor_f(sum[a][c][i], m);
        for (int q = 0; q < TURNS; ++q) {
            if (TURNS > 1) __syncthreads();  // and the last row's weights have been read
            if ((int)threadIdx.x / STEP == q && (int)threadIdx.x % STEP < G)
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    if (ok[c]) {
                        f32x8 v = sum[a][c];
                        if (q > 0) v = ld_f32x8(cols + col[c]) + v;
                        if (q < TURNS - 1) st_f32x8(cols + col[c], v);
                        else st_f32x8(to + col[c], v);
                    }
        }
        ++n;
    }
}

// Rows longer than 8192, whose sums the registers above cannot hold: the sums alone,
// with the rows' means that the kernel above has left.  A wave takes 512 columns of every
// fourth row of its workgroup's share.  4096 rows of 12288, three sums and dropout: 350 to 388 us in
// all by the box, 629 in one kernel whose sums went to memory; 604 MB and, for the sums, 403
// of them again.  Five sums 384 to 413; without dropout 283 and 307.  The row kernel spills 50 registers, 158 in fp32.
template <bool F32>
__global__ __launch_bounds__(256) void join_columns_kernel(JoinArgs g) {
    __shared__ __attribute__((aligned(16))) float red[3][512];
    constexpr int SZ = F32 ? 4 : 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int col = 512 * blockIdx.y + 8 * lane;
    const bool ok = col < g.d;
    if (!ok) col = 0;
    const long rows = (g.T + gridDim.x - 1) / gridDim.x, t0 = rows * blockIdx.x;
    const long t1 = t0 + rows < g.T ? t0 + rows : g.T;
    f32x8 sum[5], rw = zero8() + 1.f, yw = rw, gt = rw, yb = zero8();
#pragma unroll
    for (int a = 0; a < 5; ++a) sum[a] = zero8();
    if (g.r_weight) rw = ld_f32x8(g.r_weight + col);
    if (g.y_weight) yw = ld_f32x8(g.y_weight + col);
    if (g.y_bias) yb = ld_f32x8(g.y_bias + col);
    if (g.gate) gt = ld_f32x8(g.gate + col);
    uint64_t seed = 0, offset = 0;
    if (g.rng) {
        seed = (uint64_t)g.rng[0];
        offset = (uint64_t)g.rng[1];
    }
#pragma unroll 2
    for (long t = t0 + wave; t < t1; t += 4) {
        const size_t i = (size_t)(t * g.d);
        const f32x4_t st = *reinterpret_cast<const f32x4_t *>(g.stats_in + 4 * t);
        Raw<F32> rr, dr;
        Raw<false> hr, yr;
        rr.clear();
        dr.clear();
        hr.clear();
        if (g.dh && g.r_norm) rr.load((const char *)g.r_in + i * SZ, col);
        if (g.dh) hr.load(g.dh + i, col);
        if (g.dr) dr.load((const char *)g.dr + i * SZ, col);
        if (g.y) yr.load(g.y + i, col);
        f32x8 D = hr.get();
        if (g.dh && g.r_norm) {
            const f32x8 u = (rr.get() - st[2]) * st[3];
            sum[0] = sum[0] + D * u;
            sum[1] = sum[1] + D;
            D = st[3] * (D * rw - u * g.means[2 * t] - g.means[2 * t + 1]);
        }
        if (!g.y) continue;
        D = D + dr.get();
        f32x8 y = yr.get();
        if (g.y_norm) y = (y - st[0]) * st[1];
        f32x8 e = D * (g.scale * g.keep * (g.token_gate ? g.token_gate[t] : 1.f));
        f32x8 n = y * yw + yb;
        if (g.rng) {
            const Words bits = philox(seed, offset, (uint32_t)col / 8, (uint32_t)t);
            e = drop8(e, bits, g.out);
            n = drop8(n, bits, g.out);
        }
        sum[2] = sum[2] + n * e;
        e = e * gt;
        sum[3] = sum[3] + e * y;
        sum[4] = sum[4] + e;
    }
    int n = 0;
#pragma unroll
    for (int a = 0; a < 5; ++a) {
        if (!(g.sums >> a & 1)) continue;
        __syncthreads();
        if (wave) st_f32x8(red[wave - 1] + 8 * lane, sum[a]);
        __syncthreads();
        if (!wave) {
#pragma unroll
            for (int w = 0; w < 3; ++w) sum[a] = sum[a] + ld_f32x8(red[w] + 8 * lane);
            if (ok) st_f32x8(g.part + ((long)blockIdx.x * g.nsums + n) * g.d + col, sum[a]);
        }
        ++n;
    }
}

// The workgroups' sums added up, in their order within 32 strided lists whose sums are
// then added in order: array n, columns 4 at a time, 8 of those to a workgroup (768
// workgroups, 3 x 2048 columns: 5.6 us, with 16 lists of 64 columns 6.4).
constexpr int JS_LISTS = 32, JS_QUADS = 8, JS_LOADS = 8;     // loads under way in a list
__global__ __launch_bounds__(256) void join_sum_kernel(JoinArgs g, int blocks) {
    __shared__ __attribute__((aligned(16))) float red[JS_LISTS][JS_QUADS][4];
    const int quad = threadIdx.x % JS_QUADS, list = threadIdx.x / JS_QUADS, n = blockIdx.y;
    const int c = 4 * (blockIdx.x * JS_QUADS + quad);
    f32x4_t v = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (c < g.d)
        for (int b = list; b < blocks; b += JS_LISTS * JS_LOADS) {
            f32x4_t u[JS_LOADS];
#pragma unroll
            for (int j = 0; j < JS_LOADS; ++j)
                u[j] = *reinterpret_cast<const f32x4_t *>(
                    g.part + ((long)min(b + JS_LISTS * j, blocks - 1) * g.nsums + n) * g.d + c);
#pragma unroll
            for (int j = 0; j < JS_LOADS; ++j)
                if (b + JS_LISTS * j < blocks)
#pragma unroll
                    for (int q = 0; q < 4; ++q) v[q] = v[q] + u[j][q];
        }
    *reinterpret_cast<f32x4_t *>(red[list][quad]) = v;
    __syncthreads();
    if (list == 0 && c < g.d) {
#pragma unroll
        for (int l = 1; l < JS_LISTS; ++l)
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = v[q] + red[l][quad][q];
        *reinterpret_cast<f32x4_t *>(g.out_sums[n] + c) = v;
    }
}

template <bool F32>
hipError_t forward(JoinArgs g, hipStream_t st) {
    // a launch takes fewer than 2^32 threads
#define JOIN_FWD(G, CH)                                                                              \
    do {                                                                                             \
        constexpr int NT = G < 256 ? 256 : G;                                                        \
        const long per = NT / G, most = 1l << 21;                                                    \
        for (g.row0 = 0; g.row0 < g.T; g.row0 += most * per) {                                       \
            const long n = (g.T - g.row0 + per - 1) / per;                                           \
            join_forward_kernel<F32, false, NT, G, CH>                                               \
                <<<dim3((unsigned)(n < most ? n : most)), dim3(NT), 0, st>>>(g);                     \
        }                                                                                            \
        return hipGetLastError();                                                                    \
    } while (0)
#define JOIN_ROWS(G, CH)                                                                             \
    do {                                                                                             \
        join_forward_kernel<F32, true, 1024, G, CH><<<dim3(256), dim3(1024), lds, st>>>(g);          \
        return hipGetLastError();                                                                    \
    } while (0)
    const int n_w = !!g.r_weight + !!g.r_bias + !!g.y_weight + !!g.y_bias + !!g.gate;
    const size_t lds = (size_t)n_w * g.d * 4;
    if (join_forward_rows(g.T, g.d, n_w, g.y != nullptr)) {
        if (g.d <= 1024) JOIN_ROWS(128, 1);
        if (g.d <= 2048) JOIN_ROWS(256, 1);
        if (g.d <= 4096) JOIN_ROWS(512, 1);
        JOIN_ROWS(512, 2);
    }
    if (g.d <= 64) JOIN_FWD(8, 1);
    if (g.d <= 128) JOIN_FWD(16, 1);
    if (g.d <= 256) JOIN_FWD(32, 1);
    if (g.T <= JOIN_FEW_ROWS) {
        if (g.d <= 512) JOIN_FWD(64, 1);
        if (g.d <= 1024) JOIN_FWD(128, 1);
        if (g.d <= 2048) JOIN_FWD(256, 1);
        if (g.d <= 4096) JOIN_FWD(512, 1);
        if (g.d <= 8192) JOIN_FWD(1024, 1);
        JOIN_FWD(1024, 2);
    }
    if (g.d <= 512) JOIN_FWD(64, 1);
    if (g.d <= 1024) JOIN_FWD(64, 2);
    if (g.d <= 2048) JOIN_FWD(128, 2);
    if (g.d <= 4096) JOIN_FWD(256, 2);
    if (g.d <= 8192) JOIN_FWD(256, 4);
    JOIN_FWD(512, 4);
#undef JOIN_FWD
#undef JOIN_ROWS
}

template <bool F32, int SUMS, bool LAYER>
hipError_t backward(const JoinArgs &g, int blocks, hipStream_t st) {
#define JOIN_BWD(NT, G, CH)                                                                          \
    do {                                                                                             \
        const size_t lds = (size_t)(CH <= 2 ? std::max(n_w, 1) : 1) * g.d * 4;                       \
        join_backward_kernel<F32, SUMS, LAYER, NT, G, CH>                                            \
            <<<dim3((unsigned)blocks), dim3(NT), lds, st>>>(g);                                      \
        return hipGetLastError();                                                                    \
    } while (0)
#define JOIN_ONCE(NT, G)                                                                             \
    do {                                                                                             \
        join_backward_kernel<F32, SUMS, LAYER, NT, G, 1, true>                                       \
            <<<dim3((unsigned)blocks), dim3(NT), (size_t)g.d * 4, st>>>(g);                          \
        return hipGetLastError();                                                                    \
    } while (0)
    const int n_w = !!g.r_weight + !!g.y_weight + !!g.y_bias + !!g.gate;
    if (g.T <= blocks * join_rows(g.d)) {
        if (g.d <= 64) JOIN_ONCE(256, 8);
        if (g.d <= 128) JOIN_ONCE(256, 16);
        if (g.d <= 256) JOIN_ONCE(256, 32);
        if (g.d <= 512) JOIN_ONCE(256, 64);
        if (g.d <= 1024) JOIN_ONCE(256, 128);
        if (g.d <= 2048) JOIN_ONCE(256, 256);
        if (g.d <= 4096) JOIN_ONCE(512, 512);
        JOIN_ONCE(1024, 1024);
    }
    if (g.d <= 64) JOIN_BWD(256, 8, 1);
    if (g.d <= 128) JOIN_BWD(256, 16, 1);
    if (g.d <= 256) JOIN_BWD(256, 32, 1);
    if (g.d <= 512) JOIN_BWD(256, 64, 1);
    if (g.d <= 1024) JOIN_BWD(256, 128, 1);
    if (g.d <= 2048) JOIN_BWD(256, 256, 1);
    if (g.d <= 4096) JOIN_BWD(512, 512, 1);
    JOIN_BWD(512, 512, 2);
#undef JOIN_BWD
#undef JOIN_ONCE
}
template <bool F32>
hipError_t backward(JoinArgs g, int blocks, hipStream_t st) {
    if (g.d > JOIN_SUMS_D) {
        auto rows = [&](const JoinArgs &q) {
            join_backward_kernel<F32, 0, true, 512, 512, 4><<<dim3((unsigned)blocks), dim3(512), 0, st>>>(q);
        };
        auto columns = [&] {
            join_columns_kernel<F32><<<dim3((unsigned)blocks, (unsigned)((g.d + 511) / 512)), dim3(256), 0, st>>>(g);
        };
        if (!g.nsums) g.means = nullptr;
        const bool first = g.nsums && g.dx == g.dr;  // before the rows write over what the sums read
        if (first) {
            JoinArgs means = g;
            means.dx = nullptr;
            rows(means);
            columns();
        }
        rows(g);
        if (g.nsums && !first) columns();
        return hipGetLastError();
    }
    const bool layer = g.r_norm == JOIN_LAYER || g.y_norm == JOIN_LAYER;
    if (!layer && !(g.sums & ~13)) return backward<F32, 13, false>(g, blocks, st);
    if (!(g.sums & ~7)) return backward<F32, 7, true>(g, blocks, st);
    return backward<F32, 31, true>(g, blocks, st);
}

}  // namespace

int join_blocks(long T, int d) { return (int)join_workgroups(T, d); }

hipError_t launch_join_forward(const JoinArgs &g, hipStream_t st) {
    if (g.T <= 0) return hipSuccess;
    return g.f32 ? forward<true>(g, st) : forward<false>(g, st);
}

hipError_t launch_join_backward(JoinArgs g, hipStream_t st) {
    const int blocks = g.T > 0 ? join_blocks(g.T, g.d) : 0;
    if (blocks) {
        const hipError_t e = g.f32 ? backward<true>(g, blocks, st) : backward<false>(g, blocks, st);
        if (e != hipSuccess) return e;
    }
    if (!g.nsums || (blocks == 1 && g.d <= JOIN_SUMS_D)) return hipSuccess;
    join_sum_kernel<<<dim3((unsigned)((g.d + 4 * JS_QUADS - 1) / (4 * JS_QUADS)), (unsigned)g.nsums), dim3(256), 0, st>>>(
        g, blocks);
    return hipGetLastError();
}
