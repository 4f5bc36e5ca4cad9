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
DEV bool kept(const Words &w, int i, uint32_t out) {
    return (i & 1 ? w.w[i >> 1] >> 16 : w.w[i >> 1] & 0xffffu) >= out;
}

// ---------------------------------------------------------------- rows
// 8 consecutive values as they lie in memory
template <bool F32> struct Raw;
template <> struct Raw<false> {
    u32x4_t a;
    DEV void load(const void *p, long i) { a = ld_u32x4((const uint16_t *)p + i); }
    DEV void clear() { a = u32x4_t{0u, 0u, 0u, 0u}; }
    DEV f32x8 get() const {
        return f32x8{bf_lo(a[0]), bf_hi(a[0]), bf_lo(a[1]), bf_hi(a[1]),
                     bf_lo(a[2]), bf_hi(a[2]), bf_lo(a[3]), bf_hi(a[3])};
    }
};
template <> struct Raw<true> {
    u32x4_t a, b;
    DEV void load(const void *p, long i) {
        a = ld_u32x4((const float *)p + i);
        b = ld_u32x4((const float *)p + i + 4);
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
// stores v and returns what a reader of the stream finds there
template <bool F32>
DEV f32x8 put(void *p, long i, const f32x8 &v) {
    if constexpr (F32) {
        st_f32x8((float *)p + i, v);
        return v;
    } else {
        Raw<false> r;
        r.a = pack_bf8(v);
        st_u32x4((uint16_t *)p + i, r.a);
        return r.get();
    }
}

// ---------------------------------------------------------------- sums over a row
DEV float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m; m >>= 1) v = v + shfl_xor_f(v, m);
    return v;
}
// N sums over the G threads of a row, the same in each of them.  Rows of more
// than a wave meet in `red` (a slot per wave, N used of 4), which must not be
// written again before every thread has passed another barrier: callers
// alternate between slots.
template <int G, int NT, int N>
DEV void row_sums(float (&v)[N], float (*red)[4]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (G > 64) {
        const int wave = threadIdx.x >> 6, w0 = wave / (G / 64) * (G / 64);
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[wave][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = red[w0][i];
#pragma unroll
            for (int w = 1; w < G / 64; ++w) s = s + red[w0 + w][i];
            v[i] = s;
        }
    }
}

DEV float dev_inv(float var, float eps) { return 1.0f / sqrtf(var + eps); }

// ---------------------------------------------------------------- forward
template <bool F32, int G, int CH>
__global__ __launch_bounds__(G < 256 ? 256 : G) void join_forward_kernel(JoinArgs g) {
    constexpr int NT = G < 256 ? 256 : G, NW = NT / 64;
    __shared__ float red[4][NW][4];
    const int lane = threadIdx.x % G;
    const long row = g.row0 + (long)blockIdx.x * (NT / G) + threadIdx.x / G;
    if (G <= 64 && row >= g.T) return;       // a wave to a row: no barriers
    const bool on = row < g.T;
    const long t = on ? row : g.T - 1;
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
        xr[c].load(g.x, t * g.d + col[c]);
        if (g.y) yr[c].load(g.y, t * g.d + col[c]);
    }
    f32x8 r[CH];
    float ym = 0.f, ys = 0.f, rm = 0.f, rs = 0.f;
    // mean and deviation of the rows in v, two sums one after the other
    auto stats = [&](const f32x8 (&v)[CH], int kind, float eps, float &m, float &s, int at) {
        float sum[1] = {0.f};
        m = 0.f;
        if (kind == JOIN_LAYER) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] = sum[0] + (ok[c] ? v[c][i] : 0.f);
            row_sums<G, NT>(sum, red[at]);
            m = sum[0] * inv_d;
        }
        sum[0] = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = v[c][i] - m;
                sum[0] = sum[0] + (ok[c] ? u * u : 0.f);
            }
        row_sums<G, NT>(sum, red[at + 1]);
        s = dev_inv(sum[0] * inv_d, eps);
    };
    auto normed = [&](const f32x8 &v, float m, float s, const float *w, const float *b, int at) {
        f32x8 n;
        f32x8 wv, bv;
        if (w) wv = ld_f32x8(w + at);
        if (b) bv = ld_f32x8(b + at);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            n[i] = (v[i] - m) * s;
            if (w) n[i] = n[i] * wv[i];
            if (b) n[i] = n[i] + bv[i];
        }
        return n;
    };
    if (g.y) {
        f32x8 v[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = yr[c].get();
        if (g.y_norm) {
            stats(v, g.y_norm, g.y_eps, ym, ys, 0);
#pragma unroll
            for (int c = 0; c < CH; ++c) v[c] = normed(v[c], ym, ys, g.y_weight, g.y_bias, col[c]);
        }
        uint64_t seed = 0, offset = 0;
        if (g.rng) {
            seed = (uint64_t)g.rng[0];
            offset = (uint64_t)g.rng[1];
        }
        const float tg = g.token_gate ? g.token_gate[t] : 1.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            f32x8 a;
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = g.scale;
            if (g.gate) {
                const f32x8 w = ld_f32x8(g.gate + col[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) a[i] = a[i] * w[i];
            }
            if (g.rng) {
                const Words w = philox(seed, offset, (uint32_t)col[c] / 8, (uint32_t)t);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = kept(w, i, g.out) ? v[c][i] * g.keep : 0.f;
            }
            const f32x8 x = xr[c].get();
#pragma unroll
            for (int i = 0; i < 8; ++i) r[c][i] = x[i] + a[i] * tg * v[c][i];
            if constexpr (!F32) {
                Raw<false> q;
                q.a = pack_bf8(r[c]);
                r[c] = q.get();
            }
            if (on && ok[c]) put<F32>(g.r, t * g.d + col[c], r[c]);
        }
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c) r[c] = xr[c].get();
    }
    if (g.r_norm) stats(r, g.r_norm, g.r_eps, rm, rs, 2);
    if (g.h)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const f32x8 n = g.r_norm ? normed(r[c], rm, rs, g.r_weight, g.r_bias, col[c]) : r[c];
            if (on && ok[c]) st_u32x4(g.h + t * g.d + col[c], pack_bf8(n));
        }
    if (g.stats && on && lane == 0)
        *reinterpret_cast<f32x4_t *>(g.stats + 4 * t) = f32x4_t{ym, ys, rm, rs};
}

// ---------------------------------------------------------------- backward
// A workgroup takes rows in steps of the whole grid and keeps its sums over them
// in registers; each row is loaded one step ahead.
template <bool F32, int G, int CH>
__global__ __launch_bounds__(512) void join_backward_kernel(JoinArgs g) {
    constexpr int NT = 512, NG = NT / G;
    __shared__ float red[4][NT / 64][4];
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    const float inv_d = 1.0f / (float)g.d;
    bool ok[CH];
    int col[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        col[c] = 8 * (lane + G * c);
        ok[c] = col[c] < g.d;
        if (!ok[c]) col[c] = 0;
    }
    f32x8 sum[5][CH];        // weight and bias of r's norm, gate, weight and bias of y's
#pragma unroll
    for (int a = 0; a < 5; ++a)
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[a][c][i] = 0.f;
    uint64_t seed = 0, offset = 0;
    if (g.rng) {
        seed = (uint64_t)g.rng[0];
        offset = (uint64_t)g.rng[1];
    }
    Raw<F32> rr[CH], dr[CH];
    Raw<false> yr[CH], hr[CH];
    f32x4_t st4;
    const long step = (long)gridDim.x * NG;
    long row = (long)blockIdx.x * NG + group;
    const long rounds = (g.T + step - 1) / step;
    auto load = [&](long at) {
        const long t = at < g.T ? at : g.T - 1;
        st4 = *reinterpret_cast<const f32x4_t *>(g.stats_in + 4 * t);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const long i = t * g.d + col[c];
            if (g.dh) hr[c].load(g.dh, i);
            if (g.dh && g.r_norm) rr[c].load(g.r_in, i);
            if (g.dr) dr[c].load(g.dr, i);
            if (g.y) yr[c].load(g.y, i);
        }
    };
    load(row);
    for (long k = 0; k < rounds; ++k, row += step) {
        const bool on = row < g.T;
        const long t = on ? row : g.T - 1;
        const float ym = st4[0], ys = st4[1], rm = st4[2], rs = st4[3];
        f32x8 D[CH], y[CH];
        // ---- D = dr + N_r^T dh
        {
            f32x8 u[CH];
            float s[2] = {0.f, 0.f};
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const bool in = on && ok[c];
                if (g.y) y[c] = yr[c].get();
                if (g.dr) D[c] = dr[c].get();
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) D[c][i] = 0.f;
                if (!g.dh) continue;
                f32x8 dh = hr[c].get();
                if (g.r_norm) u[c] = rr[c].get();
                f32x8 w;
                if (g.r_weight) w = ld_f32x8(g.r_weight + col[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (!g.r_norm) {
                        D[c][i] = D[c][i] + dh[i];
                        continue;
                    }
                    u[c][i] = (u[c][i] - rm) * rs;
                    sum[0][c][i] = sum[0][c][i] + (in ? dh[i] * u[c][i] : 0.f);
                    sum[1][c][i] = sum[1][c][i] + (in ? dh[i] : 0.f);
                    const float gw = g.r_weight ? dh[i] * w[i] : dh[i];
                    s[0] = s[0] + (in ? gw * u[c][i] : 0.f);
                    s[1] = s[1] + (in ? gw : 0.f);
                }
            }
            if (g.dh && g.r_norm) {
                row_sums<G, NT>(s, red[2 * (k & 1)]);
                const float a = s[0] * inv_d, b = g.r_norm == JOIN_LAYER ? s[1] * inv_d : 0.f;
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const f32x8 dh = hr[c].get();
                    f32x8 w;
                    if (g.r_weight) w = ld_f32x8(g.r_weight + col[c]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float gw = g.r_weight ? dh[i] * w[i] : dh[i];
                        D[c][i] = D[c][i] + rs * (gw - u[c][i] * a - b);
                    }
                }
            }
        }
        load(row + step);
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (on && ok[c]) put<F32>(g.dx, t * g.d + col[c], D[c]);
        if (!g.y) continue;
        // ---- through the gates, the dropout and y's norm
        const float tg = g.token_gate ? g.token_gate[t] : 1.f;
        float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const bool in = on && ok[c];
            f32x8 gt, w, b;
            if (g.gate) gt = ld_f32x8(g.gate + col[c]);
            if (g.y_weight) w = ld_f32x8(g.y_weight + col[c]);
            if (g.y_bias) b = ld_f32x8(g.y_bias + col[c]);
            Words bits{};
            if (g.rng) bits = philox(seed, offset, (uint32_t)col[c] / 8, (uint32_t)t);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = g.y_norm ? (y[c][i] - ym) * ys : y[c][i];
                float n = u;
                if (g.y_weight) n = n * w[i];
                if (g.y_bias) n = n + b[i];
                const bool keep = !g.rng || kept(bits, i, g.out);
                const float mul = keep ? g.keep : 0.f;
                const float v = keep ? n * g.keep : 0.f;
                const float vd = g.scale * v * D[c][i];
                sum[2][c][i] = sum[2][c][i] + (in ? vd * tg : 0.f);
                s[2] = s[2] + (in ? (g.gate ? vd * gt[i] : vd) : 0.f);
                float a = g.scale;
                if (g.gate) a = a * gt[i];
                const float dn = keep ? a * tg * D[c][i] * mul : 0.f;
                sum[3][c][i] = sum[3][c][i] + (in ? dn * u : 0.f);
                sum[4][c][i] = sum[4][c][i] + (in ? dn : 0.f);
                const float gw = g.y_weight ? dn * w[i] : dn;
                s[0] = s[0] + (in ? gw * u : 0.f);
                s[1] = s[1] + (in ? gw : 0.f);
                D[c][i] = gw;
                y[c][i] = u;
            }
        }
        if (g.y_norm || g.token_gate) row_sums<G, NT>(s, red[2 * (k & 1) + 1]);
        if (g.dtoken_gate && on && lane == 0) g.dtoken_gate[t] = s[2];
        const float a = s[0] * inv_d, b = g.y_norm == JOIN_LAYER ? s[1] * inv_d : 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            f32x8 dy = D[c];
            if (g.y_norm)
#pragma unroll
                for (int i = 0; i < 8; ++i) dy[i] = ys * (dy[i] - y[c][i] * a - b);
            if (on && ok[c]) st_u32x4(g.dy + t * g.d + col[c], pack_bf8(dy));
        }
    }
    // ---- the workgroup's sums over its rows: groups in order, then to `part`
    extern __shared__ __attribute__((aligned(16))) float cols[];     // [d]
    int n = 0;
#pragma unroll
    for (int a = 0; a < 5; ++a) {
        if (!(g.sums >> a & 1)) continue;
        for (int q = 0; q < NG; ++q) {
            if (NG > 1) __syncthreads();
            if (group == q)
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    if (ok[c]) {
                        f32x8 v = sum[a][c];
                        if (q > 0) {
                            const f32x8 u = ld_f32x8(cols + col[c]);
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = u[i] + v[i];
                        }
                        if (q < NG - 1) st_f32x8(cols + col[c], v);
                        else st_f32x8(g.part + ((long)blockIdx.x * g.nsums + n) * g.d + col[c], v);
                    }
        }
        ++n;
    }
}

// The workgroups' sums added up, in their order within 16 strided lists whose
// sums are then added in order: out of array n, columns 4 at a time.
constexpr int JS_LISTS = 16;
__global__ __launch_bounds__(256) void join_sum_kernel(JoinArgs g, int blocks) {
    __shared__ __attribute__((aligned(16))) float red[JS_LISTS][16][4];
    const int c = 4 * (blockIdx.x * 16 + (threadIdx.x & 15)), list = threadIdx.x >> 4, n = blockIdx.y;
    f32x4_t v = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (c < g.d)
#pragma unroll 4
        for (int b = list; b < blocks; b += JS_LISTS) {
            const f32x4_t u = *reinterpret_cast<const f32x4_t *>(g.part + ((long)b * g.nsums + n) * g.d + c);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = v[q] + u[q];
        }
    *reinterpret_cast<f32x4_t *>(red[list][threadIdx.x & 15]) = v;
    __syncthreads();
    if (threadIdx.x < 16 && c < g.d) {
        for (int l = 1; l < JS_LISTS; ++l)
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = v[q] + red[l][threadIdx.x][q];
        *reinterpret_cast<f32x4_t *>(g.out_sums[n] + c) = v;
    }
}

template <bool F32>
hipError_t forward(JoinArgs g, hipStream_t st) {
    // a launch takes fewer than 2^32 threads
#define JOIN_FWD(G, CH)                                                                              \
    do {                                                                                             \
        const long per = G < 256 ? 256 / G : 1, most = 1l << 21;                                     \
        for (g.row0 = 0; g.row0 < g.T; g.row0 += most * per) {                                       \
            const long n = (g.T - g.row0 + per - 1) / per;                                           \
            join_forward_kernel<F32, G, CH>                                                          \
                <<<dim3((unsigned)(n < most ? n : most)), dim3(G < 256 ? 256 : G), 0, st>>>(g);      \
        }                                                                                            \
        return hipGetLastError();                                                                    \
    } while (0)
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
}

template <bool F32>
hipError_t backward(const JoinArgs &g, int blocks, hipStream_t st) {
#define JOIN_BWD(G, CH)                                                                              \
    do {                                                                                             \
        const size_t lds = G < 512 && g.nsums ? (size_t)g.d * 4 : 0;                                 \
        join_backward_kernel<F32, G, CH><<<dim3((unsigned)blocks), dim3(512), lds, st>>>(g);         \
        return hipGetLastError();                                                                    \
    } while (0)
    if (g.d <= 512) JOIN_BWD(64, 1);
    if (g.d <= 1024) JOIN_BWD(64, 2);
    if (g.d <= 2048) JOIN_BWD(128, 2);
    if (g.d <= 4096) JOIN_BWD(256, 2);
    if (g.d <= 8192) JOIN_BWD(512, 2);
    JOIN_BWD(512, 4);
#undef JOIN_BWD
}

}  // namespace

int join_blocks(long T, int d) {
    const long rows = d <= 1024 ? 8 : d <= 2048 ? 4 : d <= 4096 ? 2 : 1;    // of a workgroup at a time
    const long n = (T + rows - 1) / rows;
    return (int)(n < JOIN_BLOCKS ? n : JOIN_BLOCKS);
}

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
    if (!g.nsums) return hipSuccess;
    join_sum_kernel<<<dim3((unsigned)((g.d + 63) / 64), (unsigned)g.nsums), dim3(256), 0, st>>>(g, blocks);
    return hipGetLastError();
}
