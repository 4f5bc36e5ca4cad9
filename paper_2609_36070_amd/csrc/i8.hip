// Quantisation to 8-bit integers (rule in i8_common.h):
//
//   i8_quant_rows:    one scale per row of a K-contiguous matrix: tokens of X
//                     (bf16), rows of the gated activation (fp32).
//   i8_quant_weights: [E][K][N] bf16 weights -> K-contiguous [E][N][K] codes
//                     and one scale per channel [E][N], the operand layout of
//                     the int8 products.
#include "common.h"
#include "i8_common.h"
#include "kernels.h"

namespace {

template <int N> struct Const { static constexpr int value = N; };

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

// Largest of a value over a wave, or over the 4 waves of a block.
template <int W>
DEV uint32_t row_max(uint32_t x, uint32_t *red) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x = umax(x, (uint32_t)__shfl_xor((int)x, m, 64));
    if constexpr (W == 1) return x;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    return umax(umax(red[0], red[1]), umax(red[2], red[3]));
}

// Rows of a matrix to quantise.
template <typename S>
struct QuantRows {
    const S *X;
    uint8_t *q;
    float *sc;
    long rows;
    int K;
};

// Where the scale of a row goes that the quantiser of H wrote for the tile
// products: into the weight of its route, whose numbers are asked for ahead of and
// behind the row's values.
struct RouteFactor {
    const I8Factors &f;
    long row;
    int j = -1, planned = 0;
    int e = 0;
    float w = 0.f;
    DEV void ask() {                         // one thread of the row
        j = f.perm[row];                     // (past the plan: whatever is there)
        planned = f.offsets[f.E];
    }
    DEV void ask_weight(long rows) {
        if (row >= planned || j < 0 || j >= rows) j = -1;
        if (j < 0) return;
        w = f.topk_w[j];
        e = f.topk_idx[j];
    }
    DEV void put(float s) const {
        if (j >= 0) f.w[j] = w * (s * f.unit[2 * min(max(e, 0), f.E - 1) + 1]);
    }
};
struct RowScale {                            // the scale as it is, times a factor
    float *at;
    const float *unit;
    DEV void ask() {}
    DEV void ask_weight(long) {}
    DEV void put(float s) const { *at = unit ? s * *unit : s; }
};

// Row `row` by W waves, 8 elements per thread and step.  Rows of up to 512 W NC
// elements are held in registers between the two passes (NC = 0: read again).
template <typename S, int NC, int W, typename P>
DEV void quant_row(const QuantRows<S> &m, long row, uint32_t *red, P out) {
    constexpr int TH = 64 * W;
    const S *x = m.X + row * m.K;
    uint8_t *o = m.q + row * m.K;
    const int n8 = m.K / 8, tid = threadIdx.x % TH;
    float v[NC > 0 ? NC : 1][8];
    uint32_t amax = 0;
    if (tid == 0) out.ask();
    auto put = [&](const float (&y)[8], const I8Scale &s, int c) {
        *reinterpret_cast<u32x2_t *>(o + 8 * c) =
            u32x2_t{pack_i8(s.code(y[0]), s.code(y[1]), s.code(y[2]), s.code(y[3])),
                    pack_i8(s.code(y[4]), s.code(y[5]), s.code(y[6]), s.code(y[7]))};
    };
    if constexpr (NC > 0) {
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = tid + TH * i;
            if (c < n8) load8(x + 8 * c, v[i]);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        }
        if (tid == 0) out.ask_weight(m.rows);
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) amax = umax(amax, abs_bits(v[i][j]));
        const I8Scale s(row_max<W>(amax, red));
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = tid + TH * i;
            if (c < n8) put(v[i], s, c);
        }
        if (tid == 0) out.put(s.s);
    } else {
        for (int c = tid; c < n8; c += TH) {
            load8(x + 8 * c, v[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) amax = umax(amax, abs_bits(v[0][j]));
        }
        if (tid == 0) out.ask_weight(m.rows);
        const I8Scale s(row_max<W>(amax, red));
        for (int c = tid; c < n8; c += TH) {
            load8(x + 8 * c, v[0]);
            put(v[0], s, c);
        }
        if (tid == 0) out.put(s.s);
    }
}

// Rows of one matrix, then of another, 4 / W per block.  ROUTES: the scales go
// into factors of the outputs.
template <typename S, int NC, int W, bool ROUTES>
__global__ __launch_bounds__(256) void i8_quant_rows_kernel(QuantRows<S> m0, QuantRows<S> m1, I8Factors f) {
    __shared__ uint32_t red[4];
    constexpr int RB = 4 / W;
    const long n0 = (m0.rows + RB - 1) / RB, b = blockIdx.x;
    const bool first = b < n0;
    const long row = RB * (first ? b : b - n0) + threadIdx.x / (64 * W);
    if (row >= (first ? m0.rows : m1.rows)) return;
    if constexpr (ROUTES) {
        if (first) quant_row<S, NC, W>(m0, row, red, RouteFactor{f, row});
        else quant_row<S, NC, W>(m1, row, red, RowScale{m1.sc + row, f.unit + 2 * f.E + 1});
    } else {
        const QuantRows<S> &m = first ? m0 : m1;
        quant_row<S, NC, W>(m, row, red, RowScale{m.sc + row, nullptr});
    }
}

// Power of two u for an expert's down products: y / u, y = sd[n] (Hq . Wd_q) with K
// codes of at most 127 on either side, lies below 2^15 for the largest channel scale.
DEV float down_unit(uint32_t most, int K) {
    const int dot = 32 - __builtin_clz(127u * 127u * (uint32_t)K - 1u);   // |Hq . Wd_q| <= 2^dot
    const int x = dot + ((int)(most >> 23) - 126) - 15;
    return ldexpf(1.0f, min(max(x, -126), 126));
}

// The tile products' prologue in one launch: the experts' units, one per block,
// the tokens' rows, and the token of every position of the plan (0 where the plan
// has none), 256 per block.
template <int NC, int W>
__global__ __launch_bounds__(256) void i8_prologue_kernel(QuantRows<uint16_t> x, const int *__restrict__ perm,
                                                          const int *__restrict__ offsets, int k, int R,
                                                          int *__restrict__ rowidx, I8Units un) {
    __shared__ uint32_t red[4];
    constexpr int RB = 4 / W;
    const int E = un.E, units = E + (un.fs > 0 ? 1 : 0);
    if ((int)blockIdx.x < units) {
        const int e = (int)blockIdx.x, N = x.K;
        const float *s = e < E ? un.Wd_s + (long)e * N : un.Sd_s;
        uint32_t most = 0;                   // (NaN scales aside: their channels are NaN anyway)
        for (int c = 8 * threadIdx.x; c < N; c += 2048) {
            float v[8];
            load8(s + c, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) most = umax(most, abs_bits(v[j]) < 0x7f800000u ? abs_bits(v[j]) : 0u);
        }
        const float u = down_unit(row_max<4>(most, red), e < E ? un.f : un.fs);
        if (threadIdx.x == 0) {
            un.unit[2 * e] = 1.0f / u;
            un.unit[2 * e + 1] = u;
        }
        return;
    }
    const long n0 = (x.rows + RB - 1) / RB, b = (long)blockIdx.x - units;
    if (b < n0) {
        const long row = RB * b + threadIdx.x / (64 * W);
        if (row < x.rows) quant_row<uint16_t, NC, W>(x, row, red, RowScale{x.sc + row, nullptr});
        return;
    }
    const int p = (int)(b - n0) * 256 + threadIdx.x;
    if (p >= R) return;
    const int j = p < offsets[E] ? perm[p] : -1;
    rowidx[p] = j >= 0 && j < R ? j / k : 0;
}

// A block per 64 channels of an expert: the channels' largest magnitudes over
// all K rows, then the codes, 128 rows at a time through LDS so that reads
// (along n) and writes (along k) are whole 128-byte lines.  The second pass
// reads what the first left in the caches, or in HBM again where the weights in work
// are larger: 128 experts of 768, d 2048 606 us for 1.2 GB of weights and 0.6 of
// codes, which is 5 TB/s with both passes (348 at a large copy's 5.2 TB/s with one); 32 of
// 1536, d 4096 661, the same bytes.  Few experts leave it to latency, a block per 64
// channels: 8 of 2048 and a shared one, d 7168 920 us for 1.2 GB in all (229).
constexpr int QW_PITCH = 128 + 16;
__global__ __launch_bounds__(256) void i8_quant_weights_kernel(const uint16_t *__restrict__ W, int K,
                                                               int N, uint8_t *__restrict__ q,
                                                               float *__restrict__ sc) {
    __shared__ __attribute__((aligned(16))) uint8_t tile[64 * QW_PITCH];
    __shared__ uint32_t red[32][64];
    const int ntn = N / 64, e = blockIdx.x / ntn, n0 = blockIdx.x % ntn * 64;
    const int r = threadIdx.x >> 3, c = 8 * (threadIdx.x & 7);
    const uint16_t *src = W + (long)e * K * N + n0 + c;
    uint32_t amax[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int k0 = 0; k0 < K; k0 += 128) {    // K is a multiple of 256
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) load8(src + (long)(k0 + 32 * i + r) * N, v[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) amax[j] = umax(amax[j], abs_bits(v[i][j]));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) red[r][c + j] = amax[j];
    __syncthreads();
    if (threadIdx.x < 64) {
        uint32_t m = 0;
        for (int i = 0; i < 32; ++i) m = umax(m, red[i][threadIdx.x]);
        red[0][threadIdx.x] = m;
        sc[(long)e * N + n0 + threadIdx.x] = I8Scale(m).s;
    }
    __syncthreads();
    uint32_t top[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) top[j] = red[0][c + j];
    const int oc = threadIdx.x >> 2, ok = 32 * (threadIdx.x & 3);
    uint8_t *dst = q + ((long)e * N + n0 + oc) * K + ok;
    for (int k0 = 0; k0 < K; k0 += 128) {
        float v[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) load8(src + (long)(k0 + 32 * i + r) * N, v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const I8Scale s(top[j]);
#pragma unroll
            for (int i = 0; i < 4; ++i) tile[(c + j) * QW_PITCH + 32 * i + r] = (uint8_t)s.code(v[i][j]);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h)
            st_u32x4(dst + k0 + 16 * h, ld_u32x4(tile + oc * QW_PITCH + ok + 16 * h));
        __syncthreads();
    }
}

// f(NC, W) for rows of K elements, which stay in registers up to 8192: a block per
// row, or a wave if a quarter of a block's threads would have nothing to do and
// there are rows for every CU (whole forward, us by waves / by blocks: 65536 rows of
// 768 555 / 591; 32768 of 256 85 / 105; 131072 of 1536 2850 / 2867; 8000 of 1536 260.4 /
// 260.2; 36891 of 2048, all threads busy, 1772 / 1769; 128 of 1536 139 / 137).  They move
// 5.2 TB/s from 131072 rows of 1536 (186 us), and few rows take a launch's time (5 us).
// The weights of the tile products' routes cost the rows' launch three dependent
// loads: 8192 tokens to 8 of 128 experts of 768 45 -> 52 us, 4099 to 8 and a shared one
// of 2048 68 -> 82, which the down product and the sum save.
constexpr long QUANT_WAVE_ROWS = 2048;
template <typename F>
hipError_t with_chunks(long rows, int K, F f) {
    if (rows >= QUANT_WAVE_ROWS && K <= 1536) {
        if (K <= 512) f(Const<1>{}, Const<1>{});
        else if (K <= 1024) f(Const<2>{}, Const<1>{});
        else f(Const<3>{}, Const<1>{});
    }
    else if (K <= 2048) f(Const<1>{}, Const<4>{});
    else if (K <= 4096) f(Const<2>{}, Const<4>{});
    else if (K <= 8192) f(Const<4>{}, Const<4>{});
    else f(Const<0>{}, Const<4>{});
    return hipGetLastError();
}
unsigned row_blocks(long rows, int W) { return (unsigned)((rows + 4 / W - 1) / (4 / W)); }

}  // namespace

hipError_t launch_i8_quant_tokens(const uint16_t *X, long rows, int K, uint8_t *q, float *sc, hipStream_t st) {
    if (rows <= 0) return hipSuccess;
    const QuantRows<uint16_t> m{X, q, sc, rows, K};
    return with_chunks(rows, K, [&](auto nc, auto w) {
        i8_quant_rows_kernel<uint16_t, decltype(nc)::value, decltype(w)::value, false>
            <<<dim3(row_blocks(rows, w.value)), dim3(256), 0, st>>>(m, QuantRows<uint16_t>{}, I8Factors{});
    });
}
hipError_t launch_i8_prologue(const uint16_t *X, int T, int d, uint8_t *q, float *sc, const int *perm,
                              const int *offsets, int k, int *rowidx, const I8Units &units,
                              hipStream_t st) {
    if (T <= 0) return hipSuccess;
    const QuantRows<uint16_t> m{X, q, sc, T, d};
    const int R = T * k;
    return with_chunks(T, d, [&](auto nc, auto w) {
        const dim3 grid((unsigned)(units.E + (units.fs > 0)) + row_blocks(T, w.value) + (unsigned)((R + 255) / 256));
        i8_prologue_kernel<decltype(nc)::value, decltype(w)::value><<<grid, dim3(256), 0, st>>>(
            m, perm, offsets, k, R, rowidx, units);
    });
}
hipError_t launch_i8_quant_h(const float *H, long rows, int f, uint8_t *q, float *sc, const float *Hs,
                             long rows_s, int fs, uint8_t *qs, float *scs, const I8Factors &factors,
                             hipStream_t st) {
    if (rows + rows_s <= 0) return hipSuccess;
    const QuantRows<float> m{H, q, sc, rows, f}, ms{Hs, qs, scs, rows_s, fs};
    return with_chunks(rows + rows_s, rows_s > 0 && fs > f ? fs : f, [&](auto nc, auto w) {
        const dim3 grid(row_blocks(rows, w.value) + row_blocks(rows_s, w.value));
        if (factors.perm)
            i8_quant_rows_kernel<float, decltype(nc)::value, decltype(w)::value, true>
                <<<grid, dim3(256), 0, st>>>(m, ms, factors);
        else
            i8_quant_rows_kernel<float, decltype(nc)::value, decltype(w)::value, false>
                <<<grid, dim3(256), 0, st>>>(m, ms, factors);
    });
}
hipError_t launch_i8_quant_weights(const uint16_t *W, int E, int K, int N, uint8_t *q, float *sc,
                                   hipStream_t st) {
    i8_quant_weights_kernel<<<dim3((unsigned)(E * (N / 64))), dim3(256), 0, st>>>(W, K, N, q, sc);
    return hipGetLastError();
}
