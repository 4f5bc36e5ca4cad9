// Routing by scores: the experts of a token are chosen by s_e + balance_e
// among the best groups of experts and weighted by their scores s_e (sigmoid
// or softmax of the logits), and the gradient of those weights.
//
// Choosing has to be right next to a border, where two experts' scores differ
// in the last bits: the ranking value c_e = s_e + balance_e is held in 64 bits
// and ranked on its sign, exponent and the upper 44 bits of its mantissa; the
// 8 bits below hold 255 - e, so rank order, ties to the lower id, is plain
// order of unsigned 64-bit entries (and 2^-44 is far below the rounding of
// any logit).  Where the balance is null and no group adds scores, the order
// of the scores is that of the logits, which are ranked as they are.
//
// Out-of-play experts (logit or balance below MASKED or NaN) have score 0 and
// rank after every other expert of the kept groups, lower ids first.  Logits
// above FLT_MAX count as FLT_MAX.
#include <cfloat>

#include "common.h"
#include "kernels.h"
#include "topk.h"

namespace {

constexpr float MASKED = -1e38f;

DEV double shfl_xor_d(double v, int m) {
    return __longlong_as_double((long long)shfl_xor_u64((uint64_t)__double_as_longlong(v), m));
}
// Unsigned key with the order of the double, its 8 lowest bits free.
DEV uint64_t rank_key(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);   // -0 and 0 are one
    return ((b >> 63) ? ~b : (b | (1ull << 63))) & ~0xffull;
}
constexpr uint64_t MASKED_KEY = 0x100;   // below every rank_key, above the padding 0

// exp(z - m) / ... of a chosen expert; the scores are computed in 32 bits.
DEV float sigmoid32(float z) { return 1.0f / (1.0f + expf(-z)); }

constexpr int PE = 16;   // experts per lane at most

// L lanes share a token.  The groups of experts are dealt to lanes, `lpg` lanes
// to a group, each lane taking every lpg-th expert of its group, so that the
// lanes of a load read neighbouring logits and a group's best scores meet in
// log2 lpg exchanges.  Each lane sorts its entries best first in groups of KP
// (k rounded up to a power of two); the lanes' lists are merged in log2 L
// rounds, after which every lane of the token has its best KP.  Then lane j
// finishes the j-th best expert: its place in ascending id and its weight.
template <int L, int KP>
__global__ __launch_bounds__(256) void score_select_kernel(
        const float *__restrict__ part, int S, int epad, const float *__restrict__ bias,
        const float *__restrict__ balance, float *__restrict__ logits, int *__restrict__ topk_idx,
        float *__restrict__ topk_w, int T, int E, int k, int lpg, ScoreArgs a) {
    __shared__ float zs[256 * PE];           // the block's logits, clamped, by token and expert
    const int sub = threadIdx.x % L;
    const long tk = (long)blockIdx.x * (256 / L) + threadIdx.x / L;
    const int t = (int)(tk < T ? tk : T - 1);
    const bool store = tk < T;
    const int grp = sub / lpg, lane0 = sub % lpg, n = E / a.groups;
    float *const ztok = zs + (threadIdx.x / L) * (L * PE);

    // ---------------- logits ----------------
    float z[PE];
    uint32_t in = 0, live = 0;               // bit i: expert i of the lane exists, is in play
#pragma unroll
    for (int i = 0; i < PE; ++i) {
        const int off = lane0 + lpg * i, id = grp * n + off;
        z[i] = 0.f;
        if (grp < a.groups && off < n) {
            in |= 1u << i;
            if (S == 0) z[i] = logits[(long)t * E + id];
        }
    }
    if (S > 0) {
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < PE; ++i)
                if ((in >> i) & 1) {
                    const float v = part[((long)s * T + t) * epad + grp * n + lane0 + lpg * i];
                    z[i] = s == 0 ? v : z[i] + v;
                }
#pragma unroll
        for (int i = 0; i < PE; ++i)
            if ((in >> i) & 1) {
                const int id = grp * n + lane0 + lpg * i;
                if (bias) z[i] = z[i] + bias[id];
                if (store) logits[(long)t * E + id] = z[i];
            }
    }
    const bool by_score = balance || (a.groups > 1 && a.pair);
    float bal[PE];
#pragma unroll
    for (int i = 0; i < PE; ++i) {
        bal[i] = 0.f;
        if ((in >> i) & 1) {
            const int id = grp * n + lane0 + lpg * i;
            if (balance) bal[i] = balance[id];
            if (z[i] >= MASKED && bal[i] >= MASKED) live |= 1u << i;
            z[i] = fminf(z[i], FLT_MAX);
            ztok[id] = z[i];
        }
    }

    // ---------------- softmax over the row ----------------
    float zmax = -INFINITY;
    double sum = 0.0;
    if (!a.sigmoid && (by_score || !a.renorm)) {
#pragma unroll
        for (int i = 0; i < PE; ++i)
            if ((live >> i) & 1) zmax = fmaxf(zmax, z[i]);
#pragma unroll
        for (int m = 1; m < L; m <<= 1) zmax = fmaxf(zmax, shfl_xor_f(zmax, m));
    }

    // ---------------- ranking values ----------------
    double v[PE];
#pragma unroll
    for (int i = 0; i < PE; ++i) {
        v[i] = (double)z[i];
        if (a.sigmoid) {
            if (by_score) v[i] = 1.0 / (1.0 + exp(-v[i]));
        } else if (by_score || !a.renorm) {
            const double x = ((live >> i) & 1) ? exp(v[i] - (double)zmax) : 0.0;
            sum += x;
            if (by_score) v[i] = x;
        }
    }
    if (!a.sigmoid && (by_score || !a.renorm)) {
#pragma unroll
        for (int m = 1; m < L; m <<= 1) sum += shfl_xor_d(sum, m);
    }
    double b1 = -INFINITY, b2 = -INFINITY;   // the group's two largest
    uint64_t key[PE];
#pragma unroll
    for (int i = 0; i < PE; ++i) {
        const int id = grp * n + lane0 + lpg * i;
        key[i] = 0;
        if (!((in >> i) & 1)) continue;
        key[i] = MASKED_KEY | (uint64_t)(255 - id);
        if (!((live >> i) & 1)) continue;
        if (by_score) {
            if (!a.sigmoid) v[i] = v[i] / sum;
            v[i] = v[i] + (double)bal[i];
        }
        key[i] = rank_key(v[i]) | (uint64_t)(255 - id);
        b2 = fmax(b2, fmin(b1, v[i]));
        b1 = fmax(b1, v[i]);
    }

    // ---------------- the lane's best KP, sorted ----------------
    uint64_t bk[KP];
    constexpr int G = PE < KP ? PE : KP;
#pragma unroll
    for (int g0 = 0; g0 < PE; g0 += G) {
        uint64_t w[KP];
#pragma unroll
        for (int j = 0; j < KP; ++j) w[j] = j < G ? key[g0 + j] : 0ull;
        sort_desc<KP>(w);
        if (g0 == 0) {
#pragma unroll
            for (int j = 0; j < KP; ++j) bk[j] = w[j];
        } else {
            merge_best<KP>(bk, w);
        }
    }

    // ---------------- groups ----------------
    if (a.groups > 1) {
        for (int m = 1; m < lpg; m <<= 1) {
            const double o1 = shfl_xor_d(b1, m), o2 = shfl_xor_d(b2, m);
            b2 = fmax(fmin(b1, o1), fmax(b2, o2));
            b1 = fmax(b1, o1);
        }
        const double gs = a.pair && b2 > -INFINITY ? b1 + b2 : b1;
        const uint64_t gk = grp < a.groups ? rank_key(gs) | (uint64_t)(255 - grp) : 0ull;
        int better = 0;
        for (int o = 0; o < a.groups; ++o) {
            const int lo = __shfl((int)(uint32_t)gk, o * lpg, L);
            const int hi = __shfl((int)(uint32_t)(gk >> 32), o * lpg, L);
            const uint64_t og = ((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo;
            better += og > gk ? 1 : 0;
        }
        if (better >= a.top_groups) {
#pragma unroll
            for (int j = 0; j < KP; ++j) bk[j] = 0;
        }
    }

    // ---------------- the token's best KP ----------------
#pragma unroll
    for (int m = 1; m < L; m <<= 1) {
        uint64_t o[KP];
#pragma unroll
        for (int j = 0; j < KP; ++j) o[j] = shfl_xor_u64(bk[j], m);
        merge_best<KP>(bk, o);
    }
    __syncthreads();                         // ztok is written

    // ---------------- ids and weights of the chosen ----------------
    constexpr int JN = (KP + L - 1) / L;     // slots per lane
    int id[JN], at[JN];
    float zc[JN];
    bool on[JN];
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < JN; ++q) {
        const int j = q * L + sub;
        uint64_t en = 0;
#pragma unroll
        for (int i = 0; i < KP; ++i)
            if (i == j) en = bk[i];
        id[q] = 255 - (int)(en & 0xff);
        at[q] = 0;
#pragma unroll
        for (int i = 0; i < KP; ++i)
            if (i < k && 255 - (int)(bk[i] & 0xff) < id[q]) ++at[q];
        on[q] = j < k && (en >> 8) > (MASKED_KEY >> 8);
        zc[q] = on[q] ? ztok[id[q]] : 0.f;
        if (on[q]) m = fmaxf(m, a.sigmoid ? fminf(zc[q], 0.f) : zc[q]);
    }
    float u[JN], total = 1.0f;
    if (a.renorm) {
        // ratios of scores, taken to the largest of them: scores that underflow
        // together keep their ratio
#pragma unroll
        for (int x = 1; x < L; x <<= 1) m = fmaxf(m, shfl_xor_f(m, x));
        total = 0.f;
#pragma unroll
        for (int q = 0; q < JN; ++q) {
            u[q] = 0.f;
            if (on[q])
                u[q] = a.sigmoid ? expf(fminf(zc[q], 0.f) - m) / (1.0f + expf(-fabsf(zc[q]))) : expf(zc[q] - m);
            total = total + u[q];
        }
#pragma unroll
        for (int x = 1; x < L; x <<= 1) total = total + shfl_xor_f(total, x);
    } else {
#pragma unroll
        for (int q = 0; q < JN; ++q) {
            u[q] = 0.f;
            if (on[q]) u[q] = a.sigmoid ? sigmoid32(zc[q]) : expf(zc[q] - zmax) / (float)sum;
        }
    }
#pragma unroll
    for (int q = 0; q < JN; ++q)
        if (store && q * L + sub < k) {
            topk_idx[(long)t * k + at[q]] = id[q];
            topk_w[(long)t * k + at[q]] = u[q] > 0.f ? a.scale * (u[q] / total) : 0.f;
        }
}

// The gradient of the weights w_i = scale u_i with respect to the logits, for
// dw_i = dL/dw_i of the chosen experts:
//   softmax, renormalised:  dZ_i = w_i (dw_i - sum_j u_j dw_j)
//   sigmoid, renormalised:  the same times (1 - s_i)
//   sigmoid:                dZ_i = w_i (1 - s_i) dw_i
//   softmax:                dZ_e = [e chosen] w_e dw_e - s_e sum_j w_j dw_j
// and 0 elsewhere.  16 tokens per block, lane s of a token's 16 takes slot s;
// the rows are put together in LDS, where the chosen entries are scattered,
// and leave in one contiguous run (a row of E floats starts anywhere, 16 of
// them start at a multiple of 64 bytes).  Bound by that store.
constexpr int SB_BT = 16;
__global__ __launch_bounds__(256) void score_bwd_kernel(
        const float *__restrict__ logits, const float *__restrict__ balance,
        const int *__restrict__ topk_idx, const float *__restrict__ dw, const float *__restrict__ dgpart,
        int nparts, const int *__restrict__ route_pos, float *__restrict__ dg_out,
        float *__restrict__ dZ, int T, int E, int k, ScoreArgs a) {
    __shared__ __attribute__((aligned(16))) float row[SB_BT * 256];
    const int t0 = blockIdx.x * SB_BT, tl = threadIdx.x >> 4, s = threadIdx.x & 15;
    const int t = t0 + tl;
    const bool dense = !a.sigmoid && !a.renorm;
    const int total = min(SB_BT, T - t0) * E;
    const float *src = logits + (long)t0 * E;
    float *out = dZ + (long)t0 * E;
    for (int i = threadIdx.x; i < SB_BT * E / 4; i += 256) {
        f32x4_t v = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (dense) {
            if (4 * i + 3 < total) {
                v = *reinterpret_cast<const f32x4_t *>(src + 4 * i);
            } else {
                for (int q = 0; q < 4; ++q)
                    if (4 * i + q < total) v[q] = src[4 * i + q];
            }
        }
        *reinterpret_cast<f32x4_t *>(row + 4 * i) = v;
    }

    const bool slot = t < T && s < k;
    int e = -1;
    float g = 0.f;                           // dL/dw of the slot
    if (slot) {
        const long j = (long)t * k + s;
        e = topk_idx[j];
        if (dw) {
            g = dw[j];
        } else {
            const int p = route_pos[j];
            if (p >= 0 && p < T * k) {
                for (int q0 = 0; q0 < nparts; q0 += 8) {
                    float v[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        v[q] = q0 + q < nparts ? dgpart[(long)p * nparts + q0 + q] : 0.f;
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (q0 + q < nparts) g = g + v[q];
                }
                dg_out[p] = g;
            }
        }
    }
    __syncthreads();
    auto live = [&](float z, int id) { return z >= MASKED && !(balance && !(balance[id] >= MASKED)); };
    float z = 0.f;
    bool on = slot && e >= 0 && e < E;
    if (on) {
        z = dense ? row[tl * E + e] : logits[(long)t * E + e];
        on = live(z, e);
        z = fminf(z, FLT_MAX);
    }
    // reductions over the token's 16 lanes
    auto max16 = [](float x) {
#pragma unroll
        for (int m = 1; m < 16; m <<= 1) x = fmaxf(x, shfl_xor_f(x, m));
        return x;
    };
    auto sum16 = [](float x) {
#pragma unroll
        for (int m = 1; m < 16; m <<= 1) x = x + shfl_xor_f(x, m);
        return x;
    };
    float u = 0.f, zmax = -INFINITY, zsum = 1.f;
    if (a.renorm) {
        const float m = max16(on ? (a.sigmoid ? fminf(z, 0.f) : z) : -INFINITY);
        if (on) u = a.sigmoid ? expf(fminf(z, 0.f) - m) / (1.0f + expf(-fabsf(z))) : expf(z - m);
        const float tot = sum16(u);
        if (on) u = u / tot;
    } else if (a.sigmoid) {
        if (on) u = sigmoid32(z);
    } else {
        for (int i = s; i < E; i += 16) {
            const float x = row[tl * E + i];
            if (live(x, i)) zmax = fmaxf(zmax, fminf(x, FLT_MAX));
        }
        zmax = max16(zmax);
        zsum = 0.f;
        for (int i = s; i < E; i += 16) {
            const float x = row[tl * E + i];
            if (live(x, i)) zsum = zsum + expf(fminf(x, FLT_MAX) - zmax);
        }
        zsum = sum16(zsum);
        if (on) u = expf(z - zmax) / zsum;
    }
    if (!on) g = 0.f;                        // a masked expert's weight is the constant 0
    const float dot = sum16(u * g);
    float d = a.scale * u;
    d = a.renorm ? d * (g - dot) : d * g;
    if (a.sigmoid) d = d / (1.0f + expf(z)); // 1 - s
    if (dense) {
        for (int i = s; i < E; i += 16) {
            const float x = row[tl * E + i];
            const float p = live(x, i) ? expf(fminf(x, FLT_MAX) - zmax) / zsum : 0.f;
            row[tl * E + i] = -p * (a.scale * dot);
        }
    }
    __syncthreads();
    // an id listed twice gets the sum, from its first slot
    bool first = true;
    float add = 0.f;
    for (int i = 0; i < k; ++i) {
        const int ei = __shfl(e, i, 16);
        const float di = __shfl(d, i, 16);
        if (ei == e) {
            if (i < s) first = false;
            add = add + di;
        }
    }
    if (on && first) row[tl * E + e] = row[tl * E + e] + add;
    __syncthreads();
    for (int i = threadIdx.x; i < SB_BT * E / 4; i += 256) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t *>(row + 4 * i);
        if (4 * i + 3 < total) {
            *reinterpret_cast<f32x4_t *>(out + 4 * i) = v;
        } else {
            for (int q = 0; q < 4; ++q)
                if (4 * i + q < total) out[4 * i + q] = v[q];
        }
    }
}

int pow2(int x) {
    int p = 1;
    while (p < x) p *= 2;
    return p;
}

template <int L>
hipError_t select_lanes(const float *part, int S, int epad, const float *bias, const float *balance,
                        float *logits, int *idx, float *w, int T, int E, int k, int lpg,
                        const ScoreArgs &a, hipStream_t st) {
    const long per = 256 / L;
    const dim3 grid((unsigned)((T + per - 1) / per)), block(256);
#define SELECT(KP) \
    score_select_kernel<L, KP><<<grid, block, 0, st>>>(part, S, epad, bias, balance, logits, idx, w, T, E, k, lpg, a)
    switch (pow2(k)) {
        case 1: SELECT(1); break;
        case 2: SELECT(2); break;
        case 4: SELECT(4); break;
        case 8: SELECT(8); break;
        case 16: SELECT(16); break;
        default: return hipErrorInvalidValue;
    }
#undef SELECT
    return hipGetLastError();
}

}  // namespace

hipError_t launch_score_select(const float *part, int S, int epad, const float *bias,
                               const float *balance, float *logits, int *topk_idx, float *topk_w, int T,
                               int E, int k, const ScoreArgs &a, hipStream_t st) {
    if (T <= 0) return hipSuccess;
    // lanes per group: as many as hold its experts, PE each
    const int n = E / a.groups, lpg = pow2((n + PE - 1) / PE), L = pow2(a.groups) * lpg;
#define LANES(N)                                                                                        \
    case N:                                                                                             \
        return select_lanes<N>(part, S, epad, bias, balance, logits, topk_idx, topk_w, T, E, k, lpg, a, st)
    switch (L) {
        LANES(1);
        LANES(2);
        LANES(4);
        LANES(8);
        LANES(16);
        LANES(32);
        LANES(64);
        default: return hipErrorInvalidValue;
    }
#undef LANES
}

hipError_t launch_score_bwd(const float *logits, const float *balance, const int *topk_idx,
                            const float *dw, const float *dgpart, int nparts, const int *route_pos,
                            float *dg_out, float *dZ, int T, int E, int k, const ScoreArgs &a,
                            hipStream_t st) {
    if (T <= 0) return hipSuccess;
    score_bwd_kernel<<<dim3((unsigned)((T + SB_BT - 1) / SB_BT)), dim3(256), 0, st>>>(
        logits, balance, topk_idx, dw, dgpart, nparts, route_pos, dg_out, dZ, T, E, k, a);
    return hipGetLastError();
}
