// Routing by scores: the experts of a token are chosen by s_e + balance_e
// among the best groups of experts and weighted by their scores s_e (sigmoid
// or softmax of the logits), and the gradient of those weights.
//
// Choosing has to be right next to a border, where two experts' values differ
// in the last bits, and the values that are ranked, c_e = s_e + balance_e, are
// defined in 64 bits (without a balance and without sums over groups the order
// is that of the logits, which are ranked as they are).  The selection runs in
// 32 bits first: c_e is computed in fp32 and laid on 24 bits between the row's
// smallest and largest, 8 bits below hold 255 - e, and the entries go through
// sorting networks of integer maxima and minima.  The first expert left out and
// the last one taken then say whether the errors of the fp32 values could have
// swapped them, and likewise the groups; only where they could (some 15 tokens in
// 100000, and rows of exact ties) the experts that the errors reach, mostly two,
// are ranked again by 64-bit values, in compact loops.  A selection in 64 bits
// throughout spent 25-50 us, most of it on fetching its unrolled code (30 us for a
// single token); this one takes 6.7 us for one token to 256 experts in 8 groups
// (28 slices of partial logits; a launch's and a round trip's time), 13.1
// for 4099 (29 MB of partial logits) and 13.8 for 16384 to 128 experts (networks
// and exponentials; the partial logits are 17 MB).  Where every expert of every
// token ties, as with a router of zeros, whole calls take 56 us for 39 (4099 tokens)
// and 47 for 29 (16384).
//
// The 64-bit side compares all 64 bits and then the ids: saturated sigmoids, and
// small scores beside a balance, differ in their last bits alone.
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
// Unsigned key with the order of the double, above 0 and below ~0.
DEV uint64_t rank_key(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);   // -0 and 0 are one
    return (b >> 63) ? ~b : (b | (1ull << 63));
}
constexpr uint32_t MASKED_Q = 1, FIRST_Q = 3;   // 24-bit places: masked; in play, from

DEV float sigmoid32(float z) { return 1.0f / (1.0f + expf(-z)); }
DEV uint32_t umax32(uint32_t a, uint32_t b) { return a > b ? a : b; }

template <int N> struct Int { static constexpr int value = N; };

// The value of a lane at distance M, for exchanges that run M = 1, 2, 4, ... and
// leave the lanes below M equal: a mirrored half row or row then serves as
// well as the xor, and DPP moves take a few cycles where a shuffle goes through
// the LDS unit.
template <int M>
DEV uint32_t peer(uint32_t v) {
    // quads 1,0,3,2 and 2,3,0,1; half rows and rows mirrored
    constexpr int ctrl = M == 1 ? 0xB1 : M == 2 ? 0x4E : M == 4 ? 0x141 : 0x140;
    if constexpr (M <= 8) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, ctrl, 0xF, 0xF, true);
    else return (uint32_t)__shfl_xor((int)v, M, 64);
}
template <int M>
DEV float peer_f(float v) { return __uint_as_float(peer<M>(__float_as_uint(v))); }
// f<M>() for M = 1, 2, ... below L (and below `most`)
template <int L, typename F>
DEV void exchanges(int most, F f) {
    if constexpr (L > 1) { if (1 < most) f(Int<1>{}); }
    if constexpr (L > 2) { if (2 < most) f(Int<2>{}); }
    if constexpr (L > 4) { if (4 < most) f(Int<4>{}); }
    if constexpr (L > 8) { if (8 < most) f(Int<8>{}); }
    if constexpr (L > 16) { if (16 < most) f(Int<16>{}); }
    if constexpr (L > 32) { if (32 < most) f(Int<32>{}); }
}

// The 64-bit side of a token's selection: its logits, balance and row maximum.
struct Exact {
    const float *zt, *sbal;
    bool by_score, sigmoid;
    float zmax;
    double sum;
    DEV double value(int id) const {
        double v = (double)fminf(zt[id], FLT_MAX);
        if (by_score) {
            const double x = exp(sigmoid ? -v : v - (double)zmax);
            v = (sigmoid ? 1.0 / (1.0 + x) : x / sum) + (double)sbal[id];
        }
        return v;
    }
};
// The softmax's denominator.
template <int PE, int L>
DEV void exact_sum(Exact &x, uint32_t live, int first, int lpg) {
    x.sum = 0.0;
    if (!x.by_score || x.sigmoid) return;
#pragma unroll 4
    for (int i = 0; i < PE; ++i) {
        const bool on = (live >> i) & 1;
        const double v = exp((double)fminf(x.zt[on ? first + lpg * i : 0], FLT_MAX) - (double)x.zmax);
        x.sum += on ? v : 0.0;
    }
#pragma unroll 1
    for (int m = 1; m < L; m <<= 1) x.sum += shfl_xor_d(x.sum, m);
}

// The groups near the border by their 64-bit values: those surely in (`sure` >
// 0) rank before, those surely out (< 0) after all of them.  Returns whether
// this lane's group is kept.
template <int PE, int L>
DEV bool groups_64(Exact x, uint32_t live, int grp, int first, int lpg, int sure, const ScoreArgs &a) {
    exact_sum<PE, L>(x, live, first, lpg);
    double b1 = -INFINITY, b2 = -INFINITY;
    if (sure == 0) {
#pragma unroll 4
        for (int i = 0; i < PE; ++i) {
            const bool on = (live >> i) & 1;
            const double v = on ? x.value(first + lpg * i) : -INFINITY;
            b2 = fmax(b2, fmin(b1, v));
            b1 = fmax(b1, v);
        }
    }
#pragma unroll 1
    for (int m = 1; m < lpg; m <<= 1) {
        const double o1 = shfl_xor_d(b1, m), o2 = shfl_xor_d(b2, m);
        b2 = fmax(fmin(b1, o1), fmax(b2, o2));
        b1 = fmax(b1, o1);
    }
    double gs = a.pair && b2 > -INFINITY ? b1 + b2 : b1;
    const uint64_t gk = sure > 0 ? ~0ull : sure < 0 ? 0ull : rank_key(gs);
    int better = 0;
#pragma unroll 1
    for (int o = 0; o < a.groups; ++o) {
        const int lo = __shfl((int)(uint32_t)gk, o * lpg, L);
        const int hi = __shfl((int)(uint32_t)(gk >> 32), o * lpg, L);
        const uint64_t og = ((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo;
        better += og > gk || (og == gk && o < grp) ? 1 : 0;
    }
    return better < a.top_groups;
}

// Places `from` .. k - 1 of the token's chosen experts: the best, by their
// 64-bit values, ties to the lower id, of the candidates (bits of `cand` for this
// lane's experts, in ascending id; at least k - from of them in the token's lanes).
// kb: room for this lane's keys, at stride 256.
template <int PE, int L, int KP>
DEV void select_64(Exact x, uint64_t *kb, uint32_t live, uint32_t cand, int first, int lpg, int from,
                   int k, uint32_t (&bk)[KP]) {
    exact_sum<PE, L>(x, live, first, lpg);
#pragma unroll 1
    for (uint32_t m = cand; m; m &= m - 1) {
        const int i = __builtin_ctz(m);
        kb[256 * i] = rank_key(x.value(first + lpg * i));
    }
#pragma unroll 1
    for (int r = from; r < k; ++r) {
        uint64_t best = 0;
        int at = -1;
#pragma unroll 1
        for (uint32_t m = cand; m; m &= m - 1) {
            const int i = __builtin_ctz(m);
            const uint64_t key = kb[256 * i];
            if (key > best) {
                best = key;
                at = i;
            }
        }
        const int mine = at < 0 ? 256 : first + lpg * at;
        int id = mine;
#pragma unroll 1
        for (int m = 1; m < L; m <<= 1) {
            const uint64_t o = shfl_xor_u64(best, m);
            const int oid = __shfl_xor(id, m, 64);
            const bool ahead = o > best || (o == best && oid < id);
            best = ahead ? o : best;
            id = ahead ? oid : id;
        }
        if (mine == id) cand &= ~(1u << (at & 31));   // ids differ, so one lane's
        const uint32_t e = (FIRST_Q << 8) | (uint32_t)(255 - id);
#pragma unroll
        for (int j = 0; j < KP; ++j)
            if (j == r) bk[j] = e;
    }
}

// The block's 256 / L tokens go through LDS: their logits, or the partial
// logits of S slices added in slice order, 16 bytes per load.  Then L lanes
// share a token, up to PE experts each.  The groups of experts are dealt to
// lanes, `lpg` lanes to a group, each lane taking every lpg-th expert of its group,
// so that a group's best values meet in log2 lpg exchanges.  Each lane sorts its entries best
// first in groups of KP (k rounded up to a power of two); the lanes' lists are
// merged in log2 L rounds, after which every lane of the token has its best KP
// and the best entry that was left out.  Then lane j finishes the j-th best
// expert: its place in ascending id and its weight.
template <int PE, int L, int KP>
__global__ __launch_bounds__(256) void score_select_kernel(
        const float *__restrict__ part, int S, int epad, const float *__restrict__ bias,
        const float *__restrict__ balance, float *__restrict__ logits, int *__restrict__ topk_idx,
        float *__restrict__ topk_w, int T, int E, int k, int lpg, ScoreArgs a) {
    constexpr int TB = 256 / L;
    __shared__ __attribute__((aligned(16))) float zs[256 * PE];   // TB rows of E <= L PE
    __shared__ uint64_t keys[256 * PE];      // room for select_64
    __shared__ float sbal[256];
    // loads return in order: what is needed last is asked for first and used last
    const float my_bal = balance && (int)threadIdx.x < E ? balance[threadIdx.x] : 0.f;
    const long t0 = (long)blockIdx.x * TB;
    const int nt = (int)(T - t0 < TB ? T - t0 : TB);
    float *zrow = logits + t0 * E;           // 16-byte aligned: TB is a multiple of 4
    if (S == 0) {
        for (int i = 4 * threadIdx.x; i < nt * E; i += 1024) {
            if (i + 3 < nt * E) {
                *reinterpret_cast<f32x4_t *>(zs + i) = *reinterpret_cast<const f32x4_t *>(zrow + i);
            } else {
                for (int q = i; q < nt * E; ++q) zs[q] = zrow[q];
            }
        }
    } else {
        // pieces of 4 logits, NH at a time; up to NG groups of GS slices of each in flight
        const int ch = epad / 4, pieces = nt * ch;
        const long pitch = (long)T * epad;
        // 256 is a multiple of ch: a thread's pieces are of the same columns
        const int c = 4 * (threadIdx.x % ch);
        float bz[4] = {0.f, 0.f, 0.f, 0.f};
        if (bias)
#pragma unroll
            for (int q = 0; q < 4; ++q) bz[q] = bias[min(c + q, E - 1)];
        auto add = [&](auto gs, auto ng, auto nh, int i0) {
            constexpr int GS = decltype(gs)::value, NG = decltype(ng)::value, NH = decltype(nh)::value;
            // a piece's place after its slice's first, which is the same for every lane
            uint32_t at[NH];
            f32x4_t v[NH];
#pragma unroll
            for (int h = 0; h < NH; ++h) {
                const int i = min(i0 + 256 * h, pieces - 1);
                at[h] = 4 * (uint32_t)i;
                v[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
            for (int s0 = 0; s0 < S; s0 += GS * NG) {
                f32x4_t u[NG][NH][GS];
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const int s = s0 + GS * g;
                    if (s >= S) break;
#pragma unroll
                    for (int h = 0; h < NH; ++h)
#pragma unroll
                        for (int j = 0; j < GS; ++j)
                            u[g][h][j] = *reinterpret_cast<const f32x4_t *>(
                                part + t0 * epad + min(s + j, S - 1) * pitch + at[h]);
                }
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const int s = s0 + GS * g;
                    if (s >= S) break;
#pragma unroll
                    for (int h = 0; h < NH; ++h)
#pragma unroll
                        for (int j = 0; j < GS; ++j)
                            if (s + j < S)
#pragma unroll
                                for (int q = 0; q < 4; ++q) v[h][q] = v[h][q] + u[g][h][j][q];
                }
            }
#pragma unroll
            for (int h = 0; h < NH; ++h) {
                const int i = i0 + 256 * h;
                if (i >= pieces) break;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (c + q < E) zs[i / ch * E + c + q] = bias ? v[h][q] + bz[q] : v[h][q];
            }
        };
        // 28 or 16 loads in flight per thread, whatever S, and at most three past the last
        // slice (router of 256 experts, us by slices: one token, 8 10.0, 16 10.3, 28 10.7,
        // 32 11.0, 64 12.6; 16 tokens, two pieces per thread, 8 12.0, 16 13.0, 28 14.5, 32
        // 14.9, 64 18.8).  32 of them took more than 128 registers, which leaves a SIMD
        // two waves: 4099 tokens 37.4 -> 39.6, 16384 to 128 experts 27.7 -> 31.3.
        if (pieces <= 256) {
            if ((int)threadIdx.x < pieces) add(Int<4>{}, Int<7>{}, Int<1>{}, threadIdx.x);
        } else {
            for (int i = threadIdx.x; i < pieces; i += 512) {
                if (S <= 2) add(Int<2>{}, Int<1>{}, Int<2>{}, i);
                else add(Int<4>{}, Int<2>{}, Int<2>{}, i);
            }
        }
    }
    if ((int)threadIdx.x < E) sbal[threadIdx.x] = my_bal;
    __syncthreads();
    if (S > 0) {
        for (int i = 4 * threadIdx.x; i < nt * E; i += 1024) {
            if (i + 3 < nt * E) {
                *reinterpret_cast<f32x4_t *>(zrow + i) = *reinterpret_cast<const f32x4_t *>(zs + i);
            } else {
                for (int q = i; q < nt * E; ++q) zrow[q] = zs[q];
            }
        }
    }

    // ---------------- this lane's experts ----------------
    const int sub = threadIdx.x % L, tok = threadIdx.x / L;
    const bool store = tok < nt;
    const int grp = sub / lpg, lane0 = sub % lpg, n = E / a.groups;
    const float *zt = zs + (store ? tok : nt - 1) * E;
    const bool by_score = balance || (a.groups > 1 && a.pair);
    const bool row_sum = !a.sigmoid && (by_score || !a.renorm);
    float c[PE], bal[PE];
    uint32_t in = 0, live = 0;               // bit i: expert i of the lane exists, is in play
    float zmax = -INFINITY;
    // selects, no branches, here and below: the arrays stay in their registers
#pragma unroll
    for (int i = 0; i < PE; ++i) {
        const int off = lane0 + lpg * i;
        const bool is = grp < a.groups && off < n;
        const int id = is ? grp * n + off : 0;
        const float z = zt[id];
        bal[i] = sbal[id];
        const bool on = is && z >= MASKED && bal[i] >= MASKED;
        in |= is ? 1u << i : 0u;
        live |= on ? 1u << i : 0u;
        c[i] = on ? fminf(z, FLT_MAX) : 0.f;
        zmax = fmaxf(zmax, on ? c[i] : -INFINITY);
    }

    // ---------------- ranking values in 32 bits ----------------
    float sum = 0.f, smax = 0.f;
    if (row_sum) {
        exchanges<L>(L, [&](auto m) { zmax = fmaxf(zmax, peer_f<m.value>(zmax)); });
#pragma unroll
        for (int i = 0; i < PE; ++i) {
            const float x = (live >> i) & 1 ? __builtin_amdgcn_exp2f((c[i] - zmax) * 1.4426950408889634f) : 0.f;
            sum = sum + x;
            c[i] = by_score ? x : c[i];
        }
        exchanges<L>(L, [&](auto m) { sum = sum + peer_f<m.value>(sum); });
    }
    if (by_score) {
        const float inv = a.sigmoid ? 1.f : __builtin_amdgcn_rcpf(sum);
#pragma unroll
        for (int i = 0; i < PE; ++i) {
            const float s = a.sigmoid ? sigmoid_f(c[i]) : c[i] * inv;
            smax = fmaxf(smax, (live >> i) & 1 ? s : 0.f);
            c[i] = s + bal[i];
        }
    }
    float hi = -INFINITY, lo = INFINITY;
    float b1 = -INFINITY, b2 = -INFINITY;    // the group's two largest
#pragma unroll
    for (int i = 0; i < PE; ++i) {
        const bool on = (live >> i) & 1;
        const float x = on ? c[i] : -INFINITY;
        lo = fminf(lo, on ? c[i] : INFINITY);
        b2 = fmaxf(b2, fminf(b1, x));
        b1 = fmaxf(b1, x);
    }
    hi = b1;
    exchanges<L>(L, [&](auto m) {
        hi = fmaxf(hi, peer_f<m.value>(hi));
        lo = fminf(lo, peer_f<m.value>(lo));
        smax = fmaxf(smax, peer_f<m.value>(smax));
    });
    // Bound of a value's error, in units of 2^-24 (half an ulp) of the row's largest
    // score S; the hardware's exponential and reciprocal are an ulp off at most.
    // Sigmoid: the exponential's argument, its constant and rounding, is off by 1.23 |z|
    // of itself, so the score s by 1.23 |z| (1 - s) s; 2 (1 - s) s by the exponential, s
    // by the sum, 2 s by the reciprocal.  |z| s is at most 0.28, which is 1.28 S, or,
    // where all scores are small, S times the |z| of the largest, -ln S at most: 5 +
    // 1.23 max(1.28, -ln S).
    // Softmax, x = z - max: 2.23 |x| exp(-|x|) <= 0.82 by the argument, 2 by the
    // exponential, 1 by the product.  The sum and its reciprocal scale all scores of
    // the row alike and move a difference of two by 33 S at most: 2.23 times the
    // mean of |x| under the scores (3.4 for 256 experts), 2 by the exponentials, 20
    // by the additions, 3 by the reciprocal.  Half of it goes to either side: 20.5.
    // Then the addition of the balance, and what underflows.  The 24-bit places below
    // add two units each.
    const float top = fmaxf(fabsf(hi), fabsf(lo));
    const float lost = a.sigmoid ? 8.f - 1.1f * __builtin_amdgcn_logf(fmaxf(smax, 0x1p-126f)) : 21.f;
    const float err = by_score ? (lost * smax + top) * 0x1p-24f + 0x1p-124f : 0.f;
    const float range = hi - lo;
    const bool fits = range > 1e-30f && range < 1e30f;
    const float unit = fits ? 16777200.0f / range : 0.f;
    uint32_t key[PE];
#pragma unroll
    for (int i = 0; i < PE; ++i) {
        const int id = grp * n + lane0 + lpg * i;
        const uint32_t q = (live >> i) & 1 ? FIRST_Q + (uint32_t)((c[i] - lo) * unit) : MASKED_Q;
        key[i] = (in >> i) & 1 ? (q << 8) | (uint32_t)(255 - id) : 0u;
    }

    // ---------------- the lane's best KP, sorted ----------------
    uint32_t bk[KP], out = 0;                // out: the best entry left out
    constexpr int G = PE < KP ? PE : KP;
#pragma unroll
    for (int g0 = 0; g0 < PE; g0 += G) {
        uint32_t w[KP];
#pragma unroll
        for (int j = 0; j < KP; ++j) w[j] = j < G ? key[g0 + j] : 0u;
        sort_desc<KP>(w);
        if (g0 == 0) {
#pragma unroll
            for (int j = 0; j < KP; ++j) bk[j] = w[j];
        } else {
            merge_best<KP>(bk, w);
#pragma unroll
            for (int j = 0; j < KP; ++j) out = umax32(out, w[j]);
        }
    }

    const Exact ex{zt, sbal, by_score, a.sigmoid != 0, zmax, 0.0};
    const int first = grp * n + lane0;

    // ---------------- groups ----------------
    bool kept = true;
    if (a.groups > 1) {
        exchanges<L>(lpg, [&](auto m) {
            const float o1 = peer_f<m.value>(b1), o2 = peer_f<m.value>(b2);
            b2 = fmaxf(fminf(b1, o1), fmaxf(b2, o2));
            b1 = fmaxf(b1, o1);
        });
        const float gs = a.pair && b2 > -INFINITY ? b1 + b2 : b1;
        int better = 0;
        for (int o = 0; o < a.groups; ++o) {
            const float og = __shfl(gs, o * lpg, L);
            better += og > gs || (og == gs && o < grp) ? 1 : 0;
        }
        kept = better < a.top_groups && grp < a.groups;
        if (by_score) {
            // the worst kept group and the best one left out: could errors (of
            // two values and a sum on either side) have swapped them?
            float worst = kept ? gs : INFINITY, next = kept || grp >= a.groups ? -INFINITY : gs;
            exchanges<L>(L, [&](auto m) {
                worst = fminf(worst, peer_f<m.value>(worst));
                next = fmaxf(next, peer_f<m.value>(next));
            });
            const float gerr = 4.f * err + 4.f * top * 0x1p-24f;
            if (next > -INFINITY && !(worst - next > gerr)) {
                const int sure = gs > next + gerr ? 1 : gs < worst - gerr ? -1 : 0;
                kept = groups_64<PE, L>(ex, live, grp, first, lpg, sure, a) && grp < a.groups;
            }
        }
#pragma unroll
        for (int j = 0; j < KP; ++j) bk[j] = kept ? bk[j] : 0u;
        out = kept ? out : 0u;
    }

    // ---------------- the token's best KP ----------------
    exchanges<L>(L, [&](auto m) {
        uint32_t o[KP];
#pragma unroll
        for (int j = 0; j < KP; ++j) o[j] = peer<m.value>(bk[j]);
        out = umax32(out, peer<m.value>(out));
        merge_best<KP>(bk, o);
#pragma unroll
        for (int j = 0; j < KP; ++j) out = umax32(out, o[j]);
    });
    uint32_t last = 0;
#pragma unroll
    for (int j = 0; j < KP; ++j) {
        if (j == k - 1) last = bk[j];
        if (j >= k) out = umax32(out, bk[j]);
    }
    // An expert in play was left out: those that its errors, and the last
    // chosen one's, reach are ranked again.  Values that do not fit 24 bits are
    // ranked again all together.
    const float tol = fits ? fminf(2.f * err * unit + 5.f, 3e7f) : 3e7f;
    if ((out >> 8) >= FIRST_Q && (float)(last >> 8) - (float)(out >> 8) <= tol) {
        const float from_q = (float)(last >> 8) - tol, to_q = (float)(out >> 8) + tol;
        uint32_t cand = 0;
#pragma unroll
        for (int i = 0; i < PE; ++i) {
            const float q = (float)(key[i] >> 8);
            cand |= kept && ((live >> i) & 1) && q >= from_q && q <= to_q ? 1u << i : 0u;
        }
        int from = 0;
#pragma unroll
        for (int j = 0; j < KP; ++j) from += j < k && (float)(bk[j] >> 8) > to_q ? 1 : 0;
        select_64<PE, L, KP>(ex, keys + threadIdx.x, live, cand, first, lpg, from, k, bk);
    }

    // ---------------- ids and weights of the chosen ----------------
    constexpr int JN = (KP + L - 1) / L;     // slots per lane
    int id[JN], at[JN];
    float zc[JN];
    bool on[JN];
    float m = -INFINITY;
#pragma unroll
    for (int q = 0; q < JN; ++q) {
        const int j = q * L + sub;
        uint32_t en = 0;
#pragma unroll
        for (int i = 0; i < KP; ++i)
            if (i == j) en = bk[i];
        id[q] = 255 - (int)(en & 0xff);
        at[q] = 0;
#pragma unroll
        for (int i = 0; i < KP; ++i)
            if (i < k && (bk[i] & 0xff) > (en & 0xff)) ++at[q];
        on[q] = j < k && (en >> 8) >= FIRST_Q;
        zc[q] = on[q] ? fminf(zt[id[q]], FLT_MAX) : 0.f;
        if (on[q]) m = fmaxf(m, a.sigmoid ? fminf(zc[q], 0.f) : zc[q]);
    }
    float u[JN], total = 1.0f;
    if (a.renorm) {
        // ratios of scores, taken to the largest of them: scores that underflow
        // together keep their ratio
        exchanges<L>(L, [&](auto x) { m = fmaxf(m, peer_f<x.value>(m)); });
        total = 0.f;
#pragma unroll
        for (int q = 0; q < JN; ++q) {
            u[q] = 0.f;
            if (on[q])
                u[q] = a.sigmoid ? expf(fminf(zc[q], 0.f) - m) / (1.0f + expf(-fabsf(zc[q]))) : expf(zc[q] - m);
            total = total + u[q];
        }
        exchanges<L>(L, [&](auto x) { total = total + peer_f<x.value>(total); });
    } else {
#pragma unroll
        for (int q = 0; q < JN; ++q) {
            u[q] = 0.f;
            if (on[q]) u[q] = a.sigmoid ? sigmoid32(zc[q]) : expf(zc[q] - zmax) / sum;
        }
    }
#pragma unroll
    for (int q = 0; q < JN; ++q)
        if (store && q * L + sub < k) {
            topk_idx[(t0 + tok) * k + at[q]] = id[q];
            topk_w[(t0 + tok) * k + at[q]] = u[q] > 0.f ? a.scale * (u[q] / total) : 0.f;
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
// them start at a multiple of 64 bytes).  Bound by that store and the lines that
// the k logits of a row lie in: 16384 tokens to 256 experts, sigmoid, 7.3 us for
// 18 MB that a caller would count and about 25 that move; 6001 to 96, softmax, 6.8
// (8.4 with the balance read where it is compared and three passes over the row in
// LDS); a launch and its two round trips take 5.
constexpr int SB_BT = 16;
__global__ __launch_bounds__(256) void score_bwd_kernel(
        const float *__restrict__ logits, const float *__restrict__ balance,
        const int *__restrict__ topk_idx, const float *__restrict__ dw, const float *__restrict__ dgpart,
        int nparts, const int *__restrict__ route_pos, float *__restrict__ dg_out,
        float *__restrict__ dZ, int T, int E, int k, ScoreArgs a) {
    __shared__ __attribute__((aligned(16))) float row[SB_BT * 256];
    __shared__ float sbal[256];
    const int t0 = blockIdx.x * SB_BT, tl = threadIdx.x >> 4, s = threadIdx.x & 15;
    const int t = t0 + tl;
    const bool dense = !a.sigmoid && !a.renorm, slot = t < T && s < k;
    const float my_bal = balance && (int)threadIdx.x < E ? balance[threadIdx.x] : 0.f;
    const long j = (long)t * k + s;
    int e = slot ? topk_idx[j] : -1;
    float g = slot && dw ? dw[j] : 0.f;      // dL/dw of the slot
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

    if (slot && !dw) {
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
    if ((int)threadIdx.x < E) sbal[threadIdx.x] = my_bal;
    __syncthreads();
    auto live = [&](float z, int id) { return z >= MASKED && sbal[id] >= MASKED; };
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
    float x[16];                             // softmax over the row: the lane's logits, their exponentials
    if (a.renorm) {
        const float m = max16(on ? (a.sigmoid ? fminf(z, 0.f) : z) : -INFINITY);
        if (on) u = a.sigmoid ? expf(fminf(z, 0.f) - m) / (1.0f + expf(-fabsf(z))) : expf(z - m);
        const float tot = sum16(u);
        if (on) u = u / tot;
    } else if (a.sigmoid) {
        if (on) u = sigmoid32(z);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int id = s + 16 * i;
            x[i] = -INFINITY;
            if (id < E) {
                const float v = row[tl * E + id];
                if (live(v, id)) x[i] = fminf(v, FLT_MAX);
            }
            zmax = fmaxf(zmax, x[i]);
        }
        zmax = max16(zmax);
        zsum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (16 * i < E) x[i] = x[i] > -INFINITY ? expf(x[i] - zmax) : 0.f;
            if (16 * i < E) zsum = zsum + x[i];
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
#pragma unroll
        for (int i = 0; i < 16; ++i)         // (a row with nothing in play has the sum 0)
            if (s + 16 * i < E) row[tl * E + s + 16 * i] = -(x[i] > 0.f ? x[i] / zsum : 0.f) * (a.scale * dot);
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

template <int PE, int L>
hipError_t select_lanes(const float *part, int S, int epad, const float *bias, const float *balance,
                        float *logits, int *idx, float *w, int T, int E, int k, int lpg,
                        const ScoreArgs &a, hipStream_t st) {
    const long per = 256 / L;
    const dim3 grid((unsigned)((T + per - 1) / per)), block(256);
#define SELECT(KP) \
    score_select_kernel<PE, L, KP><<<grid, block, 0, st>>>(part, S, epad, bias, balance, logits, idx, w, T, E, k, \
                                                           lpg, a)
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
    // Lanes per group: as many as hold its experts, 8 each, or 16 where 8 would take
    // twice the 32 lanes (us with 8 / 16 for the whole router: 256 experts in 8
    // groups, 1 token 12.9 / 13.8; 64 experts, 512 tokens 11.6 / 13.3; 128, 8000 tokens
    // 26 / 28; 64 lanes of 8, 255 experts in 5 groups, 8000 tokens 43 / 40).
    const int n = E / a.groups, g = pow2(a.groups), wide = pow2((n + 15) / 16), narrow = pow2((n + 7) / 8);
    const int pe = g * narrow > 32 && g * wide <= 32 ? 16 : 8, lpg = pe == 16 ? wide : narrow;
#define LANES(PE, N)                                                                                       \
    case N:                                                                                                \
        return select_lanes<PE, N>(part, S, epad, bias, balance, logits, topk_idx, topk_w, T, E, k, lpg, a, \
                                   st)
    if (pe == 16) switch (g * lpg) {
        LANES(16, 32);
        default: return hipErrorInvalidValue;
    }
    switch (g * lpg) {
        LANES(8, 1);
        LANES(8, 2);
        LANES(8, 4);
        LANES(8, 8);
        LANES(8, 16);
        LANES(8, 32);
        LANES(8, 64);
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
