// Routing to a fixed number of experts, and its gradient.
//   s = softmax(z) or sigmoid(z) of a token's logits z (+inf taken as the
//   largest float); an expert whose logit or selection bias is -inf or NaN
//   takes no part.
//   c = s + sel_bias, or z itself without a selection bias (the same order).
//   Groups of E / n_groups consecutive experts: a group is worth its largest
//   c, or the sum of its two largest (of s without a bias); the top_groups
//   best groups stay.
//   Chosen: the k largest c of the groups that stay, equal ones by ascending
//   index.  w_j = scale s_j, or scale s_j / (sum of the chosen s).
//
// A token takes the 16 lanes of one DPP row, four tokens a wavefront, one
// wavefront a workgroup.  The four rows of logits are read in whole cache
// lines into LDS; a lane then holds values of one group only (16 lanes over
// the next power of two of n_groups), so a group's worth is a reduction in
// registers and over few lanes.
// c is formed in 64 bits wherever scores decide (a choice next to a border is
// that of the definition).  The k passes run on 32-bit keys: the distance from
// the row's largest c, rounded to a float, its low byte replaced by the
// expert.  Keys of other distances keep the order of c (both roundings are
// monotone); where the list has two neighbours of equal upper bits, the first
// 16 entries are put in order by their c in 64 bits, or, if that many do not
// hold every entry next to the cut, the row is chosen again from all its c.
// Weights are formed in fp32; renormalised ones from scores relative to the
// largest chosen one, so a row of scores that all underflow still has them.
// Deterministic: no floating-point atomics; a token's result does not depend
// on T.
#include <type_traits>
#include <utility>

#include "pp_select.h"

namespace pp {
namespace {

constexpr int kRowsPerWave = 4;
constexpr int kMaxGroups = 16;
constexpr int kMaxTopkRows = 1 << 22;
constexpr float kFltMax = 3.402823466e38f;

// Where a token's logits come from: an array, or the router's K-slice partial
// sums (summed in slice order, as the router's selection kernel does).
struct LogitSource {
    const float *g;       // [T][E], or NULL
    const float *gpart;   // [KSr][T][E]
    const float *bias;    // [E]
    const float *inv_temp;
    float *logits;        // [T][E] out or NULL (partial sums only)
    int KSr;
};

struct TopkParams {
    LogitSource src;
    int T, E, k, n_groups, top_groups;
    const float *sel_bias;
    float scale;
    uint32_t flags;
    int32_t *idx;
    float *w;
    // layout (topk_layout)
    int Gs;          // experts of a group
    int lanes;       // lanes of a group: 16 / (n_groups up to a power of two)
    int Gp, Rp;      // LDS floats from group to group, from row to row
    uint32_t by_Gs;  // ceil(2^16 / Gs): e / Gs = (e by_Gs) >> 16 for e < 256
};

// NaN and -inf to -inf, +inf to the largest float.
__device__ __forceinline__ float clean_logit(float z) {
    return z > -INFINITY ? fminf(z, kFltMax) : -INFINITY;
}

// ---- the 16 lanes of a DPP row
template <int CTRL>
__device__ __forceinline__ uint32_t row_u32(uint32_t v) {
    return __builtin_amdgcn_update_dpp(0u, v, CTRL, 0xF, 0xF, false);
}
template <int CTRL>
__device__ __forceinline__ float row_lane(float v) {
    return __uint_as_float(row_u32<CTRL>(__float_as_uint(v)));
}
template <int CTRL>
__device__ __forceinline__ double row_lane(double v) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    return __builtin_bit_cast(double, ((unsigned long long)row_u32<CTRL>((uint32_t)(u >> 32)) << 32) |
                                          row_u32<CTRL>((uint32_t)u));
}
// partners 1, 2, then the other half of 8 and of 16 lanes (whose values are
// equal within the half by then)
constexpr int kX1 = 0xB1, kX2 = 0x4E, kX4 = 0x141, kX8 = 0x140, kRor = 0x120;

template <typename V, typename F>
__device__ __forceinline__ V row_reduce(V v, F f) {
    v = f(v, row_lane<kX1>(v));
    v = f(v, row_lane<kX2>(v));
    v = f(v, row_lane<kX4>(v));
    return f(v, row_lane<kX8>(v));
}
__device__ __forceinline__ float row_max(float v) {
    return row_reduce(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ double row_max(double v) {
    return row_reduce(v, [](double a, double b) { return fmax(a, b); });
}
template <typename V>
__device__ __forceinline__ V row_sum(V v) {
    return row_reduce(v, [](V a, V b) { return a + b; });
}
__device__ __forceinline__ uint32_t row_min(uint32_t v) {
    v = min(v, row_u32<kX1>(v));
    v = min(v, row_u32<kX2>(v));
    v = min(v, row_u32<kX4>(v));
    return min(v, row_u32<kX8>(v));
}
// f(rotation's DPP control) for the 15 other lanes of the row
template <typename F, int... R>
__device__ __forceinline__ void rotations(F f, std::integer_sequence<int, R...>) {
    (f(std::integral_constant<int, kRor + R + 1>{}), ...);
}
template <typename F>
__device__ __forceinline__ void each_rotation(F f) {
    rotations(f, std::make_integer_sequence<int, 15>{});
}

// ---- scores
constexpr double kLn2High = 0.6931471824645996;   // ln 2 rounded to a float: n times it is exact
constexpr double kLn2Low = -1.904654299957768e-09;  // the rest
// e^x for x <= 0 in 64 bits: x = n ln 2 + r in two parts of ln 2, the Taylor
// series of e^r to r^13 / 13! (|r| <= 0.35: 3e-17 relative), times 2^n.  Below
// -746, where e^x rounds to 0, it is taken there.
__device__ __forceinline__ double exp_neg(double x) {
    x = fmax(x, -746.0);
    const double n = rint(x * 1.4426950408889634);
    double r = fma(n, -kLn2High, x);
    r = fma(n, -kLn2Low, r);
    double p = 1.0 / 6227020800.0;
    p = fma(p, r, 1.0 / 479001600.0);
    p = fma(p, r, 1.0 / 39916800.0);
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return ldexp(p, (int)n);
}
// 1 / x of a normal x of moderate size: the hardware's estimate and two Newton steps.
__device__ __forceinline__ double rcp64(double x) {
    double r = __builtin_amdgcn_rcp(x);
    r = fma(fma(-x, r, 1.0), r, r);
    return fma(fma(-x, r, 1.0), r, r);
}
__device__ __forceinline__ double sigmoid64(float z) {
    const double e = exp_neg(-fabs((double)z)), r = rcp64(1.0 + e);
    return z >= 0.0f ? r : e * r;
}
// sigmoid(z) over e^m for m = min(largest z, 0): relative scores that do not
// all underflow.
__device__ __forceinline__ float rel_sigmoid(float z, float m) {
    return expf(fminf(z, 0.0f) - m) / (1.0f + expf(-fabsf(z)));
}
__device__ __forceinline__ float exp_fast(float x) {
    return __builtin_amdgcn_exp2f(x * 1.44269504088896341f);
}

// NQ: values a lane holds.  SCORES: c is in 64 bits (a bias, or groups worth
// two scores); else c is the logit.
template <int NQ, bool SCORES>
__global__ __launch_bounds__(64) void route_topk_k(TopkParams P) {
    using C = std::conditional_t<SCORES, double, float>;
    extern __shared__ float lds[];
    float *const zs = lds;                                      // [4][Rp]
    short *const pk = reinterpret_cast<short *>(zs + 4 * P.Rp); // [4][k up to 16s]
    const int lane = threadIdx.x, c16 = lane & 15, rr = lane >> 4;
    const int E = P.E, k = P.k, t0 = (int)blockIdx.x * kRowsPerWave;
    const bool sig = (P.flags & PP_SCORE_SIGMOID) != 0;
    const bool top2 = (P.flags & PP_GROUP_TOP2) != 0;
    const bool renorm = (P.flags & PP_TOPK_RENORM) != 0;
    const int kp = (k + 15) & ~15;
    auto place = [&](int e) {
        const int g = (int)((__umul24((uint32_t)e, P.by_Gs)) >> 16);
        return g * P.Gp + e - g * P.Gs;
    };
    // the lane's group, its first value's expert and whether value q exists
    const int grp = c16 / P.lanes, sub = c16 & (P.lanes - 1);
    const bool some = grp < P.n_groups;
    auto has = [&](int q) { return some && q * P.lanes + sub < P.Gs; };
    auto expert = [&](int q) { return grp * P.Gs + q * P.lanes + sub; };
    float b[NQ];
    if (SCORES && P.sel_bias) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) b[q] = P.sel_bias[has(q) ? expert(q) : 0];
    }
    // four rows to LDS, every load issued first
    {
        float v[kRowsPerWave][kMaxExperts / 64];
        if (P.src.g) {
#pragma unroll
            for (int r = 0; r < kRowsPerWave; ++r) {
                const float *row = P.src.g + (size_t)min(t0 + r, P.T - 1) * E;
#pragma unroll
                for (int q = 0; q < kMaxExperts / 64; ++q)
                    if (64 * q < E) v[r][q] = row[min(lane + 64 * q, E - 1)];
            }
        } else {
#pragma unroll
            for (int r = 0; r < kRowsPerWave; ++r) {
                const int t = min(t0 + r, P.T - 1);
                const float it = P.src.inv_temp ? P.src.inv_temp[t] : 1.0f;
#pragma unroll
                for (int q = 0; q < kMaxExperts / 64; ++q) {
                    if (64 * q >= E) continue;
                    const int e = min(lane + 64 * q, E - 1);
                    float part[kMaxSlices];
#pragma unroll
                    for (int i = 0; i < kMaxSlices; ++i)
                        part[i] = P.src.gpart[((size_t)min(i, P.src.KSr - 1) * P.T + t) * E + e];
                    float sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < kMaxSlices; ++i)
                        if (i < P.src.KSr) sum += part[i];
                    v[r][q] = (sum + P.src.bias[e]) * it;
                    if (P.src.logits && t0 + r < P.T && lane + 64 * q < E)
                        P.src.logits[(size_t)t * E + e] = v[r][q];
                }
            }
        }
#pragma unroll
        for (int q = 0; q < kMaxExperts / 64; ++q) {
            const int e = lane + 64 * q;
            if (e >= E) continue;
            const int at = place(e);
#pragma unroll
            for (int r = 0; r < kRowsPerWave; ++r) zs[r * P.Rp + at] = clean_logit(v[r][q]);
        }
    }
    __syncthreads();
    const float *const zr = zs + rr * P.Rp;
    float z[NQ], zmax = -INFINITY;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        z[q] = zr[has(q) ? grp * P.Gp + q * P.lanes + sub : 0];
        z[q] = has(q) ? z[q] : -INFINITY;
        zmax = fmaxf(zmax, z[q]);
    }
    zmax = row_max(zmax);
    // sum of e^(z - zmax), where softmax scores are wanted
    float Sinv = 0.0f;
    double Sinv64 = 0.0;
    C c[NQ];
    if constexpr (SCORES) {
        double s[NQ], S = 0.0;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            s[q] = 0.0;
            if (sig)
                s[q] = sigmoid64(z[q] > -INFINITY ? z[q] : 0.0f);
            else if (z[q] > -INFINITY)
                s[q] = exp_neg((double)z[q] - (double)zmax);
            if (!sig) S += s[q];
        }
        if (!sig) {
            S = row_sum(S);
            Sinv64 = S > 0.0 ? rcp64(S) : 0.0;
            Sinv = (float)Sinv64;
        }
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            if (!sig) s[q] *= Sinv64;
            if (P.sel_bias) {
                b[q] = clean_logit(b[q]);
                s[q] += (double)b[q];
                c[q] = z[q] > -INFINITY && b[q] > -INFINITY ? s[q] : -INFINITY;
            } else {
                c[q] = z[q] > -INFINITY ? s[q] : -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int q = 0; q < NQ; ++q) c[q] = z[q];
        if (!sig && !renorm) {
            float S = 0.0f;
#pragma unroll
            for (int q = 0; q < NQ; ++q) S += z[q] > -INFINITY ? exp_fast(z[q] - zmax) : 0.0f;
            S = row_sum(S);
            Sinv = S > 0.0f ? 1.0f / S : 0.0f;
        }
    }
    // groups: values of those that go become -inf
    if (P.n_groups > 1) {
        C a = -INFINITY, n = -INFINITY;  // the two largest
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            n = max(n, min(a, c[q]));
            a = max(a, c[q]);
        }
        auto join = [&](C a2, C n2) {
            n = max(min(a, a2), max(n, n2));
            a = max(a, a2);
        };
        if (P.lanes > 1) join(row_lane<kX1>(a), row_lane<kX1>(n));
        if (P.lanes > 2) join(row_lane<kX2>(a), row_lane<kX2>(n));
        if (P.lanes > 4) join(row_lane<kX4>(a), row_lane<kX4>(n));
        const C v = top2 && n > -INFINITY ? a + n : a;
        int front = 0;  // lanes of better groups
        each_rotation([&](auto ctrl) {
            const C o = row_lane<decltype(ctrl)::value>(v);
            const int og = (int)row_u32<decltype(ctrl)::value>((uint32_t)grp);
            front += (o > v || (o == v && og < grp)) ? 1 : 0;
        });
        if (front >= P.top_groups * P.lanes) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) c[q] = -INFINITY;
        }
    }
    if constexpr (SCORES) {
        // without a bias the experts are in the order of the logits: scores
        // that round to the same number are not equal
        if (!P.sel_bias) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) c[q] = c[q] > -INFINITY ? (double)z[q] : -INFINITY;
        }
    }
    C cmax = -INFINITY;
#pragma unroll
    for (int q = 0; q < NQ; ++q) cmax = max(cmax, c[q]);
    cmax = row_max(cmax);
    constexpr uint32_t kNone = 0xFFFFFFFFu;
    uint32_t key[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const uint32_t d = __float_as_uint((float)(cmax - c[q]));
        key[q] = c[q] > -INFINITY ? ((d & 0xFFFFFF00u) | (uint32_t)expert(q)) : kNone;
    }
    // the next key after `last`: the smallest of key - last - 1, where keys
    // up to `last` wrap to the top
    auto next_key = [&](uint32_t last) {
        uint32_t m = kNone;
#pragma unroll
        for (int q = 0; q < NQ; ++q) m = min(m, key[q] - last - 1u);
        return row_min(m) + last + 1u;
    };
    uint32_t mine = kNone, last = kNone;
    bool close = false;  // two neighbours of the list with equal upper bits
    for (int j = 0; j < k; ++j) {
        // a list that has ended stays at kNone: the subtraction would wrap
        const bool over = j > 0 && last == kNone;
        const uint32_t n = next_key(last);
        close |= !over && n != kNone && j > 0 && ((n ^ last) < 256u);
        last = over ? kNone : n;
        mine = c16 == (j & 15) ? last : mine;
        if ((j & 15) == 15 || j == k - 1) {
            pk[rr * kp + (j & ~15) + c16] = mine == kNone ? (short)-1 : (short)(mine & 255u);
            if (j != k - 1) mine = kNone;
        }
    }
    // entries past the cut that share the upper bits of the last one
    bool full = false;
    {
        const uint32_t bucket = last;
        int m = k;
        bool more = last != kNone;
        while (true) {
            const uint32_t n = next_key(last);
            more = more && n > last && n != kNone && ((n ^ bucket) < 256u);
            if (__ballot(more) == 0ull) break;
            close |= more;
            if (m >= 16) {
                full |= more;
                break;
            }
            last = more ? n : last;
            if (more && c16 == m) mine = n;
            ++m;
        }
        full |= close && k > 16;
    }
    if (__ballot(close) != 0ull) {
        if (__ballot(full) == 0ull) {
            // up to 16 candidates, one a lane, by their c
            const bool cand = mine != kNone;
            const int e = cand ? (int)(mine & 255u) : 0;
            double v = -INFINITY;
            if (cand) {
                const float x = zr[place(e)];
                v = (double)x;
                if (SCORES && P.sel_bias) {
                    const double s = sig ? sigmoid64(x)
                                         : exp_neg((double)x - (double)zmax) * Sinv64;
                    v = s + (double)clean_logit(P.sel_bias[e]);
                }
            }
            int rank = 0;
            const uint32_t order = cand ? (uint32_t)e : 256u + (uint32_t)c16;
            each_rotation([&](auto ctrl) {
                const double o = row_lane<decltype(ctrl)::value>(v);
                const uint32_t oe = row_u32<decltype(ctrl)::value>(order);
                rank += (o > v || (o == v && oe < order)) ? 1 : 0;
            });
            if (rank < k) pk[rr * kp + rank] = cand ? (short)e : (short)-1;
        } else {
            // the row's choice from all its c
            for (int j = 0; j < k; ++j) {
                C best = -INFINITY;
                int be = 256;
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const bool up = c[q] > best;
                    best = up ? c[q] : best;
                    be = up ? expert(q) : be;
                }
                const C top = row_max(best);
                const int e = (int)row_min(best == top && top > -INFINITY ? (uint32_t)be : 256u);
                if (c16 == 0) pk[rr * kp + j] = e < 256 ? (short)e : (short)-1;
#pragma unroll
                for (int q = 0; q < NQ; ++q)
                    if (expert(q) == e && has(q)) c[q] = -INFINITY;
            }
        }
    }
    __syncthreads();
    // weights
    float m = sig ? 0.0f : zmax, scale = sig ? P.scale : P.scale * Sinv;
    if (renorm) {
        m = -INFINITY;
        for (int j = c16; j < k; j += 16) {
            const int e = pk[rr * kp + j];
            if (e >= 0) m = fmaxf(m, zr[place(e)]);
        }
        m = row_max(m);
        if (sig) m = fminf(m, 0.0f);
        float tot = 0.0f;
        for (int j = c16; j < k; j += 16) {
            const int e = pk[rr * kp + j];
            if (e >= 0) tot += sig ? rel_sigmoid(zr[place(e)], m) : expf(zr[place(e)] - m);
        }
        tot = row_sum(tot);
        scale = P.scale / tot;  // rows of empty slots do not use it
    }
    const int t = t0 + rr;
    if (t >= P.T) return;
    for (int j = c16; j < k; j += 16) {
        const int e = pk[rr * kp + j];
        float w = 0.0f;
        if (e >= 0) {
            const float x = zr[place(e)];
            w = scale * (sig ? rel_sigmoid(x, m) : expf(x - m));
        }
        P.idx[(size_t)t * k + j] = e;
        P.w[(size_t)t * k + j] = w;
    }
}

constexpr int kGradWaves = 4;  // one token each

__device__ __forceinline__ float wave_max_f32(float v) {
#pragma unroll
    for (int st = 1; st < 64; st <<= 1) v = fmaxf(v, __shfl_xor(v, st, 64));
    return v;
}
__device__ __forceinline__ float wave_sum_f32(float v) {
#pragma unroll
    for (int st = 1; st < 64; st <<= 1) v += __shfl_xor(v, st, 64);
    return v;
}

struct TopkGradParams {
    const float *g;
    int T, E, k;
    const int32_t *idx;
    const float *dw;
    float scale;
    uint32_t flags;
    float *dg;
};

// dL/dg of one token per wavefront, the chosen experts held fixed.  With
// a_j = dw_j over the slots that name an expert, q_j = w_j / scale:
//   softmax            dg_e = scale p_e ([e chosen] a_e - sum_j p_j a_j)
//   sigmoid            dg_e = scale s_e (1 - s_e) a_e
//   renormalised, D = sum_j q_j a_j:
//   softmax            dg_e = scale q_e (a_e - D)
//   sigmoid            dg_e = scale q_e (1 - s_e) (a_e - D)
__global__ __launch_bounds__(64 * kGradWaves) void route_topk_grad_k(TopkGradParams P) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int t = blockIdx.x * kGradWaves + wv;
    if (t >= P.T) return;
    const bool sig = (P.flags & PP_SCORE_SIGMOID) != 0;
    const bool renorm = (P.flags & PP_TOPK_RENORM) != 0;
    const int E = P.E;
    constexpr int NQ = kMaxExperts / 64;
    const float *row = P.g + (size_t)t * E;
    const int32_t *idx = P.idx + (size_t)t * P.k;
    const float *dw = P.dw + (size_t)t * P.k;
    float z[NQ], p[NQ], acc[NQ];
    float zmax = -INFINITY;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int e = lane + 64 * q;
        z[q] = e < E ? clean_logit(row[e]) : -INFINITY;
        zmax = fmaxf(zmax, z[q]);
        acc[q] = 0.0f;
    }
    zmax = wave_max_f32(zmax);
    float S = 0.0f;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        p[q] = z[q] > -INFINITY ? expf(z[q] - zmax) : 0.0f;
        S += p[q];
    }
    S = wave_sum_f32(S);
    // scores of the slots, relative to the largest where they are renormalised
    float m = -INFINITY;
    for (int j = 0; j < P.k; ++j) {
        const int e = idx[j];
        if ((unsigned)e < (unsigned)E) m = fmaxf(m, clean_logit(row[e]));
    }
    if (sig) m = renorm ? fminf(m, 0.0f) : 0.0f;
    if (!sig && !renorm) m = zmax;
    float tot = 0.0f, D = 0.0f;
    for (int j = 0; j < P.k; ++j) {
        const int e = idx[j];
        if ((unsigned)e >= (unsigned)E) continue;
        const float x = clean_logit(row[e]);
        if (!(x > -INFINITY)) continue;
        const float sc = sig ? rel_sigmoid(x, m) : expf(x - m);
        tot += sc;
        D += sc * dw[j];
    }
    if (!sig && !renorm) tot = S;
    const float inv = sig && !renorm ? 1.0f : (tot > 0.0f ? 1.0f / tot : 0.0f);
    D = sig && !renorm ? 0.0f : D * inv;
    for (int j = 0; j < P.k; ++j) {
        const int e = idx[j];
        if ((unsigned)e >= (unsigned)E) continue;
        const float x = clean_logit(row[e]);
        if (!(x > -INFINITY)) continue;
        const float sc = sig ? rel_sigmoid(x, m) : expf(x - m);
        float v = sc * inv * (renorm ? dw[j] - D : dw[j]);
        if (sig) v *= rel_sigmoid(-x, 0.0f);
#pragma unroll
        for (int q = 0; q < NQ; ++q) acc[q] += lane + 64 * q == e ? v : 0.0f;
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int e = lane + 64 * q;
        if (e >= E) continue;
        float v = acc[q];
        if (!sig && !renorm) v -= p[q] * inv * D;
        float *out = P.dg + (size_t)t * E + e;
        v *= P.scale;
        *out = (P.flags & PP_GRAD_ADD) ? *out + v : v;
    }
}

constexpr uint32_t kRuleFlags = PP_SCORE_SIGMOID | PP_TOPK_RENORM | PP_GROUP_TOP2;

pp_status check_rule(int32_t E, int32_t k, int32_t n_groups, int32_t top_groups,
                     const float *sel_bias, float scale, uint32_t flags, const int32_t *idx,
                     const float *w) {
    if (!idx || !w || (const void *)idx == (const void *)w) return PP_EINVAL;
    if (((uintptr_t)idx | (uintptr_t)w | (uintptr_t)sel_bias) & 3) return PP_EINVAL;
    if (flags & ~kRuleFlags) return PP_EINVAL;
    if (!(fabsf(scale) <= 3.0e38f)) return PP_EINVAL;  // also rejects NaN
    if (n_groups < 1 || E % n_groups != 0 || top_groups < 1 || top_groups > n_groups)
        return PP_EINVAL;
    if (k < 1 || k > top_groups * (E / n_groups)) return PP_EINVAL;
    if (n_groups > kMaxGroups) return PP_EUNSUPPORTED;
    return PP_OK;
}

// Values a lane holds of E experts in n_groups groups: 16 for 256 experts in
// one group, at most 28 (nine groups of 28 on a lane each).
constexpr int kLaneValues[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 28};

template <int NQ>
void launch_topk_nq(const TopkParams &P, bool scores, size_t lds, hipStream_t s) {
    const dim3 grid((P.T + kRowsPerWave - 1) / kRowsPerWave);
    if (scores)
        hipLaunchKernelGGL((route_topk_k<NQ, true>), grid, dim3(64), lds, s, P);
    else
        hipLaunchKernelGGL((route_topk_k<NQ, false>), grid, dim3(64), lds, s, P);
}
template <int... I>
bool launch_topk_for(int need, const TopkParams &P, bool scores, size_t lds, hipStream_t s,
                     std::integer_sequence<int, I...>) {
    return (... || (need <= kLaneValues[I]
                        ? (launch_topk_nq<kLaneValues[I]>(P, scores, lds, s), true)
                        : false));
}

hipError_t launch_topk(TopkParams P, hipStream_t s) {
    int p2 = 1;
    while (p2 < P.n_groups) p2 *= 2;
    P.Gs = P.E / P.n_groups;
    P.lanes = 16 / p2;
    // a group starts `lanes` banks after the one before, so that the 16 lanes
    // of a row read 16 different banks; one group: rows 16 banks apart
    P.Gp = (P.Gs + 31) / 32 * 32 + P.lanes;
    P.Rp = p2 * P.Gp;
    P.by_Gs = (uint32_t)((65536 + P.Gs - 1) / P.Gs);
    const bool scores = P.sel_bias || (P.n_groups > 1 && (P.flags & PP_GROUP_TOP2));
    const size_t lds = sizeof(float) * 4 * P.Rp + sizeof(short) * 4 * ((P.k + 15) & ~15);
    constexpr int n = sizeof(kLaneValues) / sizeof(kLaneValues[0]);
    if (!launch_topk_for((P.Gs + P.lanes - 1) / P.lanes, P, scores, lds, s,
                         std::make_integer_sequence<int, n>{}))
        return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" pp_status prunepath_route_topk(pp_layer *L, const uint16_t *x, int32_t T,
                                          const float *inv_temp, int32_t k, int32_t n_groups,
                                          int32_t top_groups, const float *sel_bias, float scale,
                                          uint32_t flags, int32_t *expert_idx, float *gate_w,
                                          float *logits, void *hip_stream) {
    if (!L || !x || T < 1 || T > L->max_tokens) return PP_EINVAL;
    if ((uintptr_t)logits & 3) return PP_EINVAL;
    const int E = L->dm.E;
    const pp_status st =
        check_rule(E, k, n_groups, top_groups, sel_bias, scale, flags, expert_idx, gate_w);
    if (st != PP_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    // the partial logits of the handle's router, in its scratch
    hipError_t e = launch_route(L, x, T, 0.0f, inv_temp, nullptr, nullptr, nullptr, false, s, false);
    if (e == hipSuccess) {
        const RouteParams R = route_params(L, x, T, 0.0f, inv_temp, nullptr, nullptr, nullptr, false);
        const TopkParams P = {{nullptr, R.gpart, R.bias, inv_temp, logits, R.KSr}, T, E, k, n_groups,
                              top_groups, sel_bias, scale, flags, expert_idx, gate_w, 0, 0, 0, 0, 0};
        prof_mark(L, PP_KERNEL_ROUTE, s, true);
        e = launch_topk(P, s);
        prof_mark(L, PP_KERNEL_ROUTE, s, false);
    }
    return e == hipSuccess ? PP_OK : PP_EHIP;
}

extern "C" pp_status prunepath_route_topk_logits(const float *g, int32_t T, int32_t E, int32_t k,
                                                 int32_t n_groups, int32_t top_groups,
                                                 const float *sel_bias, float scale,
                                                 uint32_t flags, int32_t *expert_idx,
                                                 float *gate_w, void *hip_stream) {
    if (!g || ((uintptr_t)g & 3) || T < 1 || T > kMaxTopkRows || E < 1 || E > kMaxExperts)
        return PP_EINVAL;
    const pp_status st =
        check_rule(E, k, n_groups, top_groups, sel_bias, scale, flags, expert_idx, gate_w);
    if (st != PP_OK) return st;
    const TopkParams P = {{g, nullptr, nullptr, nullptr, nullptr, 0}, T, E, k, n_groups, top_groups,
                          sel_bias, scale, flags, expert_idx, gate_w, 0, 0, 0, 0, 0};
    return launch_topk(P, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? PP_OK : PP_EHIP;
}

extern "C" pp_status prunepath_route_topk_grad(const float *g, int32_t T, int32_t E, int32_t k,
                                               const int32_t *expert_idx, const float *dgate_w,
                                               float scale, uint32_t flags, float *dg,
                                               void *hip_stream) {
    if (!g || !expert_idx || !dgate_w || !dg || dg == g || dg == dgate_w ||
        (void *)dg == (void *)expert_idx)
        return PP_EINVAL;
    if (((uintptr_t)g | (uintptr_t)expert_idx | (uintptr_t)dgate_w | (uintptr_t)dg) & 3)
        return PP_EINVAL;
    if (T < 1 || T > kMaxTopkRows || E < 1 || E > kMaxExperts || k < 1 || k > E) return PP_EINVAL;
    if (flags & ~(kRuleFlags | PP_GRAD_ADD)) return PP_EINVAL;
    if (!(fabsf(scale) <= 3.0e38f)) return PP_EINVAL;
    const TopkGradParams P = {g, T, E, k, expert_idx, dgate_w, scale, flags, dg};
    hipLaunchKernelGGL(route_topk_grad_k, dim3((T + kGradWaves - 1) / kGradWaves),
                       dim3(64 * kGradWaves), 0, static_cast<hipStream_t>(hip_stream), P);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_EHIP;
}
