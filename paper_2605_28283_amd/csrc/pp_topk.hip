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
// A token takes the 16 lanes of one DPP row, four tokens a wavefront.  The
// rows of logits (and the bias) are read in whole cache lines into LDS; a lane
// then holds values of one group only (16 lanes over the next power of two of
// n_groups), so a group's worth is a reduction in registers and over few lanes.
// The k passes run on 32-bit keys: half the distance from the row's largest c,
// its low byte replaced by the expert, so that one unsigned minimum gives value
// and index.  Scores are formed in 32 bits for that, within a stated error;
// what they leave open is decided in 64 bits by the whole wavefront: groups
// too near each other (exact_groups), neighbours of the list too near each
// other or to what was left out (the list, with all that may belong in it, is
// sorted by exact c: sort_list), and rows where that is more than 64 entries
// (choose_row).  So c is compared in 64 bits wherever it matters.  Few tokens
// pay for it while the biases are of the scores' size: the error of every c is
// taken from the largest |bias| of an expert that takes part, so a single
// finite one of -1e4 or -1e9 (a mask; -inf costs nothing) makes more or all
// rows open, 12.4 us below to 26 and 81.
// Neither memory nor one unit bounds it: 16384 tokens of 256 experts, 8 groups,
// k 8, sigmoid plus a bias take 13.4 us (12.4 among captured calls) for 17.8
// MB.  1109 vector instructions a wavefront, of which the nine passes are a
// third, issue for about 7.5 us; all wavefronts are resident at once and wait
// for half of their cycles, in the loads, the LDS round trips and the exact
// tails.  Every score in 64 bits took 28.8 us, an argmax over 64-bit values 50.7.
// Weights are formed in fp32; renormalised ones from scores relative to the
// largest chosen one, so a row of scores that all underflow still has them.
// Relative error (24 + |x|) 2^-23 with x the argument of the weight's
// exponential, of which 20 2^-23 are a plain softmax weight's sum (kSoftmaxErr).
// Deterministic: no floating-point atomics; a token's result does not depend
// on T.
#include <type_traits>
#include <utility>

#include "pp_select.h"

namespace pp {
namespace {

constexpr int kRowsPerWave = 4;
constexpr int kTopkWaves = 4;    // of a workgroup (single ones are not dispatched fast enough)
constexpr int kMaxGroups = 16;
constexpr int kMaxList = 64;     // entries put in order in 64 bits
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
    int lanes_log;
    int Gp, Rp;      // LDS floats from group to group, from row to row
    uint32_t by_Gs;  // ceil(2^16 / Gs): e / Gs = (e by_Gs) >> 16 for e < 256
    int pad;         // whether lanes read places without an expert
    int kp;          // list entries of a row in LDS: k, and room to kMaxList
    int wave_lds;    // floats of a wavefront
};

// NaN and -inf to -inf, +inf to the largest float.
__device__ __forceinline__ float clean_logit(float z) {
    return fminf(fmaxf(z, -INFINITY), kFltMax);
}
// Maximum and minimum of numbers without the quieting of NaNs that fmaxf and
// fminf are compiled to: medians with an infinity, which must not be known as
// one (else they are turned back).
struct NumExtremes {
    float inf = INFINITY;
    __device__ __forceinline__ NumExtremes() { asm("" : "+s"(inf)); }
    __device__ __forceinline__ float max(float a, float b) const {
        return __builtin_amdgcn_fmed3f(a, b, inf);
    }
    __device__ __forceinline__ float min(float a, float b) const {
        return __builtin_amdgcn_fmed3f(a, b, -inf);
    }
};

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
// Floats in the order of signed integers (its own inverse).
__device__ __forceinline__ int ordered_bits(int u) { return u ^ ((u >> 31) & 0x7FFFFFFF); }
__device__ __forceinline__ float row_max(float v) {
    int m = ordered_bits(__float_as_int(v));
    m = max(m, (int)row_u32<kX1>((uint32_t)m));
    m = max(m, (int)row_u32<kX2>((uint32_t)m));
    m = max(m, (int)row_u32<kX4>((uint32_t)m));
    m = max(m, (int)row_u32<kX8>((uint32_t)m));
    return __int_as_float(ordered_bits(m));
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
// A score and c in 64 bits, each step rounded (no product is fused into a sum),
// from 1 / (sum of e^(z - zmax)) in the order of exact_softmax_scale:
// the same bits wherever they are formed, so that c's next to each other are
// in one order in every kernel.
__device__ __forceinline__ double score64(bool sig, float z, float zmax, double scale) {
#pragma clang fp contract(off)
    return sig ? sigmoid64(z) : exp_neg((double)z - (double)zmax) * scale;
}
__device__ __forceinline__ double biased64(double s, float b) {
#pragma clang fp contract(off)
    return s + (double)b;
}
// sigmoid(z) over e^m for m = min(largest z, 0): relative scores that do not
// all underflow.
__device__ __forceinline__ float rel_sigmoid(float z, float m) {
    return expf(fminf(z, 0.0f) - m) / (1.0f + expf(-fabsf(z)));
}
// e^x with the hardware's exponential (1 ulp of a rounded product).
__device__ __forceinline__ float exp_fast(float x) {
    return __builtin_amdgcn_exp2f(x * 1.44269504088896341f);
}
// sigmoid(z) within 4e-7: e = e^-z is off by e (|z| 2^-23 + 2^-22) (the product
// with log2 e, the exponential), of which s^2 counts, at most 2.9e-7 for
// either sign of z; 1 + e and its reciprocal add (2^-24 + 2^-23) s.
constexpr float kScoreErr = 6e-7f;
// Softmax scores p = e / S: e^-x is off by e (x 2^-22.5 + 2^-22) < 3.1e-7 (also
// x = zmax - z was rounded); S, at least 1, by the mean of that over p, in
// which x averages to at most log 256 (an entropy), and by 20 roundings:
// 2.5e-6 relative.
constexpr float kSoftmaxErr = 3.2e-6f;
__device__ __forceinline__ float sigmoid_fast(float z) {
    return __builtin_amdgcn_rcpf(1.0f + exp_fast(-z));
}

// Largest and smallest over the wavefront, sum over it.
template <typename F>
__device__ __forceinline__ double wave_reduce(double v, int lane, F f) {
    auto step = [&](auto st) {
        constexpr int ST = decltype(st)::value;
        const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
        const unsigned long long o =
            ((unsigned long long)xor_lane<ST>((uint32_t)(u >> 32), lane) << 32) |
            xor_lane<ST>((uint32_t)u, lane);
        v = f(v, __builtin_bit_cast(double, o));
    };
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 4>{});
    step(std::integral_constant<int, 8>{});
    step(std::integral_constant<int, 16>{});
    step(std::integral_constant<int, 32>{});
    return v;
}
__device__ __forceinline__ uint32_t wave_min_u32(uint32_t v, int lane) {
    v = min(v, xor_lane<1>(v, lane));
    v = min(v, xor_lane<2>(v, lane));
    v = min(v, xor_lane<4>(v, lane));
    v = min(v, xor_lane<8>(v, lane));
    v = min(v, xor_lane<16>(v, lane));
    return min(v, xor_lane<32>(v, lane));
}

// A wavefront's LDS is its own: its operations on it are carried out in order,
// and this keeps the compiler from changing that order.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Logit of token t and expert e, from the router's partial sums (and stored
// for the caller, if it wants them).
__device__ __forceinline__ float summed_logit(const TopkParams &P, int t, int e, bool store) {
    const float *p = P.src.gpart + (size_t)t * P.E + e;
    const size_t slice = (size_t)P.T * P.E;
    float part[kMaxSlices];
#pragma unroll
    for (int i = 0; i < kMaxSlices; ++i) part[i] = p[min(i, P.src.KSr - 1) * slice];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kMaxSlices; ++i)
        if (i < P.src.KSr) sum += part[i];
    const float z = (sum + P.src.bias[e]) * (P.src.inv_temp ? P.src.inv_temp[t] : 1.0f);
    if (P.src.logits && store) P.src.logits[(size_t)t * P.E + e] = z;
    return z;
}

// e's place in a row in LDS.
__device__ __forceinline__ int topk_place(const TopkParams &P, int e) {
    const int g = (int)(__umul24((uint32_t)e, P.by_Gs) >> 16);
    return g * P.Gp + e - g * P.Gs;
}

// With the groups spread over 64 lanes (group lane >> (lanes_log + 2)): how
// many groups are in front of the lane's, whose lanes hold its values' two
// largest (a, n) among them.
__device__ __forceinline__ int groups_in_front(const TopkParams &P, double a, double n, int lane) {
    const int wl = P.lanes_log + 2;
    auto join = [&](auto st) {
        constexpr int ST = decltype(st)::value;
        if ((1 << wl) <= ST) return;
        auto other = [&](double v) {
            const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
            return __builtin_bit_cast(
                double, ((unsigned long long)xor_lane<ST>((uint32_t)(u >> 32), lane) << 32) |
                            xor_lane<ST>((uint32_t)u, lane));
        };
        const double a2 = other(a), n2 = other(n);
        n = fmax(fmin(a, a2), fmax(n, n2));
        a = fmax(a, a2);
    };
    join(std::integral_constant<int, 1>{});
    join(std::integral_constant<int, 2>{});
    join(std::integral_constant<int, 4>{});
    join(std::integral_constant<int, 8>{});
    join(std::integral_constant<int, 16>{});
    const double v = (P.flags & PP_GROUP_TOP2) && n > -INFINITY ? a + n : a;
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    int front = 0;
#pragma unroll 1
    for (int g = 0; g < P.n_groups; ++g) {
        const unsigned long long ou =
            ((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), g << wl)
             << 32) | (uint32_t)__builtin_amdgcn_readlane((int)u, g << wl);
        const double o = __builtin_bit_cast(double, ou);
        front += o > v || (o == v && g < lane >> wl) ? 1 : 0;
    }
    return front;
}

// 1 / (sum of e^(z - zmax)) of a row in 64 bits, by the whole wavefront, in the
// order of route_topk_wide_k: groups spread over the lanes as for
// groups_in_front, a lane's values, then pairs of lanes.
__device__ __forceinline__ double exact_softmax_scale(const TopkParams &P, const float *zr,
                                                      float zmax, int lane) {
    const int wl = P.lanes_log + 2, grp = lane >> wl;
    double S = 0.0;
    if (grp < P.n_groups) {
#pragma unroll 1
        for (int i = lane & ((1 << wl) - 1); i < P.Gs; i += 1 << wl) {
            const float z = zr[grp * P.Gp + i];
            if (z > -INFINITY) S += exp_neg((double)z - (double)zmax);
        }
    }
    S = wave_reduce(S, lane, [](double a, double b) { return a + b; });
    return S > 0.0 ? rcp64(S) : 0.0;
}

// The groups of a row that stay, by scores in 64 bits: bit g << (lanes_log + 2)
// for group g.  For a call with a bias, or worth two scores without one.
// zr, zb: the row and the bias.
__device__ __forceinline__ unsigned long long exact_groups(const TopkParams &P, const float *zr,
                                                           const float *zb, float zmax,
                                                           double scale, int lane) {
    const int wl = P.lanes_log + 2, grp = lane >> wl;
    const bool sig = (P.flags & PP_SCORE_SIGMOID) != 0;
    double a = -INFINITY, n = -INFINITY;
    if (grp < P.n_groups) {
#pragma unroll 1
        for (int i = lane & ((1 << wl) - 1); i < P.Gs; i += 1 << wl) {
            const float z = zr[grp * P.Gp + i];
            const float b = P.sel_bias ? zb[grp * P.Gp + i] : 0.0f;
            const double v = biased64(score64(sig, z, zmax, scale), b);
            if (z > -INFINITY && b > -INFINITY) {
                n = fmax(n, fmin(a, v));
                a = fmax(a, v);
            }
        }
    }
    return __ballot(groups_in_front(P, a, n, lane) < P.top_groups);
}

// Puts the n <= 64 listed experts in order of c (equal ones by index), of
// which the first k are kept.
__device__ __forceinline__ void sort_list(const double *c, short *list, int n, int k, int lane) {
    wave_sync();
    const int e = list[min(lane, n - 1)];
    const double v = c[e];
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) {
        const int oe = list[j];
        const double o = c[oe];
        rank += o > v || (o == v && oe < e) ? 1 : 0;
    }
    wave_sync();
    if (lane < n && rank < k) list[rank] = (short)e;
    wave_sync();
}

// One row's choice, all of it in 64 bits, by the whole wavefront: lane l has
// experts l, l + 64, ...  zr, zb: the row and the bias in LDS; zmax: the row's
// largest logit; worth: 256 doubles of LDS; out: [k].
__device__ __forceinline__ void choose_row(const TopkParams &P, const float *zr, const float *zb,
                                           float zmax, double *worth, short *out, int lane) {
    constexpr int NE = kMaxExperts / 64;
    const bool sig = (P.flags & PP_SCORE_SIGMOID) != 0;
    const bool top2 = (P.flags & PP_GROUP_TOP2) != 0;
    const double scale = sig ? 1.0 : exact_softmax_scale(P, zr, zmax, lane);
    double c[NE], s[NE];
#pragma unroll
    for (int q = 0; q < NE; ++q) {
        const int e = lane + 64 * q;
        const float z = e < P.E ? zr[topk_place(P, e)] : -INFINITY;
        c[q] = (double)z;
        s[q] = 0.0;
        if (z > -INFINITY) s[q] = score64(sig, z, zmax, scale);
    }
#pragma unroll
    for (int q = 0; q < NE; ++q) {
        const int e = lane + 64 * q;
        if (P.sel_bias) {
            const float b = e < P.E ? zb[topk_place(P, e)] : -INFINITY;
            const double v = biased64(s[q], b);
            c[q] = c[q] > -INFINITY && b > -INFINITY ? v : -INFINITY;
        }
        // without a bias experts are in the order of the logits
        if (P.n_groups > 1)
            worth[e] = top2 && !P.sel_bias && c[q] > -INFINITY ? s[q] : c[q];
    }
    if (P.n_groups > 1) {
        wave_sync();
        double a = -INFINITY, n = -INFINITY;
        if (lane < P.n_groups) {
#pragma unroll 4
            for (int i = 0; i < P.Gs; ++i) {
                const double v = worth[lane * P.Gs + i];
                n = fmax(n, fmin(a, v));
                a = fmax(a, v);
            }
            if (top2 && n > -INFINITY) a += n;
        }
        wave_sync();
        worth[lane] = a;
        wave_sync();
        int front = 0;
#pragma unroll 1
        for (int g = 0; g < P.n_groups; ++g) {
            const double o = worth[g];
            front += o > a || (o == a && g < lane) ? 1 : 0;
        }
        const unsigned long long stay = __ballot(front < P.top_groups && lane < P.n_groups);
        wave_sync();  // worth is free again
#pragma unroll
        for (int q = 0; q < NE; ++q) {
            const int g = (int)(__umul24((uint32_t)(lane + 64 * q), P.by_Gs) >> 16);
            if (!((stay >> (g & 63)) & 1ull)) c[q] = -INFINITY;
        }
    }
#pragma unroll 1
    for (int j = 0; j < P.k; ++j) {
        double best = -INFINITY;
        uint32_t be = 256u;
#pragma unroll
        for (int q = 0; q < NE; ++q) {
            const bool up = c[q] > best;
            best = up ? c[q] : best;
            be = up ? (uint32_t)(lane + 64 * q) : be;
        }
        const double top =
            wave_reduce(best, lane, [](double a, double b) { return fmax(a, b); });
        const uint32_t e = wave_min_u32(best == top ? be : 256u, lane);
        if (lane == 0) out[j] = e < 256u ? (short)e : (short)-1;
#pragma unroll
        for (int q = 0; q < NE; ++q)
            if ((uint32_t)(lane + 64 * q) == e) c[q] = -INFINITY;
    }
}

// Weights of a row's choice, by W lanes, and the choice itself.  zr: the row
// in LDS; zmax: its largest logit; Sinv: 1 / (sum of e^(z - zmax)).
template <int W>
__device__ __forceinline__ void store_row(const TopkParams &P, const float *zr, float zmax,
                                          float Sinv, const short *list, int t, int l) {
    const bool sig = (P.flags & PP_SCORE_SIGMOID) != 0;
    const int k = P.k;
    float m = sig ? 0.0f : zmax, scale = sig ? P.scale : P.scale * Sinv;
    if (P.flags & PP_TOPK_RENORM) {
        m = -INFINITY;
        for (int j = l; j < k; j += W) {
            const int e = list[j];
            if (e >= 0) m = fmaxf(m, zr[topk_place(P, e)]);
        }
        m = row_max(m);
        if (W == 64) {
            m = fmaxf(m, __uint_as_float(xor_lane<16>(__float_as_uint(m), l)));
            m = fmaxf(m, __uint_as_float(xor_lane<32>(__float_as_uint(m), l)));
        }
        if (sig) m = fminf(m, 0.0f);
        float tot = 0.0f;
        for (int j = l & 15; j < k; j += 16) {
            const int e = list[j];
            if (e >= 0) {
                const float x = zr[topk_place(P, e)];
                tot += sig ? rel_sigmoid(x, m) : expf(x - m);
            }
        }
        // every 16 lanes take all slots, in the same order for either W.  Over
        // twice the sum (which is 1/2 or more), and scores twice below: a scale
        // near the largest float stays one.  Rows of empty slots do not use it.
        scale = P.scale / (2.0f * row_sum(tot));
    }
    for (int j = l; j < k; j += W) {
        const int e = list[j];
        float w = 0.0f;
        if (e >= 0) {
            const float x = zr[topk_place(P, e)];
            w = sig ? rel_sigmoid(x, m) : expf(x - m);
            // (the quotient's rounding alone may pass the largest float)
            w = P.flags & PP_TOPK_RENORM
                    ? __builtin_amdgcn_fmed3f(scale * (2.0f * w), -kFltMax, kFltMax)
                    : scale * w;
        }
        P.idx[(size_t)t * k + j] = e;
        P.w[(size_t)t * k + j] = w;
    }
}

// NQ: values a lane holds.  SCORES: scores decide (a bias, or groups worth two
// scores); else c is the logit and needs no 64 bits.
template <int NQ, bool SCORES>
__global__ __launch_bounds__(64 * kTopkWaves) void route_topk_k(TopkParams P) {
    extern __shared__ __align__(16) float all_lds[];
    float *const lds = all_lds + (threadIdx.x >> 6) * P.wave_lds;
    double *const worth = reinterpret_cast<double *>(lds);   // [256]
    float *const zs = lds + 2 * kMaxExperts;                  // [4][Rp], -inf where no expert is
    float *const zb = zs + kRowsPerWave * P.Rp;               // [Rp], the selection bias
    short *const pk = reinterpret_cast<short *>(zb + (SCORES ? P.Rp : 0));  // [4][kp]
    const int lane = threadIdx.x & 63, c16 = lane & 15, rr = lane >> 4;
    const int E = P.E, k = P.k;
    const int t0 = __builtin_amdgcn_readfirstlane(
        (int)(blockIdx.x * kTopkWaves + (threadIdx.x >> 6)) * kRowsPerWave);
    if (t0 >= P.T) return;
    const bool sig = (P.flags & PP_SCORE_SIGMOID) != 0;
    const bool top2 = (P.flags & PP_GROUP_TOP2) != 0;
    const bool renorm = (P.flags & PP_TOPK_RENORM) != 0;
    const bool biased = SCORES && P.sel_bias;
    const int kp = P.kp;
    constexpr int NE = kMaxExperts / 64;
    if (P.pad) {
        const int n4 = (kRowsPerWave + (SCORES ? 1 : 0)) * P.Rp / 4;
        for (int i = lane; i < n4; i += 64)
            reinterpret_cast<float4 *>(zs)[i] =
                make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    }
    float big = 0.0f;  // largest |bias|
    // the bias and four rows to LDS, every load issued first
    if (P.src.g) {
        float v[kRowsPerWave + 1][NE];
        if (biased) {
#pragma unroll
            for (int q = 0; q < NE; ++q) v[kRowsPerWave][q] = P.sel_bias[min(lane + 64 * q, E - 1)];
        }
#pragma unroll
        for (int r = 0; r < kRowsPerWave; ++r) {
            const float *row = P.src.g + (size_t)min(t0 + r, P.T - 1) * E;
#pragma unroll
            for (int q = 0; q < NE; ++q) v[r][q] = row[min(lane + 64 * q, E - 1)];
        }
#pragma unroll
        for (int q = 0; q < NE; ++q) {
            const int e = lane + 64 * q;
            if (e >= E) break;
            const int at = topk_place(P, e);
#pragma unroll
            for (int r = 0; r < kRowsPerWave; ++r) zs[r * P.Rp + at] = clean_logit(v[r][q]);
            if (biased) {
                const float b = clean_logit(v[kRowsPerWave][q]);
                zb[at] = b;
                big = b > -INFINITY ? fmaxf(big, fabsf(b)) : big;
            }
        }
    } else {
#pragma unroll 1
        for (int e = lane; e < E; e += 64) {
            const int at = topk_place(P, e);
            if (biased) {
                const float b = clean_logit(P.sel_bias[e]);
                zb[at] = b;
                big = b > -INFINITY ? fmaxf(big, fabsf(b)) : big;
            }
#pragma unroll 1
            for (int r = 0; r < kRowsPerWave; ++r)
                zs[r * P.Rp + at] =
                    clean_logit(summed_logit(P, min(t0 + r, P.T - 1), e, t0 + r < P.T));
        }
    }
    wave_sync();
    const float *const zr = zs + rr * P.Rp;
    // the lane's group and its first value
    const int grp = c16 >> P.lanes_log, sub = c16 & (P.lanes - 1);
    const float *const mz = zr + grp * P.Gp + sub;
    const NumExtremes num;
    float c[NQ], zmax = 0.0f;
#pragma unroll
    for (int q = 0; q < NQ; ++q) c[q] = mz[q * P.lanes];
    // softmax: the row's largest logit, and 1 / sum of e^(z - zmax) where
    // weights are wanted as they are
    float Sinv = 0.0f;
    if (!sig) {
        zmax = c[0];
#pragma unroll
        for (int q = 1; q < NQ; ++q) zmax = num.max(zmax, c[q]);
        zmax = row_max(zmax);
        if (!renorm || biased) {
            float S = 0.0f;
#pragma unroll
            for (int q = 0; q < NQ; ++q) S += exp_fast(c[q] - zmax);
            Sinv = 1.0f / row_sum(S);  // a row of no experts has no weights
        }
    }
    bool unsure = false;  // whether 32 bits do not make the choice
    float err = 0.0f;     // of c
    if constexpr (SCORES) {
        // the score's error and the rounding of the sum with the bias
        if (biased) {
#pragma unroll
            for (int st = 1; st < 64; st <<= 1)
                big = fmaxf(big, __uint_as_float(xor_lane_rt(__float_as_uint(big), st, lane)));
        }
        err = (biased && !sig ? kSoftmaxErr : kScoreErr) + (1.0f + big) * 2.4e-7f;
        // (an expert that takes no part has a score of 0 here)
        float s[NQ];
        if (sig) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) s[q] = sigmoid_fast(c[q]);
        } else {
#pragma unroll
            for (int q = 0; q < NQ; ++q) s[q] = exp_fast(c[q] - zmax);
            if (biased) {
#pragma unroll
                for (int q = 0; q < NQ; ++q) s[q] *= Sinv;
            }
        }
        if (biased) {
            const float *const mb = zb + grp * P.Gp + sub;
#pragma unroll
            for (int q = 0; q < NQ; ++q) s[q] += mb[q * P.lanes];  // -inf: takes no part
        }
#pragma unroll
        for (int q = 0; q < NQ; ++q) c[q] = c[q] > -INFINITY ? s[q] : -INFINITY;
    }
    // the groups that stay
    bool out = false;
    if (P.n_groups > 1) {
        float a = c[0], n = -INFINITY;  // the two largest
#pragma unroll
        for (int q = 1; q < NQ; ++q) {
            n = __builtin_amdgcn_fmed3f(n, a, c[q]);  // n <= a: the middle one
            a = num.max(a, c[q]);
        }
        auto join = [&](float a2, float n2) {
            n = num.max(num.min(a, a2), num.max(n, n2));
            a = num.max(a, a2);
        };
        if (P.lanes > 1) join(row_lane<kX1>(a), row_lane<kX1>(n));
        if (P.lanes > 2) join(row_lane<kX2>(a), row_lane<kX2>(n));
        if (P.lanes > 4) join(row_lane<kX4>(a), row_lane<kX4>(n));
        // worths of two scores are halved (the sum of two floats may be past the
        // largest): -inf is a group of no experts and nothing else
        const float v = top2 ? fmaf(0.5f, n > -INFINITY ? n : 0.0f, 0.5f * a) : a;
        // groups in front, and those that might be if each worth is off by
        // what its two scores and their sum are
        const float off = SCORES ? (top2 ? 1.5f : 3.0f) * err : 0.0f;
        int front = 0, near = 0;
        each_rotation([&](auto ctrl) {
            constexpr int R = decltype(ctrl)::value & 15;
            if ((R & (P.lanes - 1)) != 0) return;  // from group to group
            const float o = row_lane<decltype(ctrl)::value>(v);
            if constexpr (SCORES) {
                front += o > v + off ? 1 : 0;
                near += o >= v - off ? 1 : 0;
            } else {
                const bool before = c16 >= R;  // lane c reads lane c - R, or c - R + 16
                front += o > v || (o == v && before) ? 1 : 0;
            }
        });
        out = front >= P.top_groups;
        if constexpr (SCORES) {
            const unsigned long long open =
                __ballot(v > -INFINITY && front < P.top_groups && near >= P.top_groups);
            if (open != 0ull) {
#pragma unroll 1
                for (int r = 0; r < kRowsPerWave; ++r) {
                    if (!((open >> (16 * r)) & 0xFFFFull)) continue;
                    const float top = __shfl(zmax, 16 * r, 64);
                    const double scale =
                        sig ? 1.0 : exact_softmax_scale(P, zs + r * P.Rp, top, lane);
                    const unsigned long long stay =
                        exact_groups(P, zs + r * P.Rp, zb, top, scale, lane);
                    if (rr == r) out = !((stay >> (grp << (P.lanes_log + 2))) & 1ull);
                }
            }
        }
    }
    if (SCORES && !biased) {  // then experts are in the order of the logits
        err = 0.0f;
#pragma unroll
        for (int q = 0; q < NQ; ++q) c[q] = mz[q * P.lanes];
    }
    // Keys: half the distance (which no two floats overflow) from the largest
    // c of the groups that stay; infinite for what is not there.
    constexpr uint32_t kNone = 0xFFFFFFFFu, kFirstNone = 0x7F800000u;
    uint32_t key[NQ];
    {
        float cmax = c[0];
#pragma unroll
        for (int q = 1; q < NQ; ++q) cmax = num.max(cmax, c[q]);
        // (the smallest float on top: half of an odd subnormal is not rounded
        // down, which would make a distance negative)
        const float half = fmaf(0.5f, row_max(out ? -INFINITY : cmax), 1.4e-45f);
        const float from = out ? INFINITY : half;
        uint32_t e = (uint32_t)(grp * P.Gs + sub);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            key[q] = (__float_as_uint(fmaf(c[q], -0.5f, from)) & 0xFFFFFF00u) | e;
            e += (uint32_t)P.lanes;
        }
    }
    // the next key after `last`: the smallest of key - last - 1, where keys
    // up to `last` wrap to the top
    auto next_key = [&](uint32_t last) {
        uint32_t m = key[0] + ~last;
#pragma unroll
        for (int q = 1; q < NQ; ++q) m = min(m, key[q] + ~last);
        return row_min(m) + last + 1u;
    };
    // A key's distance, and up to which one an entry may belong in front of
    // it: where c is exact, one of the same upper bits; else 2^-15 of each was
    // cut off, and c is off by err (halved like it).
    const float grow = err > 0.0f ? 1.00004f : 1.0f;
    auto distance = [](uint32_t v) { return __uint_as_float(v & 0xFFFFFF00u); };
    uint32_t last = kNone;
    float reach = 0.0f;
    bool close = false;  // whether the list's order may not be that of c
    bool more = true;    // whether the list goes on
    int len = 0;         // of the row's list
#pragma unroll 1
    for (int j = 0; j < k; ++j) {
        const uint32_t n = next_key(last);
        more = more && n < kFirstNone;
        const float d = distance(n);
        close |= more && j > 0 && d <= reach;
        reach = fmaf(d, grow, err);
        last = n;  // past the list's end: not used any more
        len += more ? 1 : 0;
        if (c16 == 0) pk[rr * kp + j] = more ? (short)(n & 255u) : (short)-1;
    }
    // entries past the cut that may belong in front of it
    for (int m = k;; ++m) {
        const uint32_t n = next_key(last);
        more = more && n > last && n < kFirstNone && distance(n) <= reach;
        if (__ballot(more) == 0ull) break;
        close |= more;
        if (m >= kMaxList) {
            unsure |= more;
            break;
        }
        if (more) {
            last = n;
            if (c16 == 0) pk[rr * kp + m] = (short)(n & 255u);
            ++len;
        }
    }
    unsure |= close && k > kMaxList;
    wave_sync();
    // rows whose list is put in order by c in 64 bits
    const unsigned long long sort = __ballot(close && !unsure);
    if (sort != 0ull) {
#pragma unroll 1
        for (int r = 0; r < kRowsPerWave; ++r) {
            if (!((sort >> (16 * r)) & 1ull)) continue;
            const int n = __builtin_amdgcn_readlane(len, 16 * r);
            const float top = __shfl(zmax, 16 * r, 64);
            double scale = 1.0;
            if (biased && !sig) scale = exact_softmax_scale(P, zs + r * P.Rp, top, lane);
            if (lane < n) {
                const int e = pk[r * kp + lane], at = topk_place(P, e);
                const float x = zs[r * P.Rp + at];
                double v = (double)x;
                if (biased) v = biased64(score64(sig, x, top, scale), zb[at]);
                worth[e] = v;
            }
            sort_list(worth, pk + r * kp, n, k, lane);
        }
    }
    const unsigned long long open = __ballot(unsure);
    if (open != 0ull) {
#pragma unroll 1
        for (int r = 0; r < kRowsPerWave; ++r)
            if ((open >> (16 * r)) & 0xFFFFull)
                choose_row(P, zs + r * P.Rp, zb, __shfl(zmax, 16 * r, 64), worth, pk + r * kp, lane);
    }
    wave_sync();
    const int t = t0 + rr;
    if (t < P.T) store_row<16>(P, zr, zmax, Sinv, pk + rr * kp, t, c16);
}

// One token a wavefront: the same choice, made in 64 bits at once, for few
// tokens of many experts (launch_topk).  A group has 64 lanes over the next power of two
// of n_groups; the passes' minimum is a scalar.
template <int NQ>
__global__ __launch_bounds__(64 * kTopkWaves) void route_topk_wide_k(TopkParams P) {
    extern __shared__ __align__(16) float all_lds[];
    float *const lds = all_lds + (threadIdx.x >> 6) * P.wave_lds;
    double *const cs = reinterpret_cast<double *>(lds);       // [256]
    float *const zs = lds + 2 * kMaxExperts;                  // [256]
    float *const zb = zs + kMaxExperts;                       // [256]
    short *const pk = reinterpret_cast<short *>(zb + kMaxExperts);  // [kp]
    const int lane = threadIdx.x & 63;
    const int t = (int)(blockIdx.x * kTopkWaves + (threadIdx.x >> 6));
    if (t >= P.T) return;
    const int E = P.E, k = P.k;
    const bool sig = (P.flags & PP_SCORE_SIGMOID) != 0;
    const bool top2 = (P.flags & PP_GROUP_TOP2) != 0;
    const bool biased = P.sel_bias != nullptr;
    const bool scores = biased || (P.n_groups > 1 && top2);
    if (P.src.g) {
        float v[kMaxExperts / 64], b[kMaxExperts / 64];
#pragma unroll
        for (int q = 0; q < kMaxExperts / 64; ++q)
            v[q] = P.src.g[(size_t)t * E + min(lane + 64 * q, E - 1)];
        if (biased) {
#pragma unroll
            for (int q = 0; q < kMaxExperts / 64; ++q) b[q] = P.sel_bias[min(lane + 64 * q, E - 1)];
        }
#pragma unroll
        for (int q = 0; q < kMaxExperts / 64; ++q) {
            zs[lane + 64 * q] = lane + 64 * q < E ? clean_logit(v[q]) : -INFINITY;
            if (biased) zb[lane + 64 * q] = clean_logit(b[q]);
        }
    } else {
#pragma unroll 1
        for (int e = lane; e < kMaxExperts; e += 64) {
            zs[e] = -INFINITY;
            if (e >= E) continue;
            zs[e] = clean_logit(summed_logit(P, t, e, true));
            if (biased) zb[e] = clean_logit(P.sel_bias[e]);
        }
    }
    wave_sync();
    const int wl = P.lanes_log + 2;  // 64 lanes: four times those of a 16-lane row
    const int grp = lane >> wl, sub = lane & ((1 << wl) - 1);
    const int e0 = grp * P.Gs + sub, held = grp < P.n_groups ? P.Gs - sub : 0;
    float z[NQ], zmax = -INFINITY;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        float x = zs[q << wl < held ? e0 + (q << wl) : 0];
        asm volatile("" : "+v"(x));
        z[q] = q << wl < held ? x : -INFINITY;
        zmax = fmaxf(zmax, z[q]);
    }
    zmax = row_max(zmax);
    zmax = fmaxf(zmax, __uint_as_float(xor_lane<16>(__float_as_uint(zmax), lane)));
    zmax = fmaxf(zmax, __uint_as_float(xor_lane<32>(__float_as_uint(zmax), lane)));
    double c[NQ], by[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) c[q] = by[q] = (double)z[q];
    if (scores) {
        double S = 0.0;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const double x = sig ? -fabs((double)z[q]) : (double)z[q] - (double)zmax;
            by[q] = z[q] > -INFINITY ? exp_neg(fmax(x, -800.0)) : 0.0;
            S += by[q];
        }
        if (sig) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const double d = rcp64(1.0 + by[q]);
                by[q] = z[q] >= 0.0f ? d : by[q] * d;
            }
        } else {
            S = wave_reduce(S, lane, [](double a, double b) { return a + b; });
            const double r = S > 0.0 ? rcp64(S) : 0.0;
#pragma unroll
            for (int q = 0; q < NQ; ++q) by[q] *= r;  // as in score64
        }
    }
    if (biased) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const float b = zb[q << wl < held ? e0 + (q << wl) : 0];
            c[q] = z[q] > -INFINITY && b > -INFINITY ? biased64(by[q], b) : -INFINITY;
        }
    }
    if (P.n_groups > 1) {
        double a = -INFINITY, n = -INFINITY;  // the two largest
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const double v =
                top2 && !biased ? (z[q] > -INFINITY ? by[q] : -INFINITY) : c[q];
            n = fmax(n, fmin(a, v));
            a = fmax(a, v);
        }
        const int front = groups_in_front(P, a, n, lane);
#pragma unroll
        for (int q = 0; q < NQ; ++q) c[q] = front < P.top_groups ? c[q] : -INFINITY;
    }
    constexpr uint32_t kNone = 0xFFFFFFFFu;
    uint32_t key[NQ];
    {
        double cmax = c[0];
#pragma unroll
        for (int q = 1; q < NQ; ++q) cmax = fmax(cmax, c[q]);
        cmax = wave_reduce(cmax, lane, [](double a, double b) { return fmax(a, b); });
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const uint32_t e = (uint32_t)(e0 + (q << wl));
            const uint32_t d = __float_as_uint((float)(cmax - c[q])) & 0xFFFFFF00u;
            key[q] = c[q] > -INFINITY ? d | e : kNone;
            if (q << wl < held) cs[e] = c[q];
        }
    }
    auto next_key = [&](uint32_t last) {
        uint32_t m = key[0] + ~last;
#pragma unroll
        for (int q = 1; q < NQ; ++q) m = min(m, key[q] + ~last);
        m = row_min(m);
        const uint32_t a = min((uint32_t)__builtin_amdgcn_readlane((int)m, 0),
                               (uint32_t)__builtin_amdgcn_readlane((int)m, 16));
        const uint32_t b = min((uint32_t)__builtin_amdgcn_readlane((int)m, 32),
                               (uint32_t)__builtin_amdgcn_readlane((int)m, 48));
        return min(a, b) + last + 1u;
    };
    // as in route_topk_k; keys of equal upper bits are the only ones in doubt
    uint32_t last = kNone;
    bool close = false, unsure = false;
    int len = 0;
    // A pass is short and its start is jumped to: near the end of a cache line
    // it costs 20 ns more (k 32: 10.7 against 9.8 us).
    asm volatile(".p2align 6");
#pragma unroll 1
    for (int j = 0; j < k; ++j) {
        const bool over = j > 0 && last == kNone;
        const uint32_t n = next_key(last);
        close |= !over && n != kNone && j > 0 && (n ^ last) < 256u;
        last = over ? kNone : n;
        len += last != kNone ? 1 : 0;
        if (lane == 0) pk[j] = last != kNone ? (short)(last & 255u) : (short)-1;
    }
    const uint32_t cut = last;
    while (last != kNone) {
        const uint32_t n = next_key(last);
        if (n <= last || n == kNone || (n ^ cut) >= 256u) break;
        close = true;
        if (len >= kMaxList) {
            unsure = true;
            break;
        }
        last = n;
        if (lane == 0) pk[len] = (short)(n & 255u);
        ++len;
    }
    unsure |= close && k > kMaxList;
    wave_sync();
    if (unsure)
        choose_row(P, zs, zb, zmax, cs, pk, lane);
    else if (close)
        sort_list(cs, pk, len, k, lane);
    wave_sync();
    float Sinv = 0.0f;
    if (!sig && !(P.flags & PP_TOPK_RENORM)) {
        // each 16 lanes take the values that they have in route_topk_k, in
        // the same order: the same bits
        const int g = (lane & 15) >> P.lanes_log;
        float S = 0.0f;
        if (g < P.n_groups) {
#pragma unroll 4
            for (int i = lane & (P.lanes - 1); i < P.Gs; i += P.lanes)
                S += exp_fast(zs[g * P.Gs + i] - zmax);
        }
        Sinv = 1.0f / row_sum(S);
    }
    store_row<64>(P, zs, zmax, Sinv, pk, t, lane);
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

// dL/dg, the chosen experts held fixed.  With a_j = dw_j over the slots that
// name an expert, q_j = w_j / scale and D = sum_j q_j a_j:
//   softmax                 dg_e = scale p_e ([e chosen] a_e - D)
//   sigmoid                 dg_e = scale s_e (1 - s_e) a_e
//   renormalised softmax    dg_e = scale q_e (a_e - D)
//   renormalised sigmoid    dg_e = scale q_e (1 - s_e) (a_e - D)
// In fp32: with A = max |a_j|, a score is off by (24 + |x|) 2^-23 of itself,
// at most 25 2^-23 (p |x| <= 1 / e), |a_e - D| is at most 2 A, and D is off by
// (24 + 6 + 9) 2^-23 A (x averages to at most log 256 over the scores; a sum of
// 256 terms): 100 2^-23 |scale| A with the last products.
// Bound by memory (dg is written whole): 16384 x 112, k 16, plain softmax
// 5.8 us for 22 MB; a wavefront a token with the slots in turn took 57.  A token takes 16 lanes: lane c has
// slots c, c + 16, ... and columns c, c + 16, ... (NQ of them); the slots'
// values meet the columns in LDS.  ROW: plain softmax, whose gradient reaches
// every expert and needs the whole row; else only the slots' logits are read.
template <int NQ, bool ROW>
__global__ __launch_bounds__(64 * kTopkWaves) void route_topk_grad_k(TopkGradParams P) {
    // rows start 16 (or 48) banks apart
    constexpr int kStride = 16 * (NQ % 2 ? NQ : NQ + 1);
    __shared__ float acc_lds[kTopkWaves][kRowsPerWave * kStride];
    __shared__ short own_lds[kTopkWaves][kRowsPerWave * kStride];
    const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63, c16 = lane & 15, rr = lane >> 4;
    const int t0 = (int)(blockIdx.x * kTopkWaves + wv) * kRowsPerWave;
    if (t0 >= P.T) return;
    float *const acc = acc_lds[wv] + rr * kStride;
    short *const own = own_lds[wv] + rr * kStride;
    const bool sig = (P.flags & PP_SCORE_SIGMOID) != 0;
    const bool renorm = (P.flags & PP_TOPK_RENORM) != 0;
    const int E = P.E, k = P.k, t = t0 + rr, tc = min(t, P.T - 1);
    const float *const row = P.g + (size_t)tc * E;
    const int32_t *const idx = P.idx + (size_t)tc * k;
    const float *const dw = P.dw + (size_t)tc * k;
    struct Slot {
        int e;      // -1: empty
        float a, z;
    };
    auto load = [&](int j) {
        Slot s = {-1, 0.0f, -INFINITY};
        if (j >= k) return s;
        const int e = idx[j];
        const float a = dw[j];
        if ((unsigned)e >= (unsigned)E) return s;
        s.z = clean_logit(row[e]);
        if (s.z > -INFINITY) s.e = e, s.a = a;
        return s;
    };
    const Slot first = load(c16);
    auto slot = [&](int j) { return j < 16 ? first : load(j); };
    float p[NQ], zmax = -INFINITY, Sinv = 0.0f;
    if constexpr (ROW) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) p[q] = row[min(c16 + 16 * q, E - 1)];
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            p[q] = c16 + 16 * q < E ? clean_logit(p[q]) : -INFINITY;
            zmax = fmaxf(zmax, p[q]);
        }
        zmax = row_max(zmax);
        float S = 0.0f;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            p[q] = p[q] > -INFINITY ? exp_fast(p[q] - zmax) : 0.0f;
            S += p[q];
        }
        S = row_sum(S);
        Sinv = S > 0.0f ? 1.0f / S : 0.0f;
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) acc[c16 + 16 * q] = 0.0f;
    // scores of the slots, relative to the largest where they are renormalised
    float m = ROW ? zmax : 0.0f, inv = ROW ? Sinv : 1.0f, D = 0.0f;
    auto score = [&](const Slot &s) { return sig ? rel_sigmoid(s.z, m) : expf(s.z - m); };
    if (renorm) {
        m = -INFINITY;
        for (int j = c16; j < k; j += 16) m = fmaxf(m, slot(j).z);
        m = row_max(m);
        if (sig) m = fminf(m, 0.0f);
    }
    if (renorm || ROW) {
        float tot = 0.0f;
        for (int j = c16; j < k; j += 16) {
            const Slot s = slot(j);
            if (s.e < 0) continue;
            const float q = score(s);
            tot += q;
            D += q * s.a;
        }
        if (renorm) {
            tot = row_sum(tot);
            inv = tot > 0.0f ? 1.0f / tot : 0.0f;
        }
        D = row_sum(D) * inv;
    }
    // whether a token names an expert twice
    bool twice = false;
    for (int j = c16; j < k; j += 16) {
        const Slot s = slot(j);
        if (s.e >= 0) own[s.e] = (short)j;
    }
    wave_sync();
    for (int j = c16; j < k; j += 16) {
        const Slot s = slot(j);
        if (s.e >= 0) twice |= own[s.e] != (short)j;
    }
    const bool add = __ballot(twice) != 0ull;
    for (int j0 = 0; j0 < k; j0 += 16) {
        const Slot s = slot(j0 + c16);
        float v = 0.0f;
        if (s.e >= 0) {
            v = score(s) * inv * (renorm ? s.a - D : s.a);
            if (sig) v *= rel_sigmoid(-s.z, 0.0f);
        }
        if (!add) {
            if (s.e >= 0) acc[s.e] = v;
        } else {
            for (int j = 0; j < 16; ++j) {  // in slot order
                if (c16 == j && s.e >= 0) acc[s.e] += v;
                wave_sync();
            }
        }
    }
    wave_sync();
    if (t >= P.T) return;
    float *const out = P.dg + (size_t)t * E;
    float old[NQ];
    if (P.flags & PP_GRAD_ADD) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) old[q] = out[min(c16 + 16 * q, E - 1)];
    } else {
#pragma unroll
        for (int q = 0; q < NQ; ++q) old[q] = 0.0f;
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        float v = acc[c16 + 16 * q];
        if constexpr (ROW) v -= p[q] * inv * D;
        if (c16 + 16 * q < E) out[c16 + 16 * q] = old[q] + P.scale * v;
    }
}

template <int NQ>
void launch_topk_grad_nq(const TopkGradParams &P, hipStream_t s) {
    constexpr int rows = kRowsPerWave * kTopkWaves;
    const dim3 grid((P.T + rows - 1) / rows), block(64 * kTopkWaves);
    if (P.flags & (PP_SCORE_SIGMOID | PP_TOPK_RENORM))
        hipLaunchKernelGGL((route_topk_grad_k<NQ, false>), grid, block, 0, s, P);
    else
        hipLaunchKernelGGL((route_topk_grad_k<NQ, true>), grid, block, 0, s, P);
}

// The builds by how many columns a lane has: every number up to 8, then every
// other one, so that at most one column of a lane is empty.
struct TopkGradBuild {
    int columns;
    void (*launch)(const TopkGradParams &, hipStream_t);
};
template <int NQ>
constexpr TopkGradBuild topk_grad_build() {
    return {NQ, launch_topk_grad_nq<NQ>};
}
constexpr TopkGradBuild kTopkGradBuilds[] = {
    topk_grad_build<1>(),  topk_grad_build<2>(),  topk_grad_build<3>(),  topk_grad_build<4>(),
    topk_grad_build<5>(),  topk_grad_build<6>(),  topk_grad_build<7>(),  topk_grad_build<8>(),
    topk_grad_build<10>(), topk_grad_build<12>(), topk_grad_build<14>(), topk_grad_build<16>()};

void launch_topk_grad(const TopkGradParams &P, hipStream_t s) {
    const TopkGradBuild *B = kTopkGradBuilds;
    while (16 * B->columns < P.E) ++B;  // at most 16: 256 experts
    B->launch(P, s);
}

constexpr uint32_t kRuleFlags = PP_SCORE_SIGMOID | PP_TOPK_RENORM | PP_GROUP_TOP2;

// in: the logits, or the tokens.  (A wavefront's outputs are other wavefronts'
// inputs if they share an array.)
pp_status check_rule(const void *in, int32_t E, int32_t k, int32_t n_groups, int32_t top_groups,
                     const float *sel_bias, float scale, uint32_t flags, const int32_t *idx,
                     const float *w) {
    if (!idx || !w || (const void *)idx == (const void *)w) return PP_EINVAL;
    if (in == (const void *)idx || in == (const void *)w) return PP_EINVAL;
    if (sel_bias == w || (const void *)sel_bias == (const void *)idx) return PP_EINVAL;
    if (((uintptr_t)idx | (uintptr_t)w | (uintptr_t)sel_bias) & 3) return PP_EINVAL;
    if (flags & ~kRuleFlags) return PP_EINVAL;
    if (!(fabsf(scale) <= kFltMax)) return PP_EINVAL;  // also rejects NaN
    if (n_groups < 1 || E % n_groups != 0 || top_groups < 1 || top_groups > n_groups)
        return PP_EINVAL;
    if (k < 1 || k > top_groups * (E / n_groups)) return PP_EINVAL;
    if (n_groups > kMaxGroups) return PP_EUNSUPPORTED;
    return PP_OK;
}

// The builds by how many values a lane holds, every number up to 8 and then in
// steps of a fifth to two fifths: 16 for 256 experts in one group, 28 for nine
// groups of 28, the most there are.
struct TopkBuild {
    int values;
    void (*scores)(TopkParams);
    void (*logits)(TopkParams);
};
template <int NQ>
constexpr TopkBuild topk_build() {
    return {NQ, route_topk_k<NQ, true>, route_topk_k<NQ, false>};
}
constexpr TopkBuild kTopkBuilds[] = {
    topk_build<1>(),  topk_build<2>(),  topk_build<3>(),  topk_build<4>(),  topk_build<5>(),
    topk_build<6>(),  topk_build<7>(),  topk_build<8>(),  topk_build<10>(), topk_build<12>(),
    topk_build<14>(), topk_build<16>(), topk_build<20>(), topk_build<28>()};

struct TopkWideBuild {
    int values;
    void (*kernel)(TopkParams);
};
constexpr TopkWideBuild kTopkWideBuilds[] = {{4, route_topk_wide_k<4>},
                                             {7, route_topk_wide_k<7>}};
// Up to so many tokens take a wavefront each if 16 lanes would hold more than
// 8 values each, which makes the passes long.  256 experts, k 8, a wavefront
// each against 16 lanes each, us:
//                            64 tokens   1024 tokens   4096 tokens
//   order of logits          5.1  5.1    5.2   5.2     7.1   5.4
//   the same, k 32           8.8  9.0   10.3  10.9    15.4  12.1
//   sigmoid + bias           6.0  6.3    6.3   7.1     9.6   7.5
//   the same, 8 groups       7.0  6.7    7.3   7.0    10.9   7.9
//   softmax + bias, groups   6.9  6.4    7.3   8.9    11.0   9.1
// With fewer values the 16 lanes are faster for few tokens and near for 1024:
// 128 experts 5.3  4.5 (order of logits, 64 tokens), 6.0  5.5 (sigmoid + bias),
// 5.3  4.8 and 6.3  6.3 at 1024.
constexpr int kWideTokens = 1024;

hipError_t launch_topk(TopkParams P, hipStream_t s) {
    P.Gs = P.E / P.n_groups;
    P.lanes_log = 4;
    while ((16 >> P.lanes_log) < P.n_groups) --P.lanes_log;
    P.lanes = 1 << P.lanes_log;
    P.by_Gs = (uint32_t)((65536 + P.Gs - 1) / P.Gs);
    P.kp = P.k > kMaxList ? (P.k + 15) & ~15 : kMaxList;
    const TopkBuild *B = kTopkBuilds;
    while (B->values * P.lanes < P.Gs) ++B;  // at most 28: nine groups of 28, a lane each
    if (P.T <= kWideTokens && B->values > 8) {
        const TopkWideBuild *W = kTopkWideBuilds;
        while (W->values * 4 * P.lanes < P.Gs) ++W;  // at most 7
        P.Gp = P.Gs;
        P.wave_lds = 4 * kMaxExperts + P.kp / 2;
        hipLaunchKernelGGL(W->kernel, dim3((P.T + kTopkWaves - 1) / kTopkWaves),
                           dim3(64 * kTopkWaves), sizeof(float) * kTopkWaves * P.wave_lds, s, P);
        return hipGetLastError();
    }
    // a group starts `lanes` banks after the one before, so that the 16 lanes
    // of a row read 16 different banks; one group: rows 16 banks apart
    P.Gp = (B->values * P.lanes + 31) / 32 * 32 + P.lanes;
    P.Rp = (16 >> P.lanes_log) * P.Gp;
    P.pad = P.n_groups << P.lanes_log != 16 || B->values * P.lanes != P.Gs;
    const bool scores = P.sel_bias || (P.n_groups > 1 && (P.flags & PP_GROUP_TOP2));
    P.wave_lds = 2 * kMaxExperts + (kRowsPerWave + (scores ? 1 : 0)) * P.Rp +
                 kRowsPerWave * P.kp / 2;
    constexpr int rows = kRowsPerWave * kTopkWaves;
    hipLaunchKernelGGL(scores ? B->scores : B->logits, dim3((P.T + rows - 1) / rows),
                       dim3(64 * kTopkWaves), sizeof(float) * kTopkWaves * P.wave_lds, s, P);
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
    if (((uintptr_t)logits | (uintptr_t)inv_temp) & 3) return PP_EINVAL;
    const void *const outs[] = {expert_idx, gate_w, logits};
    for (const void *o : outs)
        if (o && o == (const void *)inv_temp) return PP_EINVAL;
    if (logits && (logits == gate_w || logits == sel_bias || (const void *)logits == (const void *)x ||
                   (const void *)logits == (const void *)expert_idx))
        return PP_EINVAL;
    const int E = L->dm.E;
    const pp_status st =
        check_rule(x, E, k, n_groups, top_groups, sel_bias, scale, flags, expert_idx, gate_w);
    if (st != PP_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    // the partial logits of the handle's router, in its scratch
    hipError_t e = launch_route(L, x, T, 0.0f, inv_temp, nullptr, nullptr, nullptr, false, s, false);
    if (e == hipSuccess) {
        const RouteParams R = route_params(L, x, T, 0.0f, inv_temp, nullptr, nullptr, nullptr, false);
        const TopkParams P = {{nullptr, R.gpart, R.bias, inv_temp, logits, R.KSr}, T, E, k, n_groups,
                              top_groups, sel_bias, scale, flags, expert_idx, gate_w, 0, 0, 0, 0, 0, 0, 0, 0, 0};
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
        check_rule(g, E, k, n_groups, top_groups, sel_bias, scale, flags, expert_idx, gate_w);
    if (st != PP_OK) return st;
    const TopkParams P = {{g, nullptr, nullptr, nullptr, nullptr, 0}, T, E, k, n_groups, top_groups,
                          sel_bias, scale, flags, expert_idx, gate_w, 0, 0, 0, 0, 0, 0, 0, 0, 0};
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
    if (!(fabsf(scale) <= kFltMax)) return PP_EINVAL;
    const TopkGradParams P = {g, T, E, k, expert_idx, dgate_w, scale, flags, dg};
    launch_topk_grad(P, static_cast<hipStream_t>(hip_stream));
    return hipGetLastError() == hipSuccess ? PP_OK : PP_EHIP;
}
