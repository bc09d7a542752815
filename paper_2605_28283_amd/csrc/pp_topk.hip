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
// c is compared in 64 bits: a choice next to a border is that of the
// definition.  Weights are formed in fp32; renormalised ones from scores
// relative to the largest chosen one, so a row of scores that all underflow
// still has them.
// Deterministic: no floating-point atomics; a token's result does not depend
// on T.
#include "pp_select.h"

namespace pp {
namespace {

constexpr int kTopkWaves = 4;  // one token each
constexpr int kMaxGroups = 16;
constexpr int kMaxTopkRows = 1 << 22;

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
};

__device__ __forceinline__ float load_logit(const LogitSource &S, int T, int E, int t, int e) {
    if (S.g) return S.g[(size_t)t * E + e];
    float sum = 0.0f;
    for (int k = 0; k < S.KSr; ++k) sum += S.gpart[((size_t)k * T + t) * E + e];
    const float z = (sum + S.bias[e]) * (S.inv_temp ? S.inv_temp[t] : 1.0f);
    if (S.logits) S.logits[(size_t)t * E + e] = z;
    return z;
}

// NaN and -inf to -inf, +inf to the largest float.
__device__ __forceinline__ float clean_logit(float z) {
    return z > -INFINITY ? fminf(z, 3.402823466e38f) : -INFINITY;
}

__device__ __forceinline__ double wave_max_f64(double v) {
#pragma unroll
    for (int st = 1; st < 64; st <<= 1) v = fmax(v, __shfl_xor(v, st, 64));
    return v;
}
__device__ __forceinline__ float wave_max_f32(float v) {
#pragma unroll
    for (int st = 1; st < 64; st <<= 1) v = fmaxf(v, __shfl_xor(v, st, 64));
    return v;
}
__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int st = 1; st < 64; st <<= 1) v += __shfl_xor(v, st, 64);
    return v;
}
__device__ __forceinline__ float wave_sum_f32(float v) {
#pragma unroll
    for (int st = 1; st < 64; st <<= 1) v += __shfl_xor(v, st, 64);
    return v;
}

// sigmoid(z) over e^m for m = min(largest z, 0): relative scores that do not
// all underflow.
__device__ __forceinline__ float rel_sigmoid(float z, float m) {
    return expf(fminf(z, 0.0f) - m) / (1.0f + expf(-fabsf(z)));
}

__global__ __launch_bounds__(64 * kTopkWaves) void route_topk_k(TopkParams P) {
    __shared__ double cs[kTopkWaves][kMaxExperts];
    __shared__ float zs[kTopkWaves][kMaxExperts];
    __shared__ int picks[kTopkWaves][kMaxExperts];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int t = blockIdx.x * kTopkWaves + wv;
    const bool live = t < P.T;
    const int tc = live ? t : P.T - 1;
    const bool sig = (P.flags & PP_SCORE_SIGMOID) != 0;
    const bool top2 = (P.flags & PP_GROUP_TOP2) != 0;
    const int E = P.E, Gs = E / P.n_groups;
    constexpr int NQ = kMaxExperts / 64;
    float z[NQ];
    float zmax = -INFINITY;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int e = lane + 64 * q;
        z[q] = e < E ? clean_logit(load_logit(P.src, P.T, E, tc, e)) : -INFINITY;
        zmax = fmaxf(zmax, z[q]);
    }
    zmax = wave_max_f32(zmax);
    // scores in 64 bits
    double s[NQ], S = 0.0;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        s[q] = 0.0;
        if (z[q] > -INFINITY)
            s[q] = sig ? 1.0 / (1.0 + exp(-(double)z[q])) : exp((double)z[q] - (double)zmax);
        S += s[q];
    }
    S = wave_sum_f64(S);
    double c[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
        const int e = lane + 64 * q;
        if (!sig) s[q] = S > 0.0 ? s[q] / S : 0.0;
        c[q] = -INFINITY;
        double by = -INFINITY;
        if (e < E && z[q] > -INFINITY) {
            const float b = P.sel_bias ? clean_logit(P.sel_bias[e]) : 0.0f;
            if (b > -INFINITY) {
                c[q] = P.sel_bias ? s[q] + (double)b : (double)z[q];
                by = top2 && !P.sel_bias ? s[q] : c[q];
            }
        }
        if (e < E) {
            cs[wv][e] = by;
            zs[wv][e] = z[q];
        }
    }
    __syncthreads();
    if (P.n_groups > 1) {
        double v = -INFINITY;
        if (lane < P.n_groups) {
            double a = -INFINITY, b = -INFINITY;
            for (int i = 0; i < Gs; ++i) {
                const double x = cs[wv][lane * Gs + i];
                b = fmax(b, fmin(a, x));
                a = fmax(a, x);
            }
            v = top2 && b > -INFINITY ? a + b : a;
        }
        int front = 0;
        for (int g = 0; g < P.n_groups; ++g) {
            const double o = __shfl(v, g, 64);
            front += (o > v || (o == v && g < lane)) ? 1 : 0;
        }
        const unsigned long long keep = __ballot(lane < P.n_groups && front < P.top_groups);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const int e = lane + 64 * q;
            if (e < E && !((keep >> (e / Gs)) & 1ull)) c[q] = -INFINITY;
        }
    }
    int n = 0;  // experts chosen
    for (int j = 0; j < P.k; ++j) {
        double best = -INFINITY;
        int be = E;
#pragma unroll
        for (int q = 0; q < NQ; ++q)
            if (c[q] > best) {
                best = c[q];
                be = lane + 64 * q;
            }
        const double top = wave_max_f64(best);
        int e = best == top && top > -INFINITY ? be : E;
#pragma unroll
        for (int st = 1; st < 64; st <<= 1) e = min(e, __shfl_xor(e, st, 64));
        const bool some = e < E;
        n += some ? 1 : 0;
        if (lane == 0) picks[wv][j] = some ? e : -1;
#pragma unroll
        for (int q = 0; q < NQ; ++q)
            if (lane + 64 * q == e) c[q] = -INFINITY;
    }
    __syncthreads();
    // weights
    const bool renorm = (P.flags & PP_TOPK_RENORM) != 0;
    float m = -INFINITY;
    for (int j = lane; j < n; j += 64) m = fmaxf(m, zs[wv][picks[wv][j]]);
    m = wave_max_f32(m);
    if (sig) m = fminf(m, 0.0f);
    float tot = 0.0f;
    for (int j = lane; j < n; j += 64) {
        const float x = zs[wv][picks[wv][j]];
        tot += sig ? rel_sigmoid(x, m) : expf(x - m);
    }
    tot = wave_sum_f32(tot);
    if (!live) return;
    for (int j = lane; j < P.k; j += 64) {
        const int e = picks[wv][j];
        float w = 0.0f;
        if (e >= 0) {
            const float x = zs[wv][e];
            if (renorm)
                w = P.scale * ((sig ? rel_sigmoid(x, m) : expf(x - m)) / tot);
            else if (sig)
                w = P.scale * rel_sigmoid(x, 0.0f);
            else
                w = P.scale * (float)(exp((double)x - (double)zmax) / S);
        }
        P.idx[(size_t)t * P.k + j] = e;
        P.w[(size_t)t * P.k + j] = w;
    }
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
__global__ __launch_bounds__(64 * kTopkWaves) void route_topk_grad_k(TopkGradParams P) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int t = blockIdx.x * kTopkWaves + wv;
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

hipError_t launch_topk(const TopkParams &P, hipStream_t s) {
    hipLaunchKernelGGL(route_topk_k, dim3((P.T + kTopkWaves - 1) / kTopkWaves),
                       dim3(64 * kTopkWaves), 0, s, P);
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
                              top_groups, sel_bias, scale, flags, expert_idx, gate_w};
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
                          sel_bias, scale, flags, expert_idx, gate_w};
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
    hipLaunchKernelGGL(route_topk_grad_k, dim3((T + kTopkWaves - 1) / kTopkWaves),
                       dim3(64 * kTopkWaves), 0, static_cast<hipStream_t>(hip_stream), P);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_EHIP;
}
