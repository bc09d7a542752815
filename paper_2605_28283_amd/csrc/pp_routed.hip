// The experts' products on a choice that the caller gives:
//   y_t = sum_j gate_w[t][j] FFN_{expert_idx[t][j]}(x_t)   (+ the output bias),
// Eq. (moe_output) with any weights.  The gate/up and down kernels are those
// of the layer's own selection; this file turns the choice into what they
// read: per-expert token masks (decode) or per-token expert masks (prefill),
// and the weight of each kept (token, expert) pair, which scales h before it
// is rounded.
// A slot outside 0 .. E - 1 is empty; an expert named twice by a token counts
// once with the sum of its weights, added in slot order.
#include "pp_internal.h"

namespace pp {
namespace {

struct RoutedParams {
    const int32_t *idx;  // [T][k]
    const float *w;      // [T][k] or NULL (1)
    int T, k, E;
    float *gsig;         // [T][E], written for kept pairs only
};

// One token on one wavefront.  mark(e) records the pair and returns whether
// this token had named e before.
template <typename Mark>
__device__ __forceinline__ void scatter_token(const RoutedParams &P, int t, int lane, Mark mark) {
    const int32_t *idx = P.idx + (size_t)t * P.k;
    const float *w = P.w ? P.w + (size_t)t * P.k : nullptr;
    float *gs = P.gsig + (size_t)t * P.E;
    bool dup = false;
    for (int j = lane; j < P.k; j += 64) {
        const int e = idx[j];
        if ((unsigned)e < (unsigned)P.E) dup |= mark(e);
    }
    if (__ballot(dup) == 0ull) {
        for (int j = lane; j < P.k; j += 64) {
            const int e = idx[j];
            if ((unsigned)e < (unsigned)P.E) gs[e] = w ? w[j] : 1.0f;
        }
    } else if (lane == 0) {
        // an expert twice: one lane adds the weights in slot order
        for (int j = 0; j < P.k; ++j) {
            const int e = idx[j];
            if ((unsigned)e < (unsigned)P.E) gs[e] = 0.0f;
        }
        for (int j = 0; j < P.k; ++j) {
            const int e = idx[j];
            if ((unsigned)e < (unsigned)P.E) gs[e] += w ? w[j] : 1.0f;
        }
    }
}

// Decode slice (T <= 64): one workgroup, so that the masks need no clearing
// launch in front.
__global__ __launch_bounds__(1024) void routed_decode_k(RoutedParams P,
                                                        unsigned long long *__restrict__ emask) {
    __shared__ unsigned long long em[kMaxExperts];
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < kMaxExperts) em[tid] = 0ull;
    __syncthreads();
    for (int t = tid >> 6; t < P.T; t += 16)
        scatter_token(P, t, lane, [&](int e) {
            return ((atomicOr(&em[e], 1ull << t) >> t) & 1ull) != 0ull;
        });
    __syncthreads();
    if (tid < P.E) emask[tid] = em[tid];
}

__global__ __launch_bounds__(256) void routed_prefill_k(RoutedParams P,
                                                        uint32_t *__restrict__ selmask) {
    __shared__ uint32_t sm[4][8];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int t = blockIdx.x * 4 + wv;
    if (lane < 8) sm[wv][lane] = 0u;
    __syncthreads();
    if (t < P.T)
        scatter_token(P, t, lane, [&](int e) {
            return ((atomicOr(&sm[wv][e >> 5], 1u << (e & 31)) >> (e & 31)) & 1u) != 0u;
        });
    __syncthreads();
    if (t < P.T && lane < 8) selmask[(size_t)t * 8 + lane] = sm[wv][lane];
}

pp_status run_routed(pp_layer *L, const uint16_t *x, int32_t T, int32_t k, const int32_t *idx,
                     const float *w, float *y, void *hip_stream, bool prefill) {
    if (!L || !x || !idx || !y || T < 1 || T > L->max_tokens) return PP_EINVAL;
    const int E = L->dm.E, d = L->dm.d;
    if (k < 1 || k > E || (((uintptr_t)idx | (uintptr_t)w) & 3)) return PP_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const int slice = prefill ? T : kDecodeTile;
    for (int t0 = 0; t0 < T; t0 += slice) {
        const int n = T - t0 < slice ? T - t0 : slice;
        const RoutedParams P = {idx + (size_t)t0 * k, w ? w + (size_t)t0 * k : nullptr, n, k, E,
                                L->gsig};
        prof_mark(L, PP_KERNEL_ROUTE, s, true);
        if (prefill)
            hipLaunchKernelGGL(routed_prefill_k, dim3((n + 3) / 4), dim3(256), 0, s, P, L->selmask);
        else
            hipLaunchKernelGGL(routed_decode_k, dim3(1), dim3(1024), 0, s, P, L->emask);
        prof_mark(L, PP_KERNEL_ROUTE, s, false);
        hipError_t e = hipGetLastError();
        // h is scaled by gsig, whatever the layer's own aggregation
        const uint32_t flags = PP_AGG_SIGMOID;
        if (e == hipSuccess)
            e = prefill ? launch_prefill_ffn(L, x + (size_t)t0 * d, n, y + (size_t)t0 * d, flags, s)
                        : launch_decode_ffn(L, x + (size_t)t0 * d, n, y + (size_t)t0 * d, false,
                                            flags, s);
        if (e != hipSuccess) return PP_EHIP;
    }
    return PP_OK;
}

}  // namespace
}  // namespace pp

extern "C" pp_status prunepath_ffn_decode_routed(pp_layer *L, const uint16_t *x, int32_t T,
                                                 int32_t k, const int32_t *expert_idx,
                                                 const float *gate_w, float *y,
                                                 void *hip_stream) {
    return pp::run_routed(L, x, T, k, expert_idx, gate_w, y, hip_stream, false);
}

extern "C" pp_status prunepath_ffn_prefill_routed(pp_layer *L, const uint16_t *x, int32_t T,
                                                  int32_t k, const int32_t *expert_idx,
                                                  const float *gate_w, float *y,
                                                  void *hip_stream) {
    return pp::run_routed(L, x, T, k, expert_idx, gate_w, y, hip_stream, true);
}
