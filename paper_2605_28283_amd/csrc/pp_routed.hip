// The experts' products on a choice that the caller gives:
//   y_t = sum_j gate_w[t][j] FFN_{expert_idx[t][j]}(x_t)   (+ the output bias),
// Eq. (moe_output) with any weights.  The gate/up and down kernels are those
// of the layer's own selection; this file turns the choice into what they
// read: per-expert token masks (decode) or per-token expert masks (prefill),
// and the weight of each kept (token, expert) pair, which scales h before it
// is rounded.
// A slot outside 0 .. E - 1 is empty; an expert named twice by a token counts
// once with the sum of its weights, added in slot order.  A weight that is a
// NaN becomes the plain one: h is split into two bf16 numbers by adding to its
// bits, which carries a NaN of all ones over into a zero.
#include "pp_internal.h"

namespace pp {
namespace {

struct RoutedParams {
    const int32_t *idx;  // [T][k]
    const float *w;      // [T][k] or NULL (1)
    int T, k, E;
    float *gsig;         // [T][E], written for kept pairs only
};

// The slots of n tokens from t0 on, one a thread at a time.  mark(t, e) records
// that token t0 + t named e and returns whether it had named it before;
// twice: LDS flags of the n tokens, cleared by the caller.
// Bound by one round trip to memory (indices and weights are loaded together).
template <typename Mark>
__device__ __forceinline__ void scatter_tokens(const RoutedParams &P, int t0, int n, int *twice,
                                               Mark mark) {
    const int32_t *idx = P.idx + (size_t)t0 * P.k;
    const float *w = P.w ? P.w + (size_t)t0 * P.k : nullptr;
    float *gs = P.gsig + (size_t)t0 * P.E;
    const int slots = n * P.k, th = (int)blockDim.x;
    auto plain = [](float v) { return v == v ? v : __builtin_nanf(""); };
    auto store = [&](int s, int e, float v) {
        const int t = s / P.k;
        if ((unsigned)e < (unsigned)P.E && !twice[t]) gs[(size_t)t * P.E + e] = plain(v);
    };
    const int s0 = (int)threadIdx.x;
    const int e0 = s0 < slots ? idx[s0] : -1;
    const float w0 = s0 < slots && w ? w[s0] : 1.0f;
    if ((unsigned)e0 < (unsigned)P.E && mark(s0 / P.k, e0)) twice[s0 / P.k] = 1;
    for (int s = s0 + th; s < slots; s += th) {
        const int e = idx[s];
        if ((unsigned)e < (unsigned)P.E && mark(s / P.k, e)) twice[s / P.k] = 1;
    }
    __syncthreads();
    if (s0 < slots) store(s0, e0, w0);
    for (int s = s0 + th; s < slots; s += th) store(s, idx[s], w ? w[s] : 1.0f);
    for (int t = s0; t < n; t += th) {
        if (!twice[t]) continue;
        // an expert twice: one thread adds the weights in slot order
        for (int j = 0; j < P.k; ++j) {
            const int e = idx[t * P.k + j];
            if ((unsigned)e < (unsigned)P.E) gs[(size_t)t * P.E + e] = 0.0f;
        }
        for (int j = 0; j < P.k; ++j) {
            const int e = idx[t * P.k + j];
            if ((unsigned)e < (unsigned)P.E)
                gs[(size_t)t * P.E + e] += w ? plain(w[t * P.k + j]) : 1.0f;
        }
    }
}

// Decode slice (T <= 64): one workgroup, so that the masks need no clearing
// launch in front.
__global__ __launch_bounds__(1024) void routed_decode_k(RoutedParams P,
                                                        unsigned long long *__restrict__ emask) {
    __shared__ unsigned long long em[kMaxExperts];
    __shared__ int twice[kDecodeTile];
    const int tid = threadIdx.x;
    if (tid < kMaxExperts) em[tid] = 0ull;
    if (tid < kDecodeTile) twice[tid] = 0;
    __syncthreads();
    scatter_tokens(P, 0, P.T, twice, [&](int t, int e) {
        return ((atomicOr(&em[e], 1ull << t) >> t) & 1ull) != 0ull;
    });
    if (tid < P.E) emask[tid] = em[tid];
}

constexpr int kRoutedTokens = 32;  // of a prefill workgroup: 8 slots a token keep 256 threads busy
__global__ __launch_bounds__(256) void routed_prefill_k(RoutedParams P,
                                                        uint32_t *__restrict__ selmask) {
    __shared__ uint32_t sm[kRoutedTokens][8];
    __shared__ int twice[kRoutedTokens];
    const int tid = threadIdx.x, t0 = blockIdx.x * kRoutedTokens;
    const int n = min(kRoutedTokens, P.T - t0);
    static_assert(kRoutedTokens * 8 == 256, "a mask word a thread");
    sm[tid >> 3][tid & 7] = 0u;
    if (tid < kRoutedTokens) twice[tid] = 0;
    __syncthreads();
    scatter_tokens(P, t0, n, twice, [&](int t, int e) {
        return ((atomicOr(&sm[t][e >> 5], 1u << (e & 31)) >> (e & 31)) & 1u) != 0u;
    });
    if ((tid >> 3) < n) selmask[(size_t)t0 * 8 + tid] = sm[tid >> 3][tid & 7];
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
            hipLaunchKernelGGL(routed_prefill_k, dim3((n + kRoutedTokens - 1) / kRoutedTokens),
                               dim3(256), 0, s, P, L->selmask);
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
