// Residual add + layer norm between layers, and its gradient:
//   r = x + y,  mu = mean(r),  v = mean((r - mu)^2),  rstd = 1 / sqrt(v + eps)
//   u = (r - mu) rstd w + b
//   dx = dres + rstd (a - mean(a) - hat mean(a hat)),  a = w du, hat = (r - mu) rstd
//   dw = sum_t du hat,  db = sum_t du
// Not part of the paper's method: the norm of the GELU-MLP blocks whose FFN
// prunepath_create_mlp makes.  All sums are fp32 in an order fixed by (T, d).
#include "pp_internal.h"

namespace pp {
namespace {

constexpr int kLnThreads = 256;

// Sum over the workgroup, the same in every thread.
__device__ __forceinline__ float block_total(float v, float *ws) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const float t = lane_value(wave_scan_f32(v), 63);
    __syncthreads();
    if (lane == 0) ws[wv] = t;
    __syncthreads();
    return (ws[0] + ws[1]) + (ws[2] + ws[3]);
}

__device__ __forceinline__ float load_du(const void *p, size_t i, bool f32) {
    return f32 ? static_cast<const float *>(p)[i]
               : bf16_to_f32(static_cast<const uint16_t *>(p)[i]);
}

__global__ __launch_bounds__(kLnThreads) void layernorm_k(const float *x, const float *y,
                                                          float *x_out, int d, float eps,
                                                          const float *w, const float *b, void *u,
                                                          float *stats, int f32) {
    __shared__ float ws[4];
    const size_t row = (size_t)blockIdx.x * d;
    float s = 0.0f;
    for (int c = threadIdx.x; c < d; c += kLnThreads) s += x[row + c] + (y ? y[row + c] : 0.0f);
    const float mu = block_total(s, ws) / (float)d;
    s = 0.0f;
    for (int c = threadIdx.x; c < d; c += kLnThreads) {
        const float r = x[row + c] + (y ? y[row + c] : 0.0f);
        s += (r - mu) * (r - mu);
    }
    const float rstd = 1.0f / sqrtf(block_total(s, ws) / (float)d + eps);
    for (int c = threadIdx.x; c < d; c += kLnThreads) {
        const float r = x[row + c] + (y ? y[row + c] : 0.0f);
        if (x_out) x_out[row + c] = r;
        const float v = (r - mu) * rstd * (w ? w[c] : 1.0f) + (b ? b[c] : 0.0f);
        if (f32)
            static_cast<float *>(u)[row + c] = v;
        else
            static_cast<uint16_t *>(u)[row + c] = f32_to_bf16(v);
    }
    if (stats && threadIdx.x == 0) {
        stats[2 * blockIdx.x] = mu;
        stats[2 * blockIdx.x + 1] = rstd;
    }
}

__global__ __launch_bounds__(kLnThreads) void layernorm_dx_k(const float *r, const void *du,
                                                             const float *dres, int d,
                                                             const float *w, const float *stats,
                                                             float *dx, int f32) {
    __shared__ float ws[4];
    const size_t row = (size_t)blockIdx.x * d;
    const float mu = stats[2 * blockIdx.x], rstd = stats[2 * blockIdx.x + 1];
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < d; c += kLnThreads) {
        const float a = load_du(du, row + c, f32) * (w ? w[c] : 1.0f);
        s1 += a;
        s2 += a * ((r[row + c] - mu) * rstd);
    }
    const float m1 = block_total(s1, ws) / (float)d, m2 = block_total(s2, ws) / (float)d;
    for (int c = threadIdx.x; c < d; c += kLnThreads) {
        const float a = load_du(du, row + c, f32) * (w ? w[c] : 1.0f);
        const float v = rstd * (a - m1 - (r[row + c] - mu) * rstd * m2);
        dx[row + c] = dres ? dres[row + c] + v : v;
    }
}

// Column sums over kLnRows rows at a time: part [nb][2][d].
constexpr int kLnRows = 64;
__global__ __launch_bounds__(kLnThreads) void layernorm_dw_k(const float *r, const void *du, int T,
                                                             int d, const float *stats,
                                                             float *part, int f32) {
    const int c = blockIdx.x * kLnThreads + threadIdx.x, t0 = blockIdx.y * kLnRows;
    if (c >= d) return;
    float sw = 0.0f, sb = 0.0f;
    for (int t = t0; t < min(t0 + kLnRows, T); ++t) {
        const float g = load_du(du, (size_t)t * d + c, f32);
        sw += g * ((r[(size_t)t * d + c] - stats[2 * t]) * stats[2 * t + 1]);
        sb += g;
    }
    part[((size_t)blockIdx.y * 2) * d + c] = sw;
    part[((size_t)blockIdx.y * 2 + 1) * d + c] = sb;
}

__global__ __launch_bounds__(kLnThreads) void layernorm_sum_k(const float *part, int nb, int d,
                                                              float *dw, float *db) {
    const int c = blockIdx.x * kLnThreads + threadIdx.x;
    if (c >= d) return;
    double sw = 0.0, sb = 0.0;
    for (int i = 0; i < nb; ++i) {
        sw += part[((size_t)i * 2) * d + c];
        sb += part[((size_t)i * 2 + 1) * d + c];
    }
    if (dw) dw[c] = (float)sw;
    if (db) db[c] = (float)sb;
}

constexpr int kLnMaxRows = 1 << 20, kLnMaxWidth = 1 << 16;

inline int ln_blocks(int T) { return (T + kLnRows - 1) / kLnRows; }

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" pp_status prunepath_residual_layernorm(const float *x, const float *y, float *x_out,
                                                  int32_t T, int32_t d, float eps, const float *w,
                                                  const float *b, void *u, float *stats,
                                                  uint32_t flags, void *hip_stream) {
    if (!x || !u) return PP_EINVAL;
    if (T < 1 || T > kLnMaxRows || d < 1 || d > kLnMaxWidth || (flags & ~PP_NORM_F32))
        return PP_EINVAL;
    if (!(eps >= 0.0f && eps <= 3.0e38f)) return PP_EINVAL;  // also rejects NaN
    const bool f32 = (flags & PP_NORM_F32) != 0;
    if ((((uintptr_t)x | (uintptr_t)y | (uintptr_t)x_out | (uintptr_t)w | (uintptr_t)b |
          (uintptr_t)stats) & 3) || ((uintptr_t)u & (f32 ? 3 : 1)))
        return PP_EINVAL;
    if (u == (const void *)x || u == (const void *)y || u == (const void *)x_out) return PP_EINVAL;
    hipLaunchKernelGGL(layernorm_k, dim3(T), dim3(kLnThreads), 0,
                       static_cast<hipStream_t>(hip_stream), x, y, x_out, d, eps, w, b, u, stats,
                       (int)f32);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_EHIP;
}

extern "C" size_t prunepath_residual_layernorm_grad_workspace(int32_t T, int32_t d) {
    if (T < 1 || T > kLnMaxRows || d < 1 || d > kLnMaxWidth) return 0;
    return sizeof(float) * 2 * (size_t)ln_blocks(T) * (size_t)d;
}

extern "C" pp_status prunepath_residual_layernorm_grad(const float *x_out, const void *du,
                                                       const float *dres, int32_t T, int32_t d,
                                                       const float *w, const float *stats,
                                                       float *dx, float *dw, float *db,
                                                       void *workspace, uint32_t flags,
                                                       void *hip_stream) {
    if (!x_out || !du || !stats || !dx) return PP_EINVAL;
    if (T < 1 || T > kLnMaxRows || d < 1 || d > kLnMaxWidth || (flags & ~PP_NORM_F32))
        return PP_EINVAL;
    if ((dw || db) && !workspace) return PP_EINVAL;
    const bool f32 = (flags & PP_NORM_F32) != 0;
    if ((((uintptr_t)x_out | (uintptr_t)dres | (uintptr_t)w | (uintptr_t)stats | (uintptr_t)dx |
          (uintptr_t)dw | (uintptr_t)db | (uintptr_t)workspace) & 3) ||
        ((uintptr_t)du & (f32 ? 3 : 1)))
        return PP_EINVAL;
    if ((const void *)dx == du || dx == x_out || (dw && dw == db)) return PP_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    float *part = static_cast<float *>(workspace);
    if (dw || db) {
        const int nb = ln_blocks(T), nc = (d + kLnThreads - 1) / kLnThreads;
        hipLaunchKernelGGL(layernorm_dw_k, dim3(nc, nb), dim3(kLnThreads), 0, s, x_out, du, T, d,
                           stats, part, (int)f32);
        hipLaunchKernelGGL(layernorm_sum_k, dim3(nc), dim3(kLnThreads), 0, s, part, nb, d, dw, db);
    }
    hipLaunchKernelGGL(layernorm_dx_k, dim3(T), dim3(kLnThreads), 0, s, x_out, du, dres, d, w,
                       stats, dx, (int)f32);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_EHIP;
}
