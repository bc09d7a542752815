// Residual add + layer norm between layers, and its gradient:
//   r = x + y,  mu = mean(r),  v = mean((r - mu)^2),  rstd = 1 / sqrt(v + eps)
//   u = (r - mu) rstd w + b
//   dx = dres + rstd (a - mean(a) - hat mean(a hat)),  a = w du, hat = (r - mu) rstd
//   dw = sum_t du hat,  db = sum_t du
// Not part of the paper's method: the norm of the GELU-MLP blocks whose FFN
// prunepath_create_mlp makes.  Bound by memory: each input is read once and
// each output written once.  16384 x 4096 with bf16 u and du: 160 us forward
// (5.9 TB/s of 0.94 GB), 157 us back (6.0 TB/s), where a 4 GiB copy moves 4.8
// TB/s; at d 4095, column by column, 178 and 172 us.  (Rows read again for
// every sum took 910 us for both.)
//
// A row of up to 8192 values stays in registers between its sums and its
// outputs: one wavefront for up to 1024 (four rows a workgroup, no barrier; two
// forward where values are moved one at a time), four for up to 4096, eight for
// up to 8192.  Columns are moved four at a
// time where d and every array allow it, else one at a time.  Longer rows are
// read again for every sum.
// The gradient's workgroups walk over rows and keep the column sums of du hat
// and du in registers; their partial sums (at most kLnBlocks rows of 2 d) are
// added by a second launch.
// All sums are fp32, their order fixed by (T, d) and the kind of columns, that
// of a row's sums by d and that alone; the partial sums are added in fp64.
#include <type_traits>

#include "pp_internal.h"

namespace pp {
namespace {

constexpr int kLnThreads = 256;
constexpr int kLnBlocks = 512;   // gradient workgroups, two to a CU
constexpr int kLnRegWidth = 8192;

__device__ __forceinline__ float wave_total(float v) {
    return lane_value(wave_scan_f32(v), 63);
}

// Sums of n values over the WPR wavefronts of a row, the same in every
// thread.  slot: LDS for WPR * n floats that no earlier reader still needs.
template <int WPR, int n>
__device__ __forceinline__ void row_totals(float (&v)[n], float *slot) {
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = wave_total(v[i]);
    if constexpr (WPR > 1) {
        const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < n; ++i) slot[i * WPR + wv] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < n; ++i) {
            float t = slot[i * WPR];
#pragma unroll
            for (int w = 1; w < WPR; ++w) t += slot[i * WPR + w];
            v[i] = t;
        }
    }
}

// V consecutive values of a row.  NT: a nontemporal access, for arrays too
// long to be in a cache when they are met again (ln_streams).
template <int V>
struct Cols {
    float v[V];
};
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
template <typename T, bool NT>
__device__ __forceinline__ T load_as(const void *p) {
    const T *q = static_cast<const T *>(p);
    return NT ? __builtin_nontemporal_load(q) : *q;
}
template <typename T, bool NT>
__device__ __forceinline__ void store_as(void *p, T v) {
    T *q = static_cast<T *>(p);
    if constexpr (NT)
        __builtin_nontemporal_store(v, q);
    else
        *q = v;
}
template <int V, bool NT = false>
__device__ __forceinline__ Cols<V> load_f32(const float *p) {
    Cols<V> c;
    if constexpr (V == 4) {
        const f32x4 f = load_as<f32x4, NT>(p);
        c.v[0] = f.x, c.v[1] = f.y, c.v[2] = f.z, c.v[3] = f.w;
    } else {
        c.v[0] = load_as<float, NT>(p);
    }
    return c;
}
template <int V, bool NT = false>
__device__ __forceinline__ void store_f32(float *p, const Cols<V> &c) {
    if constexpr (V == 4)
        store_as<f32x4, NT>(p, f32x4{c.v[0], c.v[1], c.v[2], c.v[3]});
    else
        store_as<float, NT>(p, c.v[0]);
}
// bf16, rounded to nearest even by the hardware (NaN stays NaN).
__device__ __forceinline__ uint32_t bf16_bits(float f) {
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));
}
template <int V, bool F32, bool NT = false>
__device__ __forceinline__ void store_u(void *u, size_t i, const Cols<V> &c) {
    if constexpr (F32)
        store_f32<V, NT>(static_cast<float *>(u) + i, c);
    else if constexpr (V == 4)
        store_as<u32x2_t, NT>(static_cast<uint16_t *>(u) + i,
                              u32x2_t{bf16_bits(c.v[0]) | (bf16_bits(c.v[1]) << 16),
                                      bf16_bits(c.v[2]) | (bf16_bits(c.v[3]) << 16)});
    else
        store_as<uint16_t, NT>(static_cast<uint16_t *>(u) + i, (uint16_t)bf16_bits(c.v[0]));
}
template <int V, bool F32, bool NT = false>
__device__ __forceinline__ Cols<V> load_du(const void *p, size_t i) {
    if constexpr (F32) return load_f32<V, NT>(static_cast<const float *>(p) + i);
    Cols<V> c;
    const uint16_t *q = static_cast<const uint16_t *>(p) + i;
    if constexpr (V == 4) {
        const u32x2_t b = load_as<u32x2_t, NT>(q);
        c.v[0] = __uint_as_float(b.x << 16), c.v[1] = __uint_as_float(b.x & 0xFFFF0000u);
        c.v[2] = __uint_as_float(b.y << 16), c.v[3] = __uint_as_float(b.y & 0xFFFF0000u);
    } else {
        c.v[0] = bf16_to_f32(load_as<uint16_t, NT>(q));
    }
    return c;
}

struct LnParams {
    const float *x, *y;
    float *x_out;
    int T, d;
    float eps;
    const float *w, *b;
    void *u;
    float *stats;
};

// Threads of a workgroup: one row's, or four rows of a wavefront each.
constexpr int ln_threads(int wpr) { return wpr == 1 ? 256 : 64 * wpr; }

// Columns of V values in a thread's registers: N of them, column i at
// V (thread + i * 64 WPR); one past the row's end reads the row's last one and
// counts for nothing.
template <int WPR, int N, int V, bool F32, bool NT>
__global__ __launch_bounds__(ln_threads(WPR)) void layernorm_k(LnParams P) {
    __shared__ float slot[2][WPR];
    constexpr int kRows = WPR == 1 ? 4 : 1, kTh = 64 * WPR;
    const int tid = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int t = blockIdx.x * kRows + (WPR == 1 ? threadIdx.x >> 6 : 0);
    if (t >= P.T) return;  // whole wavefronts of a workgroup without barriers
    const int n = P.d / V;
    const size_t row = (size_t)t * P.d;
    int at[N];
    Cols<V> r[N];
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = V * min(tid + i * kTh, n - 1);
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = load_f32<V>(P.x + row + at[i]);
    if (P.y) {
        Cols<V> y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = load_f32<V>(P.y + row + at[i]);
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) r[i].v[j] += y[i].v[j];
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (tid + i * kTh < n) {
            if (P.x_out) store_f32<V, NT>(P.x_out + row + at[i], r[i]);
#pragma unroll
            for (int j = 0; j < V; ++j) s[0] += r[i].v[j];
        }
    row_totals<WPR>(s, slot[0]);
    const float mu = s[0] / (float)P.d;
    s[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            r[i].v[j] -= mu;
            if (tid + i * kTh < n) s[0] += r[i].v[j] * r[i].v[j];
        }
    row_totals<WPR>(s, slot[1]);
    const float rstd = 1.0f / sqrtf(s[0] / (float)P.d + P.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (tid + i * kTh >= n) continue;
        Cols<V> w, b;
#pragma unroll
        for (int j = 0; j < V; ++j) w.v[j] = 1.0f, b.v[j] = 0.0f;
        if (P.w) w = load_f32<V>(P.w + at[i]);
        if (P.b) b = load_f32<V>(P.b + at[i]);
#pragma unroll
        for (int j = 0; j < V; ++j) r[i].v[j] = r[i].v[j] * rstd * w.v[j] + b.v[j];
        store_u<V, F32, NT>(P.u, row + at[i], r[i]);
    }
    if (P.stats && tid == 0) {
        P.stats[2 * (size_t)t] = mu;
        P.stats[2 * (size_t)t + 1] = rstd;
    }
}

// Any row, read once for each sum and once for the outputs.
template <bool F32>
__global__ __launch_bounds__(kLnThreads) void layernorm_long_k(LnParams P) {
    __shared__ float slot[2][4];
    const size_t row = (size_t)blockIdx.x * P.d;
    float s[1] = {0.0f};
    for (int c = threadIdx.x; c < P.d; c += kLnThreads)
        s[0] += P.x[row + c] + (P.y ? P.y[row + c] : 0.0f);
    row_totals<4>(s, slot[0]);
    const float mu = s[0] / (float)P.d;
    s[0] = 0.0f;
    for (int c = threadIdx.x; c < P.d; c += kLnThreads) {
        const float v = P.x[row + c] + (P.y ? P.y[row + c] : 0.0f) - mu;
        s[0] += v * v;
    }
    row_totals<4>(s, slot[1]);
    const float rstd = 1.0f / sqrtf(s[0] / (float)P.d + P.eps);
    for (int c = threadIdx.x; c < P.d; c += kLnThreads) {
        const float r = P.x[row + c] + (P.y ? P.y[row + c] : 0.0f);
        if (P.x_out) P.x_out[row + c] = r;
        Cols<1> v;
        v.v[0] = (r - mu) * rstd * (P.w ? P.w[c] : 1.0f) + (P.b ? P.b[c] : 0.0f);
        store_u<1, F32>(P.u, row + c, v);
    }
    if (P.stats && threadIdx.x == 0) {
        P.stats[2 * (size_t)blockIdx.x] = mu;
        P.stats[2 * (size_t)blockIdx.x + 1] = rstd;
    }
}

// ------------------------------------------------------------------ gradient

struct LnGradParams {
    const float *r;
    const void *du;
    const float *dres;
    int T, d;
    const float *w, *stats;
    float *dx;
    float *part;  // [workgroups][2][d] column sums of du hat and of du, or NULL
};

template <int WPR, int N, int V, bool F32, bool NT>
__global__ __launch_bounds__(ln_threads(WPR)) void layernorm_grad_k(LnGradParams P) {
    constexpr int kRows = WPR == 1 ? 4 : 1, kTh = 64 * WPR;
    __shared__ float slot[2][2 * WPR];
    __shared__ float join[WPR == 1 ? 3 * 2 * N * V * 64 : 1];
    const int wv = threadIdx.x >> 6;
    const int tid = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int n = P.d / V;
    int at[N];
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = V * min(tid + i * kTh, n - 1);
    Cols<V> w[N], sw[N], sb[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int j = 0; j < V; ++j) w[i].v[j] = 1.0f, sw[i].v[j] = 0.0f, sb[i].v[j] = 0.0f;
        if (P.w) w[i] = load_f32<V>(P.w + at[i]);
    }
    const float inv_d = 1.0f / (float)P.d;
    int par = 0;
    for (int t = blockIdx.x * kRows + (WPR == 1 ? wv : 0); t < P.T;
         t += gridDim.x * kRows, par ^= 1) {
        const size_t row = (size_t)t * P.d;
        const float mu = P.stats[2 * (size_t)t], rstd = P.stats[2 * (size_t)t + 1];
        Cols<V> h[N], g[N], o[N];
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] = load_f32<V, NT>(P.r + row + at[i]);
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = load_du<V, F32, NT>(P.du, row + at[i]);
        if (P.dres) {
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = load_f32<V, NT>(P.dres + row + at[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) o[i].v[j] = 0.0f;
        }
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool in = tid + i * kTh < n;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                h[i].v[j] = (h[i].v[j] - mu) * rstd;
                sw[i].v[j] += g[i].v[j] * h[i].v[j];
                sb[i].v[j] += g[i].v[j];
                g[i].v[j] *= w[i].v[j];
                if (in) {
                    s[0] += g[i].v[j];
                    s[1] += g[i].v[j] * h[i].v[j];
                }
            }
        }
        // two slots in turn: a row's totals are read before the next row's
        // barrier, and written again only after it
        row_totals<WPR>(s, slot[par]);
        const float m1 = s[0] * inv_d, m2 = s[1] * inv_d;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (tid + i * kTh >= n) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) o[i].v[j] += rstd * (g[i].v[j] - m1 - h[i].v[j] * m2);
            store_f32<V, NT>(P.dx + row + at[i], o[i]);
        }
    }
    if (!P.part) return;
    if constexpr (WPR == 1) {
        // the four wavefronts' sums, in order
        if (wv > 0) {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    join[(((wv - 1) * 2 + 0) * N * V + i * V + j) * 64 + tid] = sw[i].v[j];
                    join[(((wv - 1) * 2 + 1) * N * V + i * V + j) * 64 + tid] = sb[i].v[j];
                }
        }
        __syncthreads();
        if (wv > 0) return;
        for (int q = 0; q < 3; ++q) {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    sw[i].v[j] += join[((q * 2 + 0) * N * V + i * V + j) * 64 + tid];
                    sb[i].v[j] += join[((q * 2 + 1) * N * V + i * V + j) * 64 + tid];
                }
        }
    }
    float *pw = P.part + (size_t)blockIdx.x * 2 * P.d;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (tid + i * kTh < n) {
            store_f32<V>(pw + at[i], sw[i]);
            store_f32<V>(pw + P.d + at[i], sb[i]);
        }
}

// Rows past kLnRegWidth values: dx, then the column sums.
template <bool F32>
__global__ __launch_bounds__(kLnThreads) void layernorm_dx_long_k(LnGradParams P) {
    __shared__ float slot[8];
    const size_t row = (size_t)blockIdx.x * P.d;
    const float mu = P.stats[2 * (size_t)blockIdx.x], rstd = P.stats[2 * (size_t)blockIdx.x + 1];
    float s[2] = {0.0f, 0.0f};
    for (int c = threadIdx.x; c < P.d; c += kLnThreads) {
        const float a = load_du<1, F32>(P.du, row + c).v[0] * (P.w ? P.w[c] : 1.0f);
        s[0] += a;
        s[1] += a * ((P.r[row + c] - mu) * rstd);
    }
    row_totals<4>(s, slot);
    const float m1 = s[0] / (float)P.d, m2 = s[1] / (float)P.d;
    for (int c = threadIdx.x; c < P.d; c += kLnThreads) {
        const float a = load_du<1, F32>(P.du, row + c).v[0] * (P.w ? P.w[c] : 1.0f);
        const float v = rstd * (a - m1 - (P.r[row + c] - mu) * rstd * m2);
        P.dx[row + c] = P.dres ? P.dres[row + c] + v : v;
    }
}
template <bool F32>
__global__ __launch_bounds__(kLnThreads) void layernorm_cols_long_k(LnGradParams P) {
    const int c = blockIdx.x * kLnThreads + threadIdx.x;
    if (c >= P.d) return;
    float sw = 0.0f, sb = 0.0f;
    for (int t = blockIdx.y; t < P.T; t += gridDim.y) {
        const size_t i = (size_t)t * P.d + c;
        const float g = load_du<1, F32>(P.du, i).v[0];
        sw += g * ((P.r[i] - P.stats[2 * (size_t)t]) * P.stats[2 * (size_t)t + 1]);
        sb += g;
    }
    float *pw = P.part + (size_t)blockIdx.y * 2 * P.d;
    pw[c] = sw;
    pw[P.d + c] = sb;
}

// dw and db from the nb partial rows of 2 d: 64 columns a workgroup, row
// i of the partial sums with wavefront i % 16.
__global__ __launch_bounds__(1024) void layernorm_sum_k(const float *__restrict__ part, int nb,
                                                        int d, float *__restrict__ dw,
                                                        float *__restrict__ db) {
    __shared__ double sum[16][64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    constexpr int kLoads = 8;
    double s = 0.0;
    for (int i0 = wv; i0 < nb; i0 += 16 * kLoads) {
        float v[kLoads];
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            v[q] = part[(size_t)min(i0 + 16 * q, nb - 1) * 2 * d + min(c, 2 * d - 1)];
#pragma unroll
        for (int q = 0; q < kLoads; ++q) s += i0 + 16 * q < nb ? (double)v[q] : 0.0;
    }
    sum[wv][lane] = s;
    __syncthreads();
    if (wv > 0 || c >= 2 * d) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sum[w][lane];
    float *out = c < d ? dw : db;
    if (out) out[c < d ? c : c - d] = (float)s;
}

constexpr int kLnMaxRows = 1 << 20, kLnMaxWidth = 1 << 16;
constexpr float kLnMaxEps = 3.402823466e38f;  // any float

// Gradient workgroups (and partial rows): one for each four rows or each row,
// up to kLnBlocks.
inline int ln_blocks(int T, int d) {
    const int rows = d <= 1024 ? 4 : 1, n = (T + rows - 1) / rows;
    return n < kLnBlocks ? n : kLnBlocks;
}

// Whether a call's arrays (about 14 bytes a value) do not fit `mib` of the 256
// MiB Infinity Cache: nontemporal stores of whole vectors in the forward kernel
// then, loads (its inputs are read for the last time) and stores in the
// gradient's.  Forward and gradient in turn: 16384 x 4096 343 -> 317 us, 6000 x
// 4096 137 -> 115; the gradient also where they fill half the cache, 3000 x 4096
// 69 -> 63, but not below, 2048 x 4096 46 -> 48, 512 x 4096 23.0 -> 23.7.
// (Nontemporal loads in the forward kernel: 166 -> 179 us alone, column by
// column 280.)
inline bool ln_streams(int T, int d, size_t mib) { return (size_t)T * (size_t)d * 14 > mib << 20; }

template <int WPR, int N, int V, bool F32>
void launch_ln(const LnParams &P, hipStream_t s) {
    const int rows = WPR == 1 ? 4 : 1;
    const dim3 grid((P.T + rows - 1) / rows), block(ln_threads(WPR));
    if (V == 4 && ln_streams(P.T, P.d, 256))
        hipLaunchKernelGGL((layernorm_k<WPR, N, V, F32, V == 4>), grid, block, 0, s, P);
    else
        hipLaunchKernelGGL((layernorm_k<WPR, N, V, F32, false>), grid, block, 0, s, P);
}
template <int WPR, int N, int V, bool F32>
void launch_ln(const LnGradParams &P, hipStream_t s) {
    const dim3 grid(ln_blocks(P.T, P.d)), block(ln_threads(WPR));
    if (ln_streams(P.T, P.d, 128))
        hipLaunchKernelGGL((layernorm_grad_k<WPR, N, V, F32, true>), grid, block, 0, s, P);
    else
        hipLaunchKernelGGL((layernorm_grad_k<WPR, N, V, F32, false>), grid, block, 0, s, P);
}

// The build for a row of d values: V = 4 needs d and every array in whole
// float4 (u and du of bf16: 8 bytes).
template <int V, bool F32, typename Params>
void launch_ln_width(const Params &P, hipStream_t s) {
    constexpr int q = 4 / V;  // registers' columns per float4
    // two wavefronts a row where one would hold 9 to 16 single values a lane
    // (d 1023: one row 5.4 -> 4.2 us, d 771: 1001 rows 6.1 -> 5.2, 16384 rows
    // 35.9 -> 31.9); the gradient's partial rows would double
    constexpr bool two = V == 1 && std::is_same_v<Params, LnParams>;
    if (P.d <= 256)
        launch_ln<1, 1 * q, V, F32>(P, s);
    else if (P.d <= 512)
        launch_ln<1, 2 * q, V, F32>(P, s);
    else if (P.d <= 1024)
        launch_ln<two ? 2 : 1, two ? 8 : 4 * q, V, F32>(P, s);
    else if (P.d <= 2048)
        launch_ln<4, 2 * q, V, F32>(P, s);
    else if (P.d <= 4096)
        launch_ln<4, 4 * q, V, F32>(P, s);
    else
        launch_ln<8, 4 * q, V, F32>(P, s);
}
template <typename Params>
void launch_ln_reg(const Params &P, bool vec, bool f32, hipStream_t s) {
    if (vec)
        f32 ? launch_ln_width<4, true>(P, s) : launch_ln_width<4, false>(P, s);
    else
        f32 ? launch_ln_width<1, true>(P, s) : launch_ln_width<1, false>(P, s);
}

inline bool whole_vectors(int d, uintptr_t arrays, const void *half, bool f32) {
    return d % 4 == 0 && arrays % 16 == 0 && (uintptr_t)half % (f32 ? 16 : 8) == 0;
}

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
    if (!(eps >= 0.0f && eps <= kLnMaxEps)) return PP_EINVAL;  // also rejects NaN
    const bool f32 = (flags & PP_NORM_F32) != 0;
    if ((((uintptr_t)x | (uintptr_t)y | (uintptr_t)x_out | (uintptr_t)w | (uintptr_t)b |
          (uintptr_t)stats) & 3) || ((uintptr_t)u & (f32 ? 3 : 1)))
        return PP_EINVAL;
    if (u == (const void *)x || u == (const void *)y || u == (const void *)x_out) return PP_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const LnParams P = {x, y, x_out, T, d, eps, w, b, u, stats};
    if (d <= kLnRegWidth)
        launch_ln_reg(P, whole_vectors(d, (uintptr_t)x | (uintptr_t)y | (uintptr_t)x_out |
                                              (uintptr_t)w | (uintptr_t)b, u, f32), f32, s);
    else if (f32)
        hipLaunchKernelGGL(layernorm_long_k<true>, dim3(T), dim3(kLnThreads), 0, s, P);
    else
        hipLaunchKernelGGL(layernorm_long_k<false>, dim3(T), dim3(kLnThreads), 0, s, P);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_EHIP;
}

extern "C" size_t prunepath_residual_layernorm_grad_workspace(int32_t T, int32_t d) {
    if (T < 1 || T > kLnMaxRows || d < 1 || d > kLnMaxWidth) return 0;
    return sizeof(float) * 2 * (size_t)ln_blocks(T, d) * (size_t)d;
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
    float *part = dw || db ? static_cast<float *>(workspace) : nullptr;
    const LnGradParams P = {x_out, du, dres, T, d, w, stats, dx, part};
    const int nb = ln_blocks(T, d);
    if (d <= kLnRegWidth) {
        launch_ln_reg(P, whole_vectors(d, (uintptr_t)x_out | (uintptr_t)dres | (uintptr_t)w |
                                              (uintptr_t)dx | (uintptr_t)part, du, f32), f32, s);
    } else {
        // the column sums first: dx may be dres, which they do not read
        const dim3 grid((d + kLnThreads - 1) / kLnThreads, nb);
        if (part && f32)
            hipLaunchKernelGGL(layernorm_cols_long_k<true>, grid, dim3(kLnThreads), 0, s, P);
        else if (part)
            hipLaunchKernelGGL(layernorm_cols_long_k<false>, grid, dim3(kLnThreads), 0, s, P);
        if (f32)
            hipLaunchKernelGGL(layernorm_dx_long_k<true>, dim3(T), dim3(kLnThreads), 0, s, P);
        else
            hipLaunchKernelGGL(layernorm_dx_long_k<false>, dim3(T), dim3(kLnThreads), 0, s, P);
    }
    if (part)
        hipLaunchKernelGGL(layernorm_sum_k, dim3((2 * d + 63) / 64), dim3(1024), 0, s, part, nb, d,
                           dw, db);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_EHIP;
}
