// Layer norm of token features and its backward pass.
//   forward   r = x (+ residual, rounded to the type it is stored in), u = (r - m) s gamma + beta
//   backward  dx = s (g - mean g - xh mean(g xh)) + d_sum with g = du gamma, xh = (r - m) s;  dgamma = sum_t du xh, dbeta = sum_t du
// Both are bound by memory: every row is read once into registers, where the mean, then the centred squares (or both sums of
// the backward pass) are taken in fp32, and written once.
#include "rows.hpp"

namespace swimba {

// A row lies in the registers of WPR waves, 8 NV elements to a lane: piece i of lane l are the elements from 8 (l + 64 WPR i) on.
// sums of n values over the row's waves, in every lane; `round` alternates so that one barrier a round is enough
template <int WPR, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*lds)[N][16], int round)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (WPR > 1) {
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < N; ++i) lds[round & 1][i][wave] = v[i];
        lds_barrier();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < WPR; ++w) v[i] += lds[round & 1][i][w];
        }
    }
}

constexpr int norm_threads(int WPR) { return WPR == 16 ? 1024 : 256; }

template <typename T, typename R, int NV, int WPR>
__global__ void __launch_bounds__(norm_threads(WPR))
norm_fwd_kernel(const T *x, const R *residual, const float *__restrict__ gamma, const float *__restrict__ beta, float eps,
                T *__restrict__ u, R *sum, float *__restrict__ mean, float *__restrict__ rstd, int64_t tokens, int D)
{
    __shared__ float lds[2][1][16];
    constexpr int RPB = norm_threads(WPR) / 64 / WPR;          // rows a block has at a time
    const int lane = threadIdx.x % (64 * WPR);
    const float width = (float)D;
    int round = 0;
    for (int64_t t = (int64_t)blockIdx.x * RPB + threadIdx.x / (64 * WPR); t < tokens; t += (int64_t)gridDim.x * RPB) {
        float r[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int d = 8 * (lane + 64 * WPR * i), n = D - d;
            load8(r[i], x + t * D + d, n, 0.f);
            if (residual) {
                float a[8];
                load8(a, residual + t * D + d, n, 0.f);
#pragma unroll
                for (int j = 0; j < 8; ++j) r[i][j] = to_float(from_float<R>(r[i][j] + a[j]));
                if (sum) store8(sum + t * D + d, r[i], n);
            }
        }
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += r[i][j];
        row_sums<WPR>(s, lds, round++);
        const float m = s[0] / width;       // divided, not multiplied: a constant row is centred to zero
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int n = D - 8 * (lane + 64 * WPR * i);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                r[i][j] -= m;
                s[0] += j < n ? r[i][j] * r[i][j] : 0.f;
            }
        }
        row_sums<WPR>(s, lds, round++);
        const float is = 1.0f / sqrtf(s[0] / width + eps);
        if (lane == 0) {
            if (mean) mean[t] = m;
            if (rstd) rstd[t] = is;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int d = 8 * (lane + 64 * WPR * i), n = D - d;
            float g[8], b[8];
            if (gamma) load8(g, gamma + d, n, 0.f);
            if (beta) load8(b, beta + d, n, 0.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) r[i][j] = r[i][j] * is * (gamma ? g[j] : 1.f) + (beta ? b[j] : 0.f);
            store8(u + t * D + d, r[i], n);
        }
    }
}

template <typename T, typename R, int NV, int WPR>
__global__ void __launch_bounds__(norm_threads(WPR))
norm_bwd_kernel(const T *__restrict__ du, const R *__restrict__ r, const float *__restrict__ gamma,
                const float *__restrict__ mean, const float *__restrict__ rstd, const R *d_sum, R *dx, T *__restrict__ dx_io,
                float *__restrict__ part, int64_t tokens, int D)
{
    __shared__ float lds[2][2][16];
    constexpr int RPB = norm_threads(WPR) / 64 / WPR;
    const int lane = threadIdx.x % (64 * WPR), slot = threadIdx.x / (64 * WPR);
    const float inv = 1.0f / (float)D;
    float dg[NV][8] = {}, db[NV][8] = {};
    int round = 0;
    for (int64_t t = (int64_t)blockIdx.x * RPB + slot; t < tokens; t += (int64_t)gridDim.x * RPB) {
        const float m = mean[t], is = rstd[t];
        float xh[NV][8], g[NV][8], s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int d = 8 * (lane + 64 * WPR * i), n = D - d;
            float w[8];
            load8(xh[i], r + t * D + d, n, m);
            load8(g[i], du + t * D + d, n, 0.f);
            if (gamma) load8(w, gamma + d, n, 0.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                xh[i][j] = (xh[i][j] - m) * is;
                dg[i][j] += g[i][j] * xh[i][j];
                db[i][j] += g[i][j];
                if (gamma) g[i][j] *= w[j];
                s[0] += g[i][j];
                s[1] += g[i][j] * xh[i][j];
            }
        }
        row_sums<WPR>(s, lds, round++);
        const float mg = s[0] * inv, mx = s[1] * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int d = 8 * (lane + 64 * WPR * i), n = D - d;
            float a[8];
            if (d_sum) load8(a, d_sum + t * D + d, n, 0.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[i][j] = is * (g[i][j] - mg - xh[i][j] * mx) + (d_sum ? a[j] : 0.f);
            store8(dx + t * D + d, g[i], n);
            if (dx_io) store8(dx_io + t * D + d, g[i], n);
        }
    }
    if (!part) return;
    // (blocks x RPB, 2, D)
    float *p = part + ((int64_t)blockIdx.x * RPB + slot) * 2 * D;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int d = 8 * (lane + 64 * WPR * i), n = D - d;
        store8(p + d, dg[i], n);
        store8(p + D + d, db[i], n);
    }
}

// out[c] = sum over the rows of part (rows, 2 D), in their order; columns behind D are dbeta's
__global__ void __launch_bounds__(256)
norm_reduce_kernel(const float *__restrict__ part, int rows, int D, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= 2 * D) return;
    float s = 0.f;
    for (int i = 0; i < rows; ++i) s += part[(int64_t)i * 2 * D + c];
    float *out = c < D ? dgamma : dbeta;
    if (out) out[c < D ? c : c - D] = s;
}

namespace {

// Rows of one wave up to 1024 features, of four up to 8192, of sixteen up to 16384.
int waves_per_row(int D) { return D <= 1024 ? 1 : D <= 8192 ? 4 : 16; }
int rows_per_block(int D) { return D <= 1024 ? 4 : 1; }

template <typename T, typename R>
swimba_status norm_fwd(int64_t tokens, int D, const void *x, const void *residual, const float *gamma, const float *beta,
                       float eps, void *u, void *sum, float *mean, float *rstd, hipStream_t st)
{
    const int wpr = waves_per_row(D), rpb = rows_per_block(D);
    const int64_t need = (tokens + rpb - 1) / rpb;
    const unsigned grid = (unsigned)(need < (1 << 20) ? need : (1 << 20));
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(norm_threads(wpr)), 0, st, (const T *)x, (const R *)residual, gamma, beta, eps,
                           (T *)u, (R *)sum, mean, rstd, tokens, D);
    };
    if (D <= 512) go(norm_fwd_kernel<T, R, 1, 1>);
    else if (D <= 1024) go(norm_fwd_kernel<T, R, 2, 1>);
    else if (D <= 2048) go(norm_fwd_kernel<T, R, 1, 4>);
    else if (D <= 4096) go(norm_fwd_kernel<T, R, 2, 4>);
    else if (D <= 8192) go(norm_fwd_kernel<T, R, 4, 4>);
    else go(norm_fwd_kernel<T, R, 2, 16>);
    SWIMBA_CHECK_LAUNCH();
    return SWIMBA_OK;
}

// most blocks of the backward pass, which keep sums of their own
int64_t bwd_blocks(int64_t tokens, int D)
{
    const int rpb = rows_per_block(D);
    const int64_t need = (tokens + rpb - 1) / rpb, most = waves_per_row(D) == 16 ? 256 : 512;
    return need < most ? need : most;
}

template <typename T, typename R>
swimba_status norm_bwd(int64_t tokens, int D, const void *du, const void *r, const float *gamma, const float *mean,
                       const float *rstd, const void *d_sum, void *dx, void *dx_io, float *part, hipStream_t st)
{
    const int wpr = waves_per_row(D);
    const unsigned grid = (unsigned)bwd_blocks(tokens, D);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(norm_threads(wpr)), 0, st, (const T *)du, (const R *)r, gamma, mean, rstd,
                           (const R *)d_sum, (R *)dx, (T *)dx_io, part, tokens, D);
    };
    if (D <= 512) go(norm_bwd_kernel<T, R, 1, 1>);
    else if (D <= 1024) go(norm_bwd_kernel<T, R, 2, 1>);
    else if (D <= 2048) go(norm_bwd_kernel<T, R, 1, 4>);
    else if (D <= 4096) go(norm_bwd_kernel<T, R, 2, 4>);
    else if (D <= 8192) go(norm_bwd_kernel<T, R, 4, 4>);
    else go(norm_bwd_kernel<T, R, 2, 16>);
    SWIMBA_CHECK_LAUNCH();
    return SWIMBA_OK;
}

}  // namespace

size_t layer_norm_bwd_bytes(int64_t tokens, int D)
{
    return (size_t)bwd_blocks(tokens, D) * rows_per_block(D) * 2 * D * sizeof(float);
}

swimba_status launch_layer_norm(int64_t tokens, int D, int io_dtype, int res_dtype, const void *x, const void *residual,
                                const float *gamma, const float *beta, float eps, void *u, void *sum, float *mean, float *rstd,
                                hipStream_t st)
{
    if (tokens == 0) return SWIMBA_OK;
    const auto go = io_dtype == SWIMBA_F32 ? norm_fwd<float, float> : res_dtype == SWIMBA_F32 ? norm_fwd<bf16, float> : norm_fwd<bf16, bf16>;
    return go(tokens, D, x, residual, gamma, beta, eps, u, sum, mean, rstd, st);
}

swimba_status launch_layer_norm_bwd(int64_t tokens, int D, int io_dtype, int res_dtype, const void *du, const void *r,
                                    const float *gamma, const float *mean, const float *rstd, const void *d_sum, void *dx,
                                    void *dx_io, float *dgamma, float *dbeta, float *part, hipStream_t st)
{
    const bool sums = dgamma || dbeta;
    if (tokens > 0) {
        const auto go = io_dtype == SWIMBA_F32 ? norm_bwd<float, float> : res_dtype == SWIMBA_F32 ? norm_bwd<bf16, float> : norm_bwd<bf16, bf16>;
        const swimba_status s = go(tokens, D, du, r, gamma, mean, rstd, d_sum, dx, dx_io, sums ? part : nullptr, st);
        if (s != SWIMBA_OK) return s;
    }
    if (sums) {
        hipLaunchKernelGGL(norm_reduce_kernel, dim3((unsigned)((2 * D + 255) / 256)), dim3(256), 0, st, part,
                           (int)(bwd_blocks(tokens, D) * rows_per_block(D)), D, dgamma, dbeta);
        SWIMBA_CHECK_LAUNCH();
    }
    return SWIMBA_OK;
}

}  // namespace swimba
