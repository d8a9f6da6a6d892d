// Training the router: routing with per-expert counts and a balance loss, the gradient of the logits, and the backward pass of
// the router's linear map.
//   balance   pi = softmax(logits), K = top-k;  counts[e] = #{t : e in K_t}, P[e] = mean_t pi_t[e],  loss = E sum_e f_e P_e with
//             f_e = counts[e] / (k n), over the n tokens of a group that count
//   logits    g_t[e] = [e in K_t] dw + d_loss (E / n) f_e,   d_logits = pi (g - <pi, g>)
//   linear    du = d_logits W_g + du_add,   dW_g = d_logits^T u
#include "rows.hpp"

namespace swimba {

// tokens of a slice: a block's share of a group, whose sums are added up by the second launch
constexpr int64_t BAL_SLICE = 256;
constexpr int64_t BAL_SLICES = 256;         // most slices of a group
constexpr int64_t BAL_BLOCKS = 4096;        // most blocks, where there are not more groups than that
static int64_t balance_slices(int64_t groups, int64_t tokens)
{
    const int64_t n = (tokens + BAL_SLICE - 1) / BAL_SLICE, fit = groups < BAL_BLOCKS ? BAL_BLOCKS / (groups ? groups : 1) : 1;
    const int64_t most = fit < BAL_SLICES ? fit : BAL_SLICES;
    return n < most ? n : most;
}

// part (groups, slices, E): {sum of probabilities, count}
template <typename T>
__global__ void __launch_bounds__(256)
balance_kernel(const T *__restrict__ logits, const uint8_t *__restrict__ mask, int32_t *__restrict__ topk_idx,
               float *__restrict__ topk_w, float2 *__restrict__ part, int64_t tokens, int slices, int E, int K)
{
    __shared__ float prob[4][SWIMBA_MAX_EXPERTS];
    __shared__ int count[SWIMBA_MAX_EXPERTS];
    const int64_t grp = blockIdx.x / slices;
    const int slice = blockIdx.x % slices, wave = threadIdx.x >> 6;
    for (int e = threadIdx.x; e < E; e += 256) {
        count[e] = 0;
        for (int w = 0; w < 4; ++w) prob[w][e] = 0.f;
    }
    __syncthreads();
    for (int64_t base = (int64_t)slice * 256; base < tokens; base += (int64_t)slices * 256) {
        const int64_t t = base + threadIdx.x, tt = grp * tokens + (t < tokens ? t : tokens - 1);
        const T *g = logits + tt * E;
        int32_t li[SWIMBA_MAX_TOPK];
        float lw[SWIMBA_MAX_TOPK];
        route_token([&](int e) { return to_float(g[e]); }, E, K, li, lw);
        float m = -INFINITY, Z = 0.f;
        for (int e = 0; e < E; ++e) m = fmaxf(m, to_float(g[e]));
        for (int e = 0; e < E; ++e) Z += route_exp(to_float(g[e]) - m);
        bool none = true;                                       // all -inf
        for (int e = 0; e < E; ++e) none = none && to_float(g[e]) == -INFINITY;
        const bool counts = t < tokens && (!mask || mask[tt]) && !none;
#pragma unroll
        for (int r = 0; r < SWIMBA_MAX_TOPK; ++r)
            if (r < K && t < tokens) {
                if (topk_idx) topk_idx[tt * K + r] = li[r];
                if (topk_w) topk_w[tt * K + r] = lw[r];
                if (counts) atomicAdd(&count[li[r]], 1);        // whole numbers: the order does not matter
            }
        const float invZ = 1.0f / Z;
        for (int e = 0; e < E; ++e) {
            const float p = wave_sum(counts ? route_exp(to_float(g[e]) - m) * invZ : 0.f);
            if ((threadIdx.x & 63) == 0) prob[wave][e] += p;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += 256)
        part[(int64_t)blockIdx.x * E + e] =
            make_float2(prob[0][e] + prob[1][e] + prob[2][e] + prob[3][e], __int_as_float(count[e]));
}

__global__ void __launch_bounds__(SWIMBA_MAX_EXPERTS)
balance_loss_kernel(const float2 *__restrict__ part, int slices, int E, int K, int32_t *__restrict__ counts,
                    float *__restrict__ prob_mean, float *__restrict__ loss)
{
    __shared__ double sums[SWIMBA_MAX_EXPERTS];
    const int64_t grp = blockIdx.x;
    const int e = threadIdx.x;
    int c = 0;
    float p = 0.f;
    if (e < E)
        for (int s = 0; s < slices; ++s) {
            const float2 v = part[(grp * slices + s) * E + e];
            p += v.x;
            c += __float_as_int(v.y);
        }
    auto total = [&](double v) {
        sums[e] = v;
        __syncthreads();
        double r = 0.;
        for (int i = 0; i < E; ++i) r += sums[i];
        __syncthreads();
        return r;
    };
    const double all = total(c);                                // k n
    const float mean = all > 0. ? (float)(p * K / all) : 0.f;
    const double l = total(all > 0. ? (double)c / all * mean : 0.);
    if (e < E) {
        counts[grp * E + e] = c;
        if (prob_mean) prob_mean[grp * E + e] = mean;
    }
    if (e == 0) loss[grp] = (float)(E * l);
}

size_t balance_bytes(int64_t groups, int64_t tokens, int E)
{
    return (size_t)groups * balance_slices(groups, tokens) * E * sizeof(float2);
}

swimba_status launch_router_balance(int64_t groups, int64_t tokens, int E, int K, int io_dtype, const void *logits,
                                    const uint8_t *mask, int32_t *topk_idx, float *topk_w, int32_t *counts, float *prob_mean,
                                    float *loss, void *part, hipStream_t st)
{
    if (groups == 0) return SWIMBA_OK;
    const int slices = (int)balance_slices(groups, tokens);
    if (slices > 0) {
        const dim3 grid((unsigned)(groups * slices));
        if (io_dtype == SWIMBA_BF16)
            hipLaunchKernelGGL(balance_kernel<bf16>, grid, dim3(256), 0, st, (const bf16 *)logits, mask, topk_idx, topk_w,
                               (float2 *)part, tokens, slices, E, K);
        else
            hipLaunchKernelGGL(balance_kernel<float>, grid, dim3(256), 0, st, (const float *)logits, mask, topk_idx, topk_w,
                               (float2 *)part, tokens, slices, E, K);
        SWIMBA_CHECK_LAUNCH();
    }
    hipLaunchKernelGGL(balance_loss_kernel, dim3((unsigned)groups), dim3(SWIMBA_MAX_EXPERTS), 0, st, (const float2 *)part, slices, E,
                       K, counts, prob_mean, loss);
    SWIMBA_CHECK_LAUNCH();
    return SWIMBA_OK;
}

template <typename T>
__global__ void __launch_bounds__(256)
router_bwd_kernel(const T *__restrict__ logits, const uint8_t *__restrict__ mask, const int32_t *__restrict__ topk_idx,
                  const float *__restrict__ d_topk_w, const int32_t *__restrict__ counts, const float *__restrict__ d_loss,
                  T *__restrict__ d_logits, int64_t tokens, int64_t per_group, int E, int K)
{
    __shared__ float share[SWIMBA_MAX_EXPERTS];                 // d_loss (E / n) f_e
    const int64_t grp = blockIdx.x / per_group;
    if (counts) {
        double all = 0.;
        for (int e = 0; e < E; ++e) all += counts[grp * E + e];
        for (int e = threadIdx.x; e < E; e += 256)
            share[e] = all > 0. ? (float)(d_loss[grp] * (double)counts[grp * E + e] / all * ((double)E * K / all)) : 0.f;
        __syncthreads();
    }
    for (int64_t t = (blockIdx.x % per_group) * 256 + threadIdx.x; t < tokens; t += per_group * 256) {
    const int64_t tt = grp * tokens + t;
    const T *z = logits + tt * E;
    T *out = d_logits + tt * E;
    const bool balance = counts && (!mask || mask[tt]);
    bool zero = !balance;
    if (d_topk_w)
        for (int r = 0; r < K; ++r) zero = zero && d_topk_w[tt * K + r] == 0.f;
    float m = -INFINITY, Z = 0.f, s = 0.f;
    bool none = true;
    for (int e = 0; e < E; ++e) {
        m = fmaxf(m, to_float(z[e]));
        none = none && to_float(z[e]) == -INFINITY;
    }
    if (zero || none) {
        for (int e = 0; e < E; ++e) out[e] = from_float<T>(0.f);
        continue;
    }
    auto g = [&](int e) {
        float v = balance ? share[e] : 0.f;
        if (d_topk_w)
            for (int r = 0; r < K; ++r)
                if (topk_idx[tt * K + r] == e) v += d_topk_w[tt * K + r];
        return v;
    };
    for (int e = 0; e < E; ++e) Z += route_exp(to_float(z[e]) - m);
    const float invZ = 1.0f / Z;
    for (int e = 0; e < E; ++e) s += route_exp(to_float(z[e]) - m) * invZ * g(e);
    for (int e = 0; e < E; ++e) out[e] = from_float<T>(route_exp(to_float(z[e]) - m) * invZ * (g(e) - s));
    }
}

swimba_status launch_router_bwd(int64_t groups, int64_t tokens, int E, int K, int io_dtype, const void *logits, const uint8_t *mask,
                                const int32_t *topk_idx, const float *d_topk_w, const int32_t *counts, const float *d_loss,
                                void *d_logits, hipStream_t st)
{
    if (groups == 0 || tokens == 0) return SWIMBA_OK;
    const int64_t need = (tokens + 255) / 256, fit = groups < 65536 ? 65536 / groups : 1, per_group = need < fit ? need : fit;
    const dim3 grid((unsigned)(groups * per_group));
    if (io_dtype == SWIMBA_BF16)
        hipLaunchKernelGGL(router_bwd_kernel<bf16>, grid, dim3(256), 0, st, (const bf16 *)logits, mask, topk_idx, d_topk_w, counts,
                           d_loss, (bf16 *)d_logits, tokens, per_group, E, K);
    else
        hipLaunchKernelGGL(router_bwd_kernel<float>, grid, dim3(256), 0, st, (const float *)logits, mask, topk_idx, d_topk_w, counts,
                           d_loss, (float *)d_logits, tokens, per_group, E, K);
    SWIMBA_CHECK_LAUNCH();
    return SWIMBA_OK;
}

// ---- backward pass of the linear map ------------------------------------------------------------------------------------
constexpr int64_t RLB_SLICE = 512, RLB_SLICES = 64;            // tokens of a slice of dW_g, most slices
static int64_t linear_slices(int64_t tokens)
{
    const int64_t n = (tokens + RLB_SLICE - 1) / RLB_SLICE;
    return n < RLB_SLICES ? n : RLB_SLICES;
}

template <typename T>
__global__ void __launch_bounds__(256)
linear_du_kernel(const T *__restrict__ Wg, const T *__restrict__ dl, const T *du_add, T *du, int64_t tokens, int D, int E)
{
    const int64_t t = blockIdx.y + (int64_t)blockIdx.z * 65535;
    const int d = blockIdx.x * 256 + threadIdx.x;
    if (t >= tokens || d >= D) return;
    float s = 0.f;
    for (int e = 0; e < E; ++e) s += to_float(dl[t * E + e]) * to_float(Wg[(int64_t)e * D + d]);
    if (du_add) s += to_float(du_add[t * D + d]);
    du[t * D + d] = from_float<T>(s);
}

template <typename T>
__global__ void __launch_bounds__(256)
linear_dw_kernel(const T *__restrict__ u, const T *__restrict__ dl, float *__restrict__ part, int64_t tokens, int D, int E)
{
    const int d = blockIdx.x * 256 + threadIdx.x, e = blockIdx.y, slices = gridDim.z;
    if (d >= D) return;
    const int64_t n = (tokens + slices - 1) / slices, t0 = blockIdx.z * n, t1 = t0 + n < tokens ? t0 + n : tokens;
    float s = 0.f;
    for (int64_t t = t0; t < t1; ++t) s += to_float(dl[t * E + e]) * to_float(u[t * D + d]);
    part[((int64_t)blockIdx.z * E + e) * D + d] = s;
}

__global__ void __launch_bounds__(256)
linear_reduce_kernel(const float *__restrict__ part, int slices, int64_t n, float *__restrict__ dW)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float s = 0.f;
    for (int k = 0; k < slices; ++k) s += part[k * n + i];
    dW[i] = s;
}

size_t router_linear_bwd_bytes(int64_t tokens, int D, int E) { return (size_t)linear_slices(tokens) * E * D * sizeof(float); }

template <typename T>
static swimba_status linear_bwd(int64_t tokens, int D, int E, const void *u, const void *Wg, const void *dl, const void *du_add,
                                void *du, float *dW, float *part, hipStream_t st)
{
    const unsigned cols = (unsigned)((D + 255) / 256);
    const int slices = (int)linear_slices(tokens);
    if (du && tokens > 0) {
        hipLaunchKernelGGL(linear_du_kernel<T>, dim3(cols, (unsigned)(tokens < 65535 ? tokens : 65535), (unsigned)((tokens + 65534) / 65535)),
                           dim3(256), 0, st, (const T *)Wg, (const T *)dl, (const T *)du_add, (T *)du, tokens, D, E);
        SWIMBA_CHECK_LAUNCH();
    }
    if (dW) {
        if (slices > 0) {
            hipLaunchKernelGGL(linear_dw_kernel<T>, dim3(cols, (unsigned)E, (unsigned)slices), dim3(256), 0, st, (const T *)u,
                               (const T *)dl, part, tokens, D, E);
            SWIMBA_CHECK_LAUNCH();
        }
        const int64_t n = (int64_t)E * D;
        hipLaunchKernelGGL(linear_reduce_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, part, slices, n, dW);
        SWIMBA_CHECK_LAUNCH();
    }
    return SWIMBA_OK;
}

swimba_status launch_router_linear_bwd(int64_t tokens, int D, int E, int io_dtype, const void *u, const void *Wg, const void *dl,
                                       const void *du_add, void *du, float *dW, void *part, hipStream_t st)
{
    return (io_dtype == SWIMBA_BF16 ? linear_bwd<bf16> : linear_bwd<float>)(tokens, D, E, u, Wg, dl, du_add, du, dW, (float *)part, st);
}

}  // namespace swimba
