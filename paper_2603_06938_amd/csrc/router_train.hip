// Training the router: routing with per-expert counts and a balance loss, and the gradient of the logits.
//   balance   pi = softmax(logits), K = top-k;  counts[e] = #{t : e in K_t}, P[e] = mean_t pi_t[e],  loss = E sum_e f_e P_e with
//             f_e = counts[e] / (k n), over the n tokens of a group that count
//   logits    g_t[e] = [e in K_t] dw + d_loss (E / n) f_e,   d_logits = pi (g - <pi, g>)
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

}  // namespace swimba
