// Training the router: routing with per-expert counts and a balance loss, and the gradient of the logits.
//   balance   pi = softmax(logits), K = top-k;  counts[e] = #{t : e in K_t}, P[e] = mean_t pi_t[e],  loss = E sum_e f_e P_e with
//             f_e = counts[e] / (k n), over the n tokens of a group that count
//   logits    g_t[e] = [e in K_t] dw + d_loss (E / n) f_e,   d_logits = pi (g - <pi, g>)
// A token lies in G lanes, eight consecutive experts to a lane: one 16-byte piece of a bf16 row, so that a wave's loads are
// contiguous where the experts fill the lanes.
#include "rows.hpp"

namespace swimba {

constexpr int RT_MOST = 1024;              // threads of the largest block

// Order of logits as unsigned numbers: -0 as +0, NaN outside the numbers by sign.
__device__ __forceinline__ uint32_t order_of(float f)
{
    const uint32_t u = __float_as_uint(f + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_order(uint32_t s) { return __uint_as_float(s & 0x80000000u ? s ^ 0x80000000u : ~s); }

// One token in G lanes.  Keys are larger the earlier an expert is picked, and 0 past the last expert; bf16 logits leave room for
// the expert in the lower half, so that their keys are all different and carry it.
template <typename T, int G> struct Token {
    static constexpr bool PACKED = sizeof(T) == 2;
    static constexpr int ROUNDS = 8 * G < SWIMBA_MAX_TOPK ? 8 * G : SWIMBA_MAX_TOPK, SLOTS = (ROUNDS + G - 1) / G;
    float f[8];
    uint32_t key[8];
    __device__ __forceinline__ void take(const Piece<T, 8> &p, int l, int E)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = p.get(j);
            const uint32_t s = order_of(f[j]);
            key[j] = 8 * l + j >= E ? 0 : PACKED ? (s & 0xffff0000u) | (uint32_t)(0xffff - 8 * l - j) : s > 1 ? s : 1;
        }
    }
    static __device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
    static __device__ __forceinline__ uint32_t umin(uint32_t a, uint32_t b) { return a < b ? a : b; }
    __device__ __forceinline__ uint32_t first() const
    {
        uint32_t b = key[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) b = umax(b, key[j]);
        return over_group<G>(b, umax);
    }
    // largest key below `best`: at the smallest distance under it, those at and above it being far away
    __device__ __forceinline__ uint32_t next(uint32_t best) const
    {
        uint32_t d = best - 1 - key[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) d = umin(d, best - 1 - key[j]);
        return best - 1 - over_group<G>(d, umin);
    }
    // lowest expert behind `after` with this key; a number past all experts where there is none
    __device__ __forceinline__ int holder(uint32_t best, int after, int l) const
    {
        uint32_t e = 1 << 20;
#pragma unroll
        for (int j = 7; j >= 0; --j)
            if (key[j] == best && 8 * l + j > after) e = 8 * l + j;
        return (int)over_group<G>(e, umin);
    }
    static __device__ __forceinline__ float value(uint32_t k)
    {
        return PACKED ? __uint_as_float(__float_as_uint(of_order(k)) & 0xffff0000u) : of_order(k);
    }

    // The K picks: lane l keeps those of rounds l, l + G, ... in (e, k); bit j of the result: the lane's expert j is one of them.
    __device__ __forceinline__ uint32_t picks(uint32_t best, int K, int l, int (&e)[SLOTS], uint32_t (&k)[SLOTS]) const
    {
        uint32_t b = best;
        bool falls = true;
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            if (r < K) {
                if (r) {
                    const uint32_t n = next(b);
                    falls = falls && n < b;
                    b = n;
                }
                const int x = PACKED ? (int)(0xffff - (b & 0xffff)) : holder(b, -1, l);
                if (l == r % G) { e[r / G] = x; k[r / G] = b; }
            }
        }
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) bits |= key[j] >= b ? 1u << j : 0u;
        if constexpr (!PACKED) {
            // equal logits among the picks: more than K keys reach the last, or the keys ran out
            const int reach = (int)over_group<G>(__popc(bits), [](uint32_t p, uint32_t q) { return p + q; });
            if (__any(reach != K || !falls)) {
                b = best;
                bits = 0;
                int x = holder(b, -1, l);
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) {
                    if (r < K) {
                        if (r) {
                            const int same = holder(b, x, l);
                            const uint32_t n = next(b);
                            const int other = holder(n, -1, l);
                            if (same < 8 * G) x = same;
                            else { b = n; x = other; }
                        }
                        if (l == r % G) { e[r / G] = x; k[r / G] = b; }
                        if (x / 8 == l) bits |= 1u << x % 8;
                    }
                }
            }
        }
        return bits;
    }
};

// loss of a group from the sums of its probabilities and its counts, which the threads below E hold
__device__ __forceinline__ void balance_finish(float p, int c, int64_t grp, int E, int K, int32_t *counts, float *prob_mean,
                                               float *loss, double (*lds)[4])
{
    // E <= 256: four waves hold the experts
    const int e = threadIdx.x;
    auto total = [&](double v, int row) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
        if (e < 256 && (e & 63) == 0) lds[row][e >> 6] = v;
        __syncthreads();
        return lds[row][0] + lds[row][1] + lds[row][2] + lds[row][3];
    };
    const double all = total(e < E ? (double)c : 0., 0);       // k n
    const float mean = all > 0. ? (float)((double)p * K / all) : 0.f;
    const double l = total(e < E && all > 0. ? (double)c / all * mean : 0., 1);
    if (e < E) {
        counts[grp * E + e] = c;
        if (prob_mean) prob_mean[grp * E + e] = mean;
    }
    if (e == 0) loss[grp] = (float)(E * l);
}

// A block walks its slice of a group's tokens; part (groups, slices, E): {sum of probabilities, count}.  With one slice to a
// group the block has all of it and finishes the loss itself.
template <typename T, int G, bool TAIL>
__global__ void __launch_bounds__(RT_MOST)
balance_kernel(const T *__restrict__ logits, const uint8_t *__restrict__ mask, int32_t *__restrict__ topk_idx,
               float *__restrict__ topk_w, float2 *__restrict__ part, int64_t tokens, int slices, int E, int K,
               int32_t *__restrict__ counts, float *__restrict__ prob_mean, float *__restrict__ loss)
{
    __shared__ float psum[RT_MOST / 64][8 * G];
    __shared__ int csum[RT_MOST / 64][8 * G];
    __shared__ double fin[2][4];
    const int64_t grp = blockIdx.x / slices;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane % G, at = lane / G;
    const int64_t stride = (int64_t)slices * (blockDim.x / G);
    const T *const z = logits + grp * tokens * E;
    float acc[8] = {};
    int cnt[8] = {};
    struct Step {
        Piece<T, 8> p;
        uint8_t on;
    };
    auto fetch = [&](Step &s, int64_t t) __attribute__((always_inline)) {        // t: first token of the wave
        const bool in = t + at < tokens;
        s.p.template load<TAIL>(z + t * E + (uint32_t)(at * E + 8 * l), in ? E - 8 * l : 0);
        s.on = in && (!mask || mask[grp * tokens + t + at]);
    };
    int64_t t = (int64_t)(blockIdx.x % slices) * (blockDim.x / G) + wave * (64 / G);
    Step next;
    if (t < tokens) fetch(next, t);
    for (; t < tokens; t += stride) {
        const Step s = next;
        if (t + stride < tokens) fetch(next, t + stride);
        Token<T, G> tok;
        tok.take(s.p, l, E);
        const uint32_t best = tok.first();
        int e[Token<T, G>::SLOTS];
        uint32_t k[Token<T, G>::SLOTS];
        const uint32_t bits = tok.picks(best, K, l, e, k);
        const float m = tok.value(best);
        bool on = s.on;
        if (__any(m == -INFINITY)) {                           // a token without a logit above it counts nothing
            uint32_t some = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) some |= 8 * l + j < E && tok.f[j] != -INFINITY;
            on = on && over_group<G>(some, [](uint32_t a, uint32_t b) { return a | b; });
        }
        float p[8], Z = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p[j] = 8 * l + j < E ? route_exp(tok.f[j] - m) : 0.f;
            Z += p[j];
        }
        const float invZ = 1.0f / group_sum<G>(Z);
        if (t + at < tokens) {
            const int64_t row = (grp * tokens + t + at) * K;
#pragma unroll
            for (int i = 0; i < Token<T, G>::SLOTS; ++i) {
                const int r = i * G + l;
                if (r < K) {
                    if (topk_idx) topk_idx[row + r] = e[i];
                    if (topk_w) topk_w[row + r] = route_exp(tok.value(k[i]) - m) * invZ;
                }
            }
        }
        if (on) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                acc[j] += p[j] * invZ;
                cnt[j] += bits >> j & 1;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float v = __uint_as_float(over_lanes<G, 64>(__float_as_uint(acc[j]), add_f32));
        const int c = (int)over_lanes<G, 64>((uint32_t)cnt[j], [](uint32_t a, uint32_t b) { return a + b; });
        if (lane < G) { psum[wave][8 * l + j] = v; csum[wave][8 * l + j] = c; }
    }
    __syncthreads();
    const int x = threadIdx.x;
    float v = 0.f;
    int c = 0;
    if (x < E)
        for (int w = 0; w < (int)blockDim.x / 64; ++w) { v += psum[w][x]; c += csum[w][x]; }
    if (slices == 1) balance_finish(v, c, grp, E, K, counts, prob_mean, loss, fin);
    else if (x < E) part[(int64_t)blockIdx.x * E + x] = make_float2(v, __int_as_float(c));
}

// the slices joined, each thread every (1024 / width)-th of an expert
__global__ void __launch_bounds__(1024)
balance_loss_kernel(const float2 *__restrict__ part, int slices, int width, int E, int K, int32_t *__restrict__ counts,
                    float *__restrict__ prob_mean, float *__restrict__ loss)
{
    __shared__ float2 lds[1024];
    __shared__ double fin[2][4];
    const int64_t grp = blockIdx.x;
    const int e = threadIdx.x % width, n = 1024 / width;
    int c = 0;
    float p = 0.f;
    if (e < E) {
#pragma unroll 8
        for (int s = threadIdx.x / width; s < slices; s += n) {
            const float2 v = part[(grp * slices + s) * E + e];
            p += v.x;
            c += __float_as_int(v.y);
        }
    }
    lds[threadIdx.x] = make_float2(p, __int_as_float(c));
    __syncthreads();
    p = 0.f;
    c = 0;
    if (threadIdx.x < width)
        for (int i = 0; i < n; ++i) {
            p += lds[i * width + e].x;
            c += __float_as_int(lds[i * width + e].y);
        }
    balance_finish(p, c, grp, E, K, counts, prob_mean, loss, fin);
}

namespace {

int lanes_of(int E)                        // of a token
{
    int g = 1;
    while (8 * g < E) g *= 2;
    return g;
}

// Threads of a block and slices of a group.  A group that a block of 1024 threads walks in four steps or less stays with one
// block, without a second launch; beyond, a slice is a step or more, and the slices of all groups are some 256 (a few more
// where groups are many), which fill the chip with waves and are soon added up.
struct Slices { int threads; int64_t count; };
Slices balance_slices(int64_t groups, int64_t tokens, int E)
{
    const int64_t threads = tokens * lanes_of(E), steps = (threads + RT_MOST - 1) / RT_MOST;
    if (steps <= 4 || groups >= 256) {
        int n = 256;
        while (n < RT_MOST && n < threads) n *= 2;
        return {n, 1};
    }
    const int64_t most = 256 / groups + 1;
    return {RT_MOST, steps < most ? steps : most};
}

template <typename F>
void with_lanes(int E, F &&f)
{
    using std::integral_constant;
    auto tail = [&](auto g) {
        if (E % 8) f(g, std::true_type());
        else f(g, std::false_type());
    };
    switch (lanes_of(E)) {
    case 1: return tail(integral_constant<int, 1>());
    case 2: return tail(integral_constant<int, 2>());
    case 4: return tail(integral_constant<int, 4>());
    case 8: return tail(integral_constant<int, 8>());
    case 16: return tail(integral_constant<int, 16>());
    default: return tail(integral_constant<int, 32>());
    }
}

}  // namespace

size_t balance_bytes(int64_t groups, int64_t tokens, int E)
{
    const int64_t n = balance_slices(groups, tokens, E).count;
    return n > 1 ? (size_t)groups * n * E * sizeof(float2) : 0;
}

swimba_status launch_router_balance(int64_t groups, int64_t tokens, int E, int K, int io_dtype, const void *logits,
                                    const uint8_t *mask, int32_t *topk_idx, float *topk_w, int32_t *counts, float *prob_mean,
                                    float *loss, void *part, hipStream_t st)
{
    if (groups == 0) return SWIMBA_OK;
    const Slices s = balance_slices(groups, tokens, E);
    with_lanes(E, [&](auto g, auto tail) {
        auto go = [&](auto kernel, auto *z) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(groups * s.count)), dim3(s.threads), 0, st, z, mask, topk_idx, topk_w, (float2 *)part,
                               tokens, (int)s.count, E, K, counts, prob_mean, loss);
        };
        if (io_dtype == SWIMBA_BF16) go(balance_kernel<bf16, g(), tail()>, (const bf16 *)logits);
        else go(balance_kernel<float, g(), tail()>, (const float *)logits);
    });
    SWIMBA_CHECK_LAUNCH();
    if (s.count > 1) {
        int width = 1;
        while (width < E) width *= 2;
        hipLaunchKernelGGL(balance_loss_kernel, dim3((unsigned)groups), dim3(1024), 0, st, (const float2 *)part, (int)s.count, width, E, K,
                           counts, prob_mean, loss);
        SWIMBA_CHECK_LAUNCH();
    }
    return SWIMBA_OK;
}

// The gradients of a token's routing weights are laid at their experts through LDS: a wave's 64 / G tokens are 512 floats,
// element j of lane i at 8 i + j.
template <typename T, int G, bool TAIL>
__global__ void __launch_bounds__(256)
router_bwd_kernel(const T *__restrict__ logits, const uint8_t *__restrict__ mask, const int32_t *__restrict__ topk_idx,
                  const float *__restrict__ d_topk_w, const int32_t *__restrict__ counts, const float *__restrict__ d_loss,
                  T *__restrict__ d_logits, int64_t tokens, int64_t per_group, int E, int K)
{
    constexpr int SLOTS = Token<T, G>::SLOTS;
    __shared__ float lds[4][512];
    const int64_t grp = blockIdx.x / per_group;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane % G, at = lane / G;
    float *const mine = lds[wave] + 8 * lane, *const token = lds[wave] + 8 * (lane - l);
    float share[8] = {};                                        // d_loss (E / n) f_e
    if (counts) {
        double all = 0.;
        int c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            c[j] = 8 * l + j < E ? counts[grp * E + 8 * l + j] : 0;
            all += c[j];
        }
#pragma unroll
        for (int o = 1; o < G; o *= 2) all += __shfl_xor(all, o);
        const double scale = all > 0. ? (double)d_loss[grp] * E * K / all : 0.;
#pragma unroll
        for (int j = 0; j < 8; ++j) share[j] = all > 0. ? (float)(scale * (c[j] / all)) : 0.f;
    }
    const T *const z = logits + grp * tokens * E;
    T *const out = d_logits + grp * tokens * E;
    const int64_t stride = per_group * (256 / G);
    struct Step {
        Piece<T, 8> p;
        float dw[SLOTS];
        int e[SLOTS];
        uint8_t on;
    };
    auto fetch = [&](Step &s, int64_t t) __attribute__((always_inline)) {
        const bool in = t + at < tokens;
        const int64_t row = grp * tokens + t + at;
        s.p.template load<TAIL>(z + t * E + (uint32_t)(at * E + 8 * l), in ? E - 8 * l : 0);
        s.on = in && counts && (!mask || mask[row]);
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            const int r = i * G + l;
            s.e[i] = -1;
            s.dw[i] = 0.f;
            if (d_topk_w && in && r < K) {
                s.e[i] = topk_idx[row * K + r];
                s.dw[i] = d_topk_w[row * K + r];
            }
        }
    };
    int64_t t = (blockIdx.x % per_group) * (256 / G) + wave * (64 / G);
    Step next;
    if (t < tokens) fetch(next, t);
    for (; t < tokens; t += stride) {
        const Step s = next;
        if (t + stride < tokens) fetch(next, t + stride);
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = s.on ? share[j] : 0.f;
        uint32_t some = s.on;                                   // whether the token has a gradient at all
        if (d_topk_w) {
#pragma unroll
            for (int j = 0; j < 8; ++j) mine[j] = g[j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                some |= s.dw[i] != 0.f;
                if ((uint32_t)s.e[i] < (uint32_t)E) atomicAdd(token + s.e[i], s.dw[i]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = mine[j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        float f[8], m = -INFINITY;
        uint32_t any = 0;                                       // whether it has a logit above -inf
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] = 8 * l + j < E ? s.p.get(j) : -INFINITY;
            m = fmaxf(m, f[j]);
            any |= f[j] != -INFINITY;
        }
        m = __uint_as_float(over_group<G>(__float_as_uint(m), [](uint32_t a, uint32_t b) {
            return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
        }));
        const uint32_t both = over_group<G>(any | some << 1, [](uint32_t a, uint32_t b) { return a | b; });
        float p[8], Z = 0.f, dot = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p[j] = 8 * l + j < E ? route_exp(f[j] - m) : 0.f;
            Z += p[j];
            dot += 8 * l + j < E ? p[j] * g[j] : 0.f;
        }
        const float invZ = 1.0f / group_sum<G>(Z);
        dot = group_sum<G>(dot) * invZ;
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = both == 3 ? p[j] * invZ * (g[j] - dot) : 0.f;
        if (t + at < tokens) store_piece<TAIL>(out + t * E + (uint32_t)(at * E + 8 * l), p, E - 8 * l);
    }
}

swimba_status launch_router_bwd(int64_t groups, int64_t tokens, int E, int K, int io_dtype, const void *logits, const uint8_t *mask,
                                const int32_t *topk_idx, const float *d_topk_w, const int32_t *counts, const float *d_loss,
                                void *d_logits, hipStream_t st)
{
    if (groups == 0 || tokens == 0) return SWIMBA_OK;
    const int64_t need = (tokens * lanes_of(E) + 255) / 256, fit = groups < 2048 ? 2048 / groups : 1, per_group = need < fit ? need : fit;
    with_lanes(E, [&](auto g, auto tail) {
        auto go = [&](auto kernel, auto *z, auto *out) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(groups * per_group)), dim3(256), 0, st, z, mask, topk_idx, d_topk_w, counts, d_loss, out,
                               tokens, per_group, E, K);
        };
        if (io_dtype == SWIMBA_BF16) go(router_bwd_kernel<bf16, g(), tail()>, (const bf16 *)logits, (bf16 *)d_logits);
        else go(router_bwd_kernel<float, g(), tail()>, (const float *)logits, (float *)d_logits);
    });
    SWIMBA_CHECK_LAUNCH();
    return SWIMBA_OK;
}

}  // namespace swimba
